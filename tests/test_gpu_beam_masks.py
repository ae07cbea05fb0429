"""Selections whose logits are masked by finite values, with more sets of tokens within a rounding of each other than are looked at together."""
import pytest
import torch

import continuations_plain as plain

pytestmark = pytest.mark.gpu


def masked(rows, vocab, allowed, mask, seed):
    g = torch.Generator().manual_seed(seed)
    x, at = 2.5 * torch.randn(rows, vocab, generator=g), torch.randint(0, vocab, (rows, allowed), generator=g)
    return torch.full((rows, vocab), mask).scatter(1, at, x.gather(1, at)), -torch.rand(rows, generator=g)


@pytest.mark.parametrize("mask", [-1e9, -1e4, float(torch.finfo(torch.float32).min) / 2])
@pytest.mark.parametrize("groups,beams,vocab,k", [(2, 8, 40000, 32), (1, 4, 128256, 12), (1, 4, 128256, 33), (3, 64, 2000, 64), (1, 1, 300000, 17)])
@pytest.mark.parametrize("allowed", [1, 5, 60])
def test_candidates_behind_the_allowed_tokens(groups, beams, vocab, k, allowed, mask):
    from paper_2502_09922_amd import beam_select

    x, scores = masked(groups * beams, vocab, allowed, mask, vocab + allowed)
    ended = (torch.arange(groups * beams) % 5 == 4).int()
    for e in (None, ended):
        got = [t.cpu() for t in beam_select(x.cuda(), scores.cuda(), beams=beams, k=k, ended=None if e is None else e.cuda(), eos=vocab // 3)]
        want = plain.select(x, scores, e, beams, k, vocab // 3)
        # what is allowed, and beams that have ended, stand in front: scores far apart next to the sums' 32 bits, but for two beams' that meet
        same = (got[0] == want[0]) & (got[1] == want[1])
        assert ((got[2].double() - want[2]).abs() <= 2.0**-18 + 2.0**-23 * want[2].abs()).all()
        # behind them equal logits, a beam's in the order of their tokens: (mask - largest logit) rounds in 64 bits where it is 2^53 and more of it
        assert same[want[2] > -1e3].float().mean() > 0.99
        for g in range(groups):
            rest = got[2][g].double() < -1e3
            for row in set(got[0][g][rest].tolist()):
                tokens = got[1][g][rest & (got[0][g] == row)].tolist()
                free = [t for t in range(vocab) if x[row, t] == mask][: len(tokens)]
                assert tokens == free, (g, row)


def test_masks_cost_little():
    from paper_2502_09922_amd import beam_select

    x, scores = masked(64, 128256, 5, -1e9, 1)
    plainly = 2.5 * torch.randn(64, 128256, generator=torch.Generator().manual_seed(2))

    def fastest(logits):
        logits, s, times = logits.cuda(), scores.cuda(), []
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(5):
                beam_select(logits, s, beams=8, k=32)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    fastest(x)
    masks, none = fastest(x), fastest(plainly)
    assert masks <= 4 * none  # 20 times where candidates are taken one after the other
