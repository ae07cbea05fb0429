"""Beam selection and cache reordering (ls_beam_select, ls_kv_reorder) against plain 64-bit arithmetic."""
import math

import pytest
import torch

import continuations_plain as plain

pytestmark = pytest.mark.gpu


def check(logits, scores, beams, k, ended=None, eos=0):
    from paper_2502_09922_amd import beam_select

    got = beam_select(logits.cuda(), scores.cuda(), beams=beams, k=k, ended=None if ended is None else ended.cuda(), eos=eos)
    rows, tokens, best = (t.cpu() for t in got)
    want = plain.select(logits, scores, ended, beams, k, eos)
    assert torch.equal(rows.long(), want[0]) and torch.equal(tokens.long(), want[1])
    # fp32 exponentials of exponents rounded in 32 bits (of size up to 100: 100 2^-24 of an addend that counts exp(-100)), the rest in 64
    inf = want[2].isinf()
    assert torch.equal(best.double()[inf], want[2][inf])
    assert ((best.double() - want[2])[~inf].abs() <= 2.0**-24 * want[2][~inf].abs() + 2.0**-21).all()


@pytest.mark.parametrize("groups,beams,vocab,k", [(1, 1, 1, 1), (1, 1, 5, 5), (3, 2, 3, 6), (1, 4, 32000, 4), (5, 3, 1001, 6), (2, 64, 700, 64), (7, 5, 4099, 10),
                                                  (2, 1, 63, 63), (40, 4, 2050, 8), (1, 8, 50257, 16), (1, 2, 131072, 64)])
def test_select(groups, beams, vocab, k):
    g = torch.Generator().manual_seed(vocab + k)
    logits = 2.5 * torch.randn(groups * beams, vocab, generator=g)
    scores = -(3 * torch.randn(groups * beams, generator=g)).abs()
    check(logits, scores, beams, k)
    ended = (torch.rand(groups * beams, generator=g) < 0.4).int()
    check(logits, scores, beams, k, ended, eos=vocab // 2)


@pytest.mark.parametrize("vocab", [7, 1000, 9001])
def test_equal_candidates_go_by_their_index(vocab):
    """Logits of a few values, beams that are copies of each other (the same bits, so the same sums), and no differences at all."""
    g = torch.Generator().manual_seed(vocab)
    logits = torch.randint(-2, 3, (1, vocab), generator=g).float().repeat(6, 1)
    check(logits, torch.tensor([-1.0, -1.0, -1.0, -2.0, -2.0, -1.0]), 3, 7)
    check(torch.zeros(4, vocab), torch.zeros(4), 2, min(14, 2 * vocab))


@pytest.mark.parametrize("vocab", [5, 2000])
def test_dead_beams_masked_tokens_and_nonfinite_logits(vocab):
    g = torch.Generator().manual_seed(vocab)
    logits = torch.randn(12, vocab, generator=g)
    scores = -torch.rand(12, generator=g)
    scores[1] = -math.inf            # a beam that is not there yet
    logits[2] = -math.inf            # everything masked
    logits[3, 1:] = -math.inf        # one token allowed
    logits[4, 2] = math.inf
    logits[5, 3] = math.nan
    logits[8:12] = -math.inf         # a request with nothing left
    scores[9] = math.nan
    logits[0] = torch.finfo(torch.float32).min  # masked by the type's lowest value: all alike
    check(logits, scores, 4, 8)
    check(logits, scores, 4, 3)
    check(logits, scores, 2, 9 if vocab > 5 else 10)


def test_select_captured_and_replayed():
    from paper_2502_09922_amd import beam_select

    logits, scores = torch.empty(8, 5003, device="cuda"), torch.empty(8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    logits.zero_(), scores.zero_()
    beam_select(logits, scores, beams=4, k=4)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rows, tokens, best = beam_select(logits, scores, beams=4, k=4)
    for seed in (1, 2, 3):
        g = torch.Generator().manual_seed(seed)
        x, s = torch.randn(8, 5003, generator=g), torch.randn(8, generator=g)
        logits.copy_(x), scores.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        want = plain.select(x, s, None, 4, 4, 0)
        assert torch.equal(rows.cpu().long(), want[0]) and torch.equal(tokens.cpu().long(), want[1])
        check(x, s, 2, 5)


@pytest.mark.parametrize("heads,dtype", [((4, 64), torch.bfloat16), ((3, 128), torch.float32), ((2, 6), torch.bfloat16), ((2, 80), torch.bfloat16)],
                         ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else "")
@pytest.mark.parametrize("group", [1, 2, 3, 4, 5, 8, 9, 16, 24, 40, 64])
def test_reorder(heads, dtype, group):
    """Sources that repeat, rotate or stay, lengths and shared prefixes of their own, sources outside the group."""
    from paper_2502_09922_amd import kv_reorder

    hkv, hd = heads
    layers, groups, S = 2, 3, 50
    g = torch.Generator().manual_seed(group)
    B = groups * group
    k, v = (torch.randn(layers, B + 1, hkv, S, hd, generator=g).to(dtype) for _ in range(2))
    lens = torch.randint(0, S + 1, (B + 1,), generator=g).int()
    first = torch.randint(0, 20, (B,), generator=g).int()
    src = torch.randint(0, group, (B,), generator=g).int() + torch.arange(B).int() // group * group
    src[:group] = (torch.arange(group) + 1) % group  # a rotation
    src[-1] = -3
    if B > group:
        src[group] = 0
    for f in (first, None):
        gk, gv, gl = k.cuda(), v.cuda(), lens.cuda()
        kv_reorder(src.cuda(), group, gk, gv, gl, max_ctx=45, first=None if f is None else f.cuda())
        wk, wv, wl = k.clone(), v.clone(), lens.clone()
        for b in range(B):
            s = int(src[b])
            if s // group != b // group or s < 0:
                continue
            at = slice(int(f[b]) if f is not None else 0, min(45, int(lens[s])))
            if group > 1 and s != b and at.start < at.stop:
                wk[:, b, :, at], wv[:, b, :, at] = k[:, s, :, at], v[:, s, :, at]
            wl[b] = lens[s]
        # positions behind max_ctx may move or not
        assert torch.equal(gk.cpu()[..., :45, :], wk[..., :45, :]) and torch.equal(gv.cpu()[..., :45, :], wv[..., :45, :]) and torch.equal(gl.cpu(), wl)


@pytest.mark.parametrize("beams,vocab,k", [(1, 40000, 64), (8, 9001, 40), (64, 300, 64), (64, 4000, 50)])
def test_the_best_lie_side_by_side(beams, vocab, k):
    """Logits that fall along the vocabulary, and all alike: the best candidates, or as good ones, are many in few places."""
    fall = -torch.arange(vocab).float() / 1000
    check(fall.repeat(beams, 1), -torch.arange(beams).float() / 1e5, beams, k)
    check(torch.zeros(beams, vocab), torch.zeros(beams), beams, k)
    check(torch.full((beams, vocab), -math.inf), torch.zeros(beams), beams, k)


def test_reorder_captured_and_replayed():
    from paper_2502_09922_amd import kv_reorder

    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(2, 8, 2, 40, 64, generator=g).bfloat16() for _ in range(2))
    gk, gv = k.cuda(), v.cuda()
    src, lens = torch.arange(8, dtype=torch.int32).cuda(), torch.full((8,), 33, dtype=torch.int32).cuda()
    kv_reorder(src, 4, gk, gv, lens, max_ctx=40)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kv_reorder(src, 4, gk, gv, lens, max_ctx=40)
    assert torch.equal(gk.cpu(), k)
    n = torch.full((8,), 33, dtype=torch.int32)
    for moves in ([1, 2, 3, 0, 4, 4, 4, 5], [0, 0, 0, 0, 7, 6, 5, 4], [3, 3, 1, 2, 4, 5, 6, 7]):
        src.copy_(torch.tensor(moves, dtype=torch.int32))
        lens[7] = 20 + moves[0]
        n[7] = 20 + moves[0]
        graph.replay()
        torch.cuda.synchronize()
        old = k.clone(), v.clone()
        for b, s in enumerate(moves):
            k[:, b, :, : n[s]], v[:, b, :, : n[s]] = old[0][:, s, :, : n[s]], old[1][:, s, :, : n[s]]
        n = n[moves]
        assert torch.equal(gk.cpu(), k) and torch.equal(gv.cpu(), v) and torch.equal(lens.cpu(), n)


def test_calls_on_streams_of_their_own():
    """Selections and reorderings on two streams at once, each behind the work that makes its inputs."""
    from paper_2502_09922_amd import beam_select, kv_reorder

    sides, runs = [torch.cuda.Stream() for _ in range(2)], []
    for i in range(6):
        g = torch.Generator().manual_seed(i)
        logits, scores = torch.randn(12, 20011, generator=g), torch.randn(12, generator=g)
        k = torch.randn(1, 12, 2, 30, 64, generator=g)
        want = beam_select(logits.cuda(), scores.cuda(), beams=4, k=4)
        torch.cuda.synchronize()
        with torch.cuda.stream(sides[i % 2]):
            a, gk = logits.cuda() * 1, k.cuda() * 1
            got = beam_select(a, scores.cuda(), beams=4, k=4)
            gv, lens = gk.clone(), torch.full((12,), 30, dtype=torch.int32, device="cuda")
            kv_reorder(got[0].view(-1), 4, gk, gv, lens, max_ctx=30)
            runs.append((want, got, k, gk, gv))
    for s in sides:
        s.synchronize()
    for want, got, k, gk, gv in runs:
        assert all(torch.equal(x, y) for x, y in zip(want, got))
        moved = k[:, want[0].view(-1).long().cpu()]
        assert torch.equal(gk.cpu(), moved) and torch.equal(gv.cpu(), moved)


@pytest.mark.parametrize("vocab", [16, 1023, 8200, 33000])
@pytest.mark.parametrize("k", [1, 15, 16, 17])
def test_sets_of_one_thread_and_of_four(k, vocab):
    """Up to 16 candidates and more, whose sets of tokens differ; equal logits within and across sets; the end token anywhere."""
    from paper_2502_09922_amd import beam_select

    g = torch.Generator().manual_seed(vocab + k)
    for i in range(6):
        logits = torch.randn(12, vocab, generator=g) * 3
        logits = logits.round() if i % 2 else logits
        scores, ended = -torch.rand(12, generator=g), (torch.rand(12, generator=g) < 0.25).int()
        eos = int(torch.randint(vocab, (1,), generator=g))
        got = [t.cpu() for t in beam_select(logits.cuda(), scores.cuda(), beams=6, k=k, ended=ended.cuda(), eos=eos)]
        want = plain.select(logits, scores, ended, 6, k, eos)
        assert torch.equal(got[0], want[0].int()) and torch.equal(got[1], want[1].int())
        # the sum: 32 terms, each off by 2^-22 (difference, product, exponential), added in 32 bits; its logarithm; the output's rounding
        assert ((got[2].double() - want[2]).abs() <= 2.0**-18 + 2.0**-23 * want[2].abs()).all()
