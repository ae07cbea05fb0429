"""Draft trees and beams through a stage: the pass over a tree's nodes against the oracle's prompt passes over their paths, and
the whole loops: drafts that are checked, accepted and kept step after step say what plain generation says, and beams that are
selected and reordered are those of an exhaustive search with prompt passes."""
import random

import numpy as np
import pytest
import torch

import continuations_plain as plain
import synth
from helpers import check_close, make_gpu, make_oracle, to_dev, to_host

pytestmark = pytest.mark.gpu

F32 = synth.CONFIGS["tiny_f32"]
BF16 = synth.StageShape("bf16", 2, 512, 8, 2, 128, 1408, 1000)
GENERIC = synth.StageShape("f32", 2, 96, 4, 2, 24, 160, 77)  # no kernel but those for every shape
WIDE = synth.StageShape("bf16", 2, 256, 2, 2, 64, 512, 301)  # logits of an odd width


def bounds(trees):
    cu = np.cumsum([0] + [len(t) for t in trees]).astype(np.int32)
    return torch.tensor([p for t in trees for p in t], dtype=torch.int32).cuda(), torch.from_numpy(cu).cuda(), cu


@pytest.mark.parametrize("shape", [F32, BF16, GENERIC, WIDE], ids=["f32", "bf16", "generic", "wide"])
@pytest.mark.parametrize("nodes", [[1, 3], [7, 0, 12], [40, 64, 5]], ids=str)
def test_tree_pass_equals_prompt_passes_over_paths(shape, nodes):
    r = random.Random(sum(nodes))
    lengths = [9, 30, 14][: len(nodes)]
    trees = [plain.random_tree(r, n) if n else [] for n in nodes]
    st = make_gpu(shape, 3, 0, 2, 3, 110, 120)
    prompts = [synth.token_ids(20 + b, n, shape.vocab) for b, n in enumerate(lengths)]
    st.prefill(to_dev(shape, np.concatenate(prompts)), lengths)
    tokens = [synth.token_ids(30 + b, len(t), shape.vocab) if t else np.zeros(0, np.int32) for b, t in enumerate(trees)]
    k0, v0 = (c.clone() for c in st.caches())
    parents, cu, host = bounds(trees)
    feed = torch.from_numpy(np.concatenate(tokens)).cuda()
    said, logits = st.tree(feed, parents, cu, host, max(lengths), want_logits=True)
    alone = st.tree(feed, parents, cu, host, max(lengths))  # logits in the workspace, max_batch rows at a time
    torch.cuda.synchronize()
    assert torch.equal(st.seq_lens[: len(nodes)].cpu(), torch.tensor(lengths, dtype=torch.int32))
    for b, n in enumerate(lengths):  # cached positions and what lies behind the trees
        for c, c0 in zip(st.caches(), (k0, v0)):
            assert torch.equal(c[:, b, :, :n], c0[:, b, :, :n]) and torch.equal(c[:, b, :, n + nodes[b] :], c0[:, b, :, n + nodes[b] :])
    paths = [(b, plain.path(t, i)) for b, t in enumerate(trees) for i in range(len(t))]
    seqs = [np.concatenate([prompts[b], tokens[b][p]]) for b, p in paths]
    ora = make_oracle(shape, 3, 0, 2, len(seqs), 110)
    want_said, want = ora.prefill(np.concatenate(seqs), [len(s) for s in seqs])
    check_close(to_host(logits), want, shape.dtype, "tree %s %s" % (shape.dtype, nodes))
    if shape.dtype == "f32":
        assert said.cpu().tolist() == list(want_said)
    assert torch.equal(said, logits.argmax(1).int())
    # other numbers of rows may take other GEMM kernels: tokens agree but where two logits are next to each other
    assert (alone != said).float().mean() <= (0 if shape.dtype == "f32" else 0.1)
    st.close()


ODD = synth.StageShape("bf16", 2, 160, 3, 1, 80, 224, 301)  # heads that only the kernels for every shape take


@pytest.mark.parametrize("shape", [BF16, WIDE, ODD], ids=["bf16", "wide", "odd"])
@pytest.mark.parametrize("lo,hi", [(0, 2), (0, 1), (1, 2)], ids=str)
@pytest.mark.parametrize("nodes", [[1], [3], [0, 2, 1], [9, 3, 4]], ids=str)
def test_passes_of_few_rows(shape, lo, hi, nodes):
    """Stages with or without embedding and head, whose rows are few enough for norms inside the GEMMs: the rows that a stage has
    to say, with logits and without, and each sequence's chain of the deepest node against generation steps along it."""
    r = random.Random(sum(nodes))
    lengths = [9, 30, 14][: len(nodes)]
    trees = [plain.random_tree(r, n) if n else [] for n in nodes]
    outs = []
    for steps in (False, True):
        st = make_gpu(shape, 3, lo, hi, 3, 60, 60)
        g = torch.Generator().manual_seed(1)
        rows = lambda n: (torch.randint(0, shape.vocab, (n,), dtype=torch.int32, generator=g).cuda() if lo == 0  # noqa: E731
                          else torch.randn(n, shape.hidden, generator=g).bfloat16().cuda())
        st.prefill(rows(sum(lengths)), lengths)
        feed = rows(sum(nodes))
        parents, cu, host = bounds(trees)
        if not steps:
            out = st.tree(feed, parents, cu, host, max(lengths), want_logits=hi == 2)
            if hi == 2:
                assert torch.equal(out[0], out[1].argmax(1).int())
                alone = st.tree(feed, parents, cu, host, max(lengths))
                assert (alone != out[0]).float().mean() <= 0.1 + 1.0 / sum(nodes) * (sum(nodes) > 3)  # see above: other kernels
                out = out[1]
            assert torch.equal(st.seq_lens[: len(nodes)].cpu(), torch.tensor(lengths, dtype=torch.int32))
            outs.append(out.clone())
        else:
            paths = [max((plain.path(t, i) for i in range(len(t))), key=len, default=[]) for t in trees]
            for b, p in enumerate(paths):
                for j, node in enumerate(p):
                    st.seq_lens.copy_(torch.tensor([(n + j if i == b else n) for i, n in enumerate(lengths)] + [0] * (3 - len(lengths)), dtype=torch.int32))
                    at = int(host[b]) + node
                    got = st.decode(feed[at : at + 1].repeat(*([len(nodes)] + [1] * (feed.dim() - 1))), len(nodes), 40, want_logits=hi == 2)
                    got = got[1] if hi == 2 else got
                    check_close(to_host(got[b : b + 1]), to_host(outs[0][at : at + 1]), "bf16", "few rows")
        torch.cuda.synchronize()
        st.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_middle_stages_and_pipelines_of_them(dtype):
    """Hidden rows in and out; two stages one behind the other, each with its own cache."""
    shape = (F32 if dtype == "f32" else BF16).with_(n_layers_total=4, vocab=0)
    r, lengths = random.Random(5), [12, 25]
    trees = [plain.random_tree(r, 9), plain.random_tree(r, 30)]
    stages = [make_gpu(shape, 4, 1, 2, 2, 70, 64), make_gpu(shape, 4, 2, 3, 2, 70, 64)]
    prompt, rows = synth.hidden_states(shape, 6, sum(lengths)), synth.hidden_states(shape, 7, 39)
    x, y = to_dev(shape, prompt), to_dev(shape, rows)
    parents, cu, host = bounds(trees)
    for st in stages:
        x = st.prefill(x, lengths)
        y = st.tree(y, parents, cu, host, 25)
    ora = make_oracle(shape, 4, 1, 3, 39, 70)
    starts, seqs = np.cumsum([0] + lengths), []
    for b, t in enumerate(trees):
        for i in range(len(t)):
            seqs.append(np.concatenate([prompt[starts[b] : starts[b + 1]], rows[[host[b] + j for j in plain.path(t, i)]]]))
    want = ora.prefill(np.concatenate(seqs), [len(s) for s in seqs])
    check_close(to_host(y), want[np.cumsum([len(s) for s in seqs]) - 1], dtype, "two tree stages")
    for st in stages:
        st.close()


def generate(shape, prompt, steps):
    st = make_gpu(shape, 8, 0, 2, 1, len(prompt) + steps + 1, len(prompt))
    tok, out = st.prefill(to_dev(shape, prompt), [len(prompt)]), []
    for t in range(steps):
        out.append(int(tok))
        tok = st.decode(tok, 1, len(prompt) + t)
    k, v = (c[:, 0, :, : len(prompt) + steps].clone() for c in st.caches())
    torch.cuda.synchronize()
    st.close()
    return out, k, v


@pytest.mark.parametrize("captured", [False, True], ids=["eager", "captured"])
def test_drafted_generation_says_what_generation_says(captured):
    """Two sequences, trees of seven nodes that hold the right continuation to a random depth among wrong ones; the tree
    pass, acceptance and compaction as one captured step that is replayed with other trees, tokens and lengths."""
    from paper_2502_09922_amd import tree_accept, tree_keep

    steps, lengths = 24, [11, 18]
    prompts = [synth.token_ids(40 + b, n, F32.vocab) for b, n in enumerate(lengths)]
    plain_runs = [generate(F32, p, steps + 12) for p in prompts]
    st = make_gpu(F32, 8, 0, 2, 2, 80, 40)
    tok = st.prefill(to_dev(F32, np.concatenate(prompts)), lengths)
    got, r = [[int(t)] for t in tok.cpu()], random.Random(9)
    host = np.array([0, 7, 14], np.int32)
    cu, parents = torch.from_numpy(host).cuda(), torch.zeros(14, dtype=torch.int32).cuda()
    feed, (k, v) = torch.zeros(14, dtype=torch.int32).cuda(), st.caches()

    def step(stream=None):
        said = st.tree(feed, parents, cu, host, 70, stream=stream)
        answer = tree_accept(feed, said, parents, cu, host)
        tree_keep(answer[0], cu, host, k, v, st.seq_lens)
        return answer

    lens = st.seq_lens.clone()
    answer = step()  # a first one on what lies there, and back
    torch.cuda.synchronize()
    st.seq_lens.copy_(lens)
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            answer = step(torch.cuda.current_stream())
    while min(len(g) for g in got) <= steps:
        trees, tokens = [], []
        for b in range(2):
            right = plain_runs[b][0][len(got[b]) :]
            t, depth, toks = plain.random_tree(r, 7), [0] * 7, [got[b][-1]]
            for i in range(1, 7):
                depth[i] = depth[t[i]] + 1
                toks.append(right[depth[i] - 1] if r.random() < 0.6 else r.randrange(F32.vocab))
            trees.append(t)
            tokens.append(toks)
        parents.copy_(torch.tensor(trees[0] + trees[1], dtype=torch.int32))
        feed.copy_(torch.tensor(tokens[0] + tokens[1], dtype=torch.int32))
        if captured:
            graph.replay()
        else:
            answer = step()
        _, count, emitted, following = (t.cpu() for t in answer)
        for b in range(2):
            n = int(count[b])
            got[b] += emitted[b, :n].tolist()
            assert got[b][-1] == int(following[b])
    for b in range(2):
        assert got[b][: steps + 1] == plain_runs[b][0][: steps + 1]
        n = int(st.seq_lens[b])
        assert n == lengths[b] + len(got[b]) - 1
        n = min(n, lengths[b] + steps)
        for c, want in zip(st.caches(), plain_runs[b][1:]):
            c, want = c[:, b, :, :n].double(), want[:, :, :n].double()
            assert (c - want).norm() <= 1e-5 * want.norm()
    st.close()


def test_beam_search_through_a_stage():
    """Two requests of three beams over six steps, caches behind a shared prompt reordered in place; the reference searches with
    the oracle's prompt passes over whole sequences."""
    from paper_2502_09922_amd import beam_select, kv_reorder

    W, steps, lengths = 3, 6, [10, 13]
    prompts = [synth.token_ids(50 + b, n, F32.vocab) for b, n in enumerate(lengths)]
    st = make_gpu(F32, 8, 0, 2, 2 * W, 30, 100)
    rows = [p for p in prompts for _ in range(W)]
    _, logits = st.prefill(to_dev(F32, np.concatenate(rows)), [len(p) for p in rows], want_logits=True)
    first, (k, v) = torch.tensor([len(p) for p in rows], dtype=torch.int32).cuda(), st.caches()
    scores = torch.tensor([0.0, -np.inf, -np.inf] * 2).cuda()  # one beam to begin with
    seqs, best = [list(p) for p in rows], None
    for t in range(steps):
        src, tokens, best = beam_select(logits, scores.view(-1), beams=W, k=W)
        kv_reorder(src.view(-1), W, k, v, st.seq_lens, max_ctx=max(lengths) + t, first=first)
        scores = best
        seqs = [seqs[int(s)] + [int(x)] for s, x in zip(src.view(-1).cpu(), tokens.view(-1).cpu())]
        _, logits = st.decode(tokens.view(-1), 2 * W, max(lengths) + t, want_logits=True)
    torch.cuda.synchronize()
    ora = make_oracle(F32, 8, 0, 2, W, 30)
    for q, p in enumerate(prompts):
        beams = [(0.0, list(p))]
        for t in range(steps):
            _, lg = ora.prefill(np.concatenate([np.array(s, np.int32) for _, s in beams]), [len(s) for _, s in beams])
            lg = torch.from_numpy(np.asarray(lg))
            at = plain.select(lg, torch.tensor([b[0] for b in beams], dtype=torch.float64), None, len(beams), W, 0)
            beams = [(float(s), beams[int(b)][1] + [int(x)]) for b, x, s in zip(at[0][0], at[1][0], at[2][0])]
        assert seqs[q * W : (q + 1) * W] == [s for _, s in beams]
        # sums of steps scores, each off by the logits' error (1e-4 of their size, at most 2.5) at most twice
        assert (best[q].cpu().double() - torch.tensor([b[0] for b in beams])).abs().max() <= steps * 2 * 2.5e-4
    st.close()


def test_refusals_of_the_tree_pass():
    from paper_2502_09922_amd import LsError, binding as b

    st = make_gpu(F32, 8, 0, 2, 2, 40, 16)
    one = torch.zeros(1, dtype=torch.int32).cuda()
    for counts, ctx, status in (([9, 8], 5, b.LS_ERR_INVALID_ARG), ([3, 3], 38, b.LS_ERR_KV_OVERFLOW), ([3, 3], -1, b.LS_ERR_INVALID_ARG), ([1, 1, 1], 0, b.LS_ERR_INVALID_ARG)):
        cu = np.cumsum([0] + counts).astype(np.int32)
        rows = one.expand(int(cu[-1])).contiguous()
        with pytest.raises(LsError) as e:
            st.tree(rows, rows, torch.from_numpy(cu).cuda(), cu, ctx)
        assert e.value.status == status
    cu = torch.tensor([0, 1], dtype=torch.int32).cuda()
    for bad in (one.long(), one.expand(2).contiguous(), one.cpu()):
        with pytest.raises(ValueError):
            st.tree(bad, one, cu, [0, 1], 3)
    st.reset_blocks()
    with pytest.raises(LsError) as e:
        st.tree(one, one, cu, [0, 1], 3)
    assert e.value.status == b.LS_ERR_NOT_LOADED
    st.close()


@pytest.mark.parametrize("shape", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("nodes", [[5, 1], [33, 14]], ids=str)
def test_a_pass_while_blocks_arrive(shape, nodes):
    """The first pass of a stage whose blocks are on their way, last ones first, over trees without a context: the bits of a stage that has them."""
    from helpers import packed_blocks

    r = random.Random(3)
    trees = [plain.random_tree(r, n) for n in nodes]
    parents, cu, host = bounds(trees)
    feed = torch.from_numpy(synth.token_ids(9, sum(nodes), shape.vocab)).cuda()
    outs = []
    for streamed in (False, True):
        n = shape.n_layers_total
        st = make_gpu(shape, 3, 0, n, 2, 80, 80, load=not streamed)
        st.seq_lens.zero_()
        if streamed:
            torch.cuda.synchronize()
            copy, blocks = torch.cuda.Stream(), [(i, st.stage_host_block(i, buf)) for i, buf in packed_blocks(st, 3).items()]
            for i, buf in reversed(blocks):
                st.load_block(i, buf, stream=copy)
        outs.append([t.clone() for t in st.tree(feed, parents, cu, host, 0, want_logits=True)])
        torch.cuda.synchronize()
        st.close()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
