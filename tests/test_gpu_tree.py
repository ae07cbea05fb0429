"""Trees of drafted tokens over a cache (ls_tree_attention, ls_tree_accept, ls_tree_keep) against plain 64-bit arithmetic."""
import math
import random

import numpy as np
import pytest
import torch

import continuations_plain as plain

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}  # half a step of a stored value, relative


def make(heads, dtype, ctxs, nodes, seed, max_seq=None, max_batch=None):
    """Queries, keys and values, cache (NaN wherever nothing is cached), table and trees of a call."""
    hq, hkv, hd = heads
    r, g = random.Random(seed), torch.Generator().manual_seed(seed)
    trees = [plain.random_tree(r, n) if n else [] for n in nodes]
    B, S = max_batch or len(ctxs) + 1, max_seq or max(c + n for c, n in zip(ctxs, nodes)) + 3
    cu = np.cumsum([0] + list(nodes)).astype(np.int32)
    qkv = torch.randn(int(cu[-1]), (hq + 2 * hkv) * hd, generator=g).to(dtype)
    k, v = (torch.randn(B, hkv, S, hd, generator=g).to(dtype) for _ in range(2))
    for b in range(B):
        k[b, :, ctxs[b] if b < len(ctxs) else 0 :] = v[b, :, ctxs[b] if b < len(ctxs) else 0 :] = math.nan
    at = torch.arange(S, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)
    rope = torch.stack([at.cos(), at.sin()], -1).float()
    lens = torch.tensor(list(ctxs) + [0] * (B - len(ctxs)), dtype=torch.int32)
    parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32)
    return dict(heads=heads, ctxs=list(ctxs), trees=trees, cu=cu, qkv=qkv, k=k, v=v, rope=rope, lens=lens, parents=parents)


def call(c, turn=True, max_ctx=None, **kw):
    """(out, k, v) of the call, on the host."""
    from paper_2502_09922_amd import tree_attention

    d = {n: c[n].cuda() for n in ("qkv", "k", "v", "rope", "lens", "parents")}
    out = tree_attention(d["qkv"], d["parents"], torch.from_numpy(c["cu"]).cuda(), c["cu"], d["rope"] if turn else None, d["k"], d["v"], d["lens"],
                         max(c["ctxs"]) if max_ctx is None else max_ctx, **kw)
    torch.cuda.synchronize()
    assert torch.equal(d["lens"].cpu(), c["lens"])
    return out.cpu(), d["k"].cpu(), d["v"].cpu()


def same(a, b):
    return torch.equal(a.view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32), b.view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32))


def check(c, got, turn=True, skipped=()):
    """Every output of a call.  Cached rows: values as they came, keys turned in 32 bits (two products and a sum of values of at
    most the pair's size: 3 2^-24 of it) and rounded once; everything else as it was.  Attention over the rows that the cache
    then holds: with scores off by `ds` every weight is off by a factor of at most exp(2 ds), the weights of a bf16 product
    are rounded once, sums of m terms in 32 bits are off by m 2^-24 of the sum of their sizes."""
    out, k, v = got
    hq, hkv, hd = c["heads"]
    dtype, u = c["qkv"].dtype, U[c["qkv"].dtype]
    k_left, v_left = k.clone(), v.clone()
    errs, sizes = [], []
    for b, t in enumerate(c["trees"]):
        n, ctx, r = len(t), c["ctxs"][b], int(c["cu"][b])
        if b in skipped:
            assert (out[r : r + n] == 0).all()
            continue
        if not n:
            continue
        rows = c["qkv"][r : r + n].double().view(n, hq + 2 * hkv, hd)
        pos = [ctx + len(plain.path(t, i)) - 1 for i in range(n)]
        qk = plain.turned(rows[:, : hq + hkv], c["rope"].double() if turn else None, pos)
        here = slice(ctx, ctx + n)
        assert same(v[b, :, here], c["qkv"][r : r + n].view(n, -1, hd)[:, hq + hkv :].transpose(0, 1).contiguous())
        want, pair = qk[:, hq:].transpose(0, 1), rows[:, hq : hq + hkv].abs().view(n, hkv, -1, 2).sum(-1).repeat_interleave(2, -1).transpose(0, 1)
        assert ((k[b, :, here].double() - want).abs() <= u * want.abs() + 2 * 3 * 2.0**-24 * pair).all()
        k_left[b, :, here], v_left[b, :, here] = c["k"][b, :, here], c["v"][b, :, here]
        want, weighted, size = plain.attend(qk[:, :hq], k[b, :, : ctx + n].double(), v[b, :, : ctx + n].double(), ctx, t)
        # queries turned in 32 bits, for matrix products split into two bf16 parts (2^-16 left out); hd products summed in 32 bits
        ds = (hd + 8) * 2.0**-24 * size + (2.0**-16 * size if dtype == torch.bfloat16 else 2.0**-21)
        weights = (2.0**-8 if dtype == torch.bfloat16 else 0.0) + 2 * ds + (ctx + n + 16) * 2.0**-24
        err = (out[r : r + n].double().view(n, hq, hd) - want).abs()
        bound = u * want.abs() + weights * weighted * 1.01 + 1e-30
        assert (err <= bound).all(), (b, n, ctx, float((err / bound).max()), (err / bound).argmax())
        errs.append(err.reshape(-1))
        sizes.append(want.reshape(-1))
    assert same(k_left, c["k"]) and same(v_left, c["v"])  # nothing else was written
    if dtype == torch.bfloat16 and errs:  # two roundings of at most 2^-8, root mean squares 2^-8 / sqrt(3): the output's and the weights'
        assert torch.cat(errs).norm() <= math.sqrt(2 / 3) * 2.0**-8 * torch.cat(sizes).norm()


HEADS = [(4, 4, 64), (4, 4, 128), (8, 2, 128), (8, 1, 128), (16, 2, 64), (32, 2, 64), (3, 1, 128), (6, 2, 80), (2, 1, 256), (5, 5, 2)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%dx%dx%d" % h)
def test_ragged_trees(heads, dtype):
    c = make(heads, dtype, [0, 1, 31, 32, 33, 100, 5], [1, 5, 2, 7, 0, 16, 3], 1)
    check(c, call(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 2, 128), (8, 2, 64), (8, 1, 128)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("nodes", [1, 15, 16, 17, 32, 33, 63, 64])
def test_tree_sizes(heads, dtype, nodes):
    c = make(heads, dtype, [63, 0, 130], [nodes, 64, max(1, nodes // 2)], nodes)
    check(c, call(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 2, 128), (8, 1, 128), (2, 2, 64), (3, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("ctx", [600, 1023, 2500])
def test_long_contexts(heads, dtype, ctx):
    """Contexts that several workgroups share; an understated bound of their length changes nothing but the speed."""
    c = make(heads, dtype, [ctx, 7, ctx // 2], [9, 4, 20], ctx)
    got = call(c)
    check(c, got)
    check(c, call(c, max_ctx=64))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_many_sequences(dtype):
    r = random.Random(4)
    c = make((4, 2, 128), dtype, [r.randrange(150) for _ in range(70)], [r.randrange(9) for _ in range(70)], 5)
    check(c, call(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", ["chain", "star", "two roots"])
def test_shapes_of_trees(shape, dtype):
    """A chain sees all in front of it, leaves of a star the root alone; a parent that is none starts a tree of its own."""
    c = make((4, 2, 64), dtype, [40, 3], [64, 12], 3)
    for t in c["trees"]:
        for i in range(1, len(t)):
            t[i] = i - 1 if shape == "chain" else 0 if shape == "star" else (-1 if i == 2 else 7 if i == 5 else i // 2)
    c["parents"] = torch.tensor([p for t in c["trees"] for p in t], dtype=torch.int32)
    check(c, call(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(4, 2, 128), (4, 4, 80)], ids=lambda h: "%dx%dx%d" % h)
def test_rows_that_come_turned(heads, dtype):
    c = make(heads, dtype, [20, 70], [6, 11], 8)
    check(c, call(c, turn=False), turn=False)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(4, 2, 128), (4, 4, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
def test_sequences_without_room_are_left_alone(heads, dtype):
    """Lengths that the device alone knows: a tree that does not fit behind them, a negative one."""
    c = make(heads, dtype, [50, 58, 20, 30], [6, 6, 6, 6], 9, max_seq=60)
    c["lens"][1], c["lens"][2] = 55, -1
    check(c, call(c, max_ctx=54), skipped=(1, 2))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 2, 128), (8, 1, 128), (2, 2, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_nonfinite_rows_reach_only_who_sees_them(heads, dtype, bad):
    """Node 3's key and value, then a cached key's and value's: rows that do not see them keep their bits."""
    hq, hkv, hd = heads
    c = make(heads, dtype, [45, 50], [12, 5], 10)
    clean = call(c)
    for what in ("key", "value"):
        d = dict(c, qkv=c["qkv"].clone())
        col = (hq if what == "key" else hq + hkv) * hd + 1
        d["qkv"][3, col] = bad
        out = call(d)[0]
        sees = [3 in plain.path(c["trees"][0], i) for i in range(12)] + [False] * 5
        keep = torch.tensor([not s for s in sees])
        assert same(out[keep], clean[0][keep]), what
        assert torch.isfinite(out[keep]).all()
        if what == "value" and not math.isnan(bad):
            assert (out[~keep].view(-1, hq, hd)[:, : hq // hkv, 1] == bad).all()
        if math.isnan(bad):
            assert out[~keep].view(-1, hq, hd)[:, : hq // hkv].isnan().any(-1).all()
    d = dict(c, v=c["v"].clone())
    d["v"][0, 0, 10, 2] = bad
    out = call(d)[0]
    assert not torch.isfinite(out[:12].view(-1, hq, hd)[:, : hq // hkv, 2]).any()
    assert same(out[12:], clean[0][12:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_scores_of_the_types_lowest_values(dtype):
    """Keys whose scores with every query are far below zero, and equal: the softmax is over what is left of them."""
    c = make((4, 2, 128), dtype, [40], [5], 11)
    c["qkv"][:, : 4 * 128], c["k"][0, :, :40] = 8.0, -8.0
    c["qkv"][:, 4 * 128 : 6 * 128] = -8.0
    check(c, call(c, turn=False), turn=False)


def test_streams_and_replays():
    """Captured once, replayed with other contents and lengths, with eager calls between; and on a stream of its own."""
    from paper_2502_09922_amd import tree_attention

    cases = [make((8, 2, 128), torch.bfloat16, ctxs, [9, 4, 16], s, max_seq=1200) for s, ctxs in ((1, [1000, 3, 700]), (2, [20, 900, 0]), (3, [1000, 999, 998]))]
    want = [call(c, max_ctx=1000) for c in cases]
    d = {n: cases[0][n].cuda() for n in ("qkv", "k", "v", "rope", "lens", "parents")}
    cu = torch.from_numpy(cases[0]["cu"]).cuda()

    def run():
        return tree_attention(d["qkv"], d["parents"], cu, cases[0]["cu"], d["rope"], d["k"], d["v"], d["lens"], 1000)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = run()
    side.synchronize()
    assert same(out.cpu(), want[0][0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in (1, 2, 0, 1, 2):
        for n in d:
            d[n].copy_(cases[i][n])
        graph.replay()
        torch.cuda.synchronize()
        assert same(out.cpu(), want[i][0]) and same(d["k"].cpu(), want[i][1]) and same(d["v"].cpu(), want[i][2]), i
        assert same(call(cases[i], max_ctx=1000)[0], want[i][0])


# ---- acceptance and compaction ---------------------------------------------------------------------------------------------
def drafts(nodes, seed):
    """Trees whose tokens agree with the model in six of ten places, with equal tokens among siblings."""
    r = random.Random(seed)
    trees = [plain.random_tree(r, n) if n else [] for n in nodes]
    said = [[r.randrange(4) for _ in t] for t in trees]
    tokens = [[s[max(p, 0)] if r.random() < 0.6 else r.randrange(4) for p in t] for t, s in zip(trees, said)]
    return trees, tokens, said


@pytest.mark.parametrize("nodes", [[1], [64], [0, 5, 64, 1, 0], [2, 3, 63, 33, 17, 9] * 20], ids=["root", "full", "ragged", "many"])
@pytest.mark.parametrize("seed", [1, 2, 3])
def test_accept(nodes, seed):
    from paper_2502_09922_amd import tree_accept

    trees, tokens, said = drafts(nodes, seed)
    cu = np.cumsum([0] + nodes).astype(np.int32)
    flat = lambda v: torch.tensor([x for t in v for x in t], dtype=torch.int32).cuda()  # noqa: E731
    kept, count, emitted, following = (t.cpu() for t in tree_accept(flat(tokens), flat(said), flat(trees), torch.from_numpy(cu).cuda(), cu))
    for b, t in enumerate(trees):
        p = plain.accepted(t, tokens[b], said[b]) if t else []
        assert int(kept[b]) & (2**64 - 1) == sum(1 << i for i in p)
        assert int(count[b]) == len(p)
        assert emitted[b].tolist() == [said[b][i] for i in p] + [-1] * (64 - len(p))
        assert int(following[b]) == (said[b][p[-1]] if p else -1)


def test_accept_of_parents_that_are_none():
    from paper_2502_09922_amd import tree_accept

    cu, said = np.array([0, 5], np.int32), torch.tensor([1, 1, 1, 1, 1], dtype=torch.int32).cuda()
    parents = torch.tensor([-1, 3, -1, 0, 3], dtype=torch.int32).cuda()  # of 1: behind it; of 2: none
    kept, count, emitted, _ = tree_accept(said, said, parents, torch.from_numpy(cu).cuda(), cu)
    assert int(kept) == 0b11001 and int(count) == 3


@pytest.mark.parametrize("heads,dtype", [((4, 64), torch.bfloat16), ((3, 128), torch.float32), ((2, 6), torch.bfloat16), ((2, 80), torch.bfloat16)],
                         ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else "")
@pytest.mark.parametrize("layers", [1, 5])
def test_keep(heads, dtype, layers):
    from paper_2502_09922_amd import tree_keep

    (hkv, hd), r = heads, random.Random(6)
    nodes, ctxs, S = [64, 0, 7, 33, 9, 1], [10, 4, 0, 60, 92, 8], 100  # the fifth has no room
    masks = [r.getrandbits(n) | 1 if n else 0 for n in nodes]
    masks[0] |= 1 << 63
    masks[2] |= 1 << 20  # bits behind the tree
    g = torch.Generator().manual_seed(6)
    k, v = (torch.randn(layers, len(nodes) + 2, hkv, S, hd, generator=g).to(dtype) for _ in range(2))
    cu = np.cumsum([0] + nodes).astype(np.int32)
    lens = torch.tensor(ctxs + [5, 6], dtype=torch.int32)
    gk, gv, gl = k.cuda(), v.cuda(), lens.cuda()
    signed = [m - 2**64 if m >> 63 else m for m in masks]
    tree_keep(torch.tensor(signed).cuda(), torch.from_numpy(cu).cuda(), cu, gk, gv, gl)
    for b, (n, ctx, m) in enumerate(zip(nodes, ctxs, masks)):
        if ctx + n > S:
            continue
        kept = [i for i in range(n) if m >> i & 1]
        for c in (k, v):
            c[:, b, :, ctx : ctx + len(kept)] = c[:, b, :, [ctx + i for i in kept]].clone()
        lens[b] = ctx + len(kept)
    assert torch.equal(gk.cpu(), k) and torch.equal(gv.cpu(), v) and torch.equal(gl.cpu(), lens)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_offsets_beyond_32_bits(dtype):
    """A cache of 2^32 values and more: keys are all alike, so that the softmax counts them; nodes, values and moved rows lie at its end."""
    from paper_2502_09922_amd import kv_reorder, tree_attention, tree_keep

    S, hd, n = 1 << 24, 64, 5
    ctx = S - 9
    k, v = (torch.zeros(5, 1, S, hd, dtype=dtype, device="cuda") for _ in range(2))
    v[4, 0, ctx - 1000 : ctx] = 1.0
    qkv = torch.zeros(n, 3 * hd, dtype=dtype, device="cuda")
    qkv[:, 2 * hd :] = torch.arange(1, n + 1, device="cuda")[:, None] * 256.0
    cu_host = np.array([0, 0, 0, 0, 0, n], np.int32)
    cu, parents = torch.from_numpy(cu_host).cuda(), torch.tensor([-1, 0, 0, 2, 1], dtype=torch.int32).cuda()
    lens = torch.tensor([0, 0, 0, 0, ctx], dtype=torch.int32).cuda()
    out = tree_attention(qkv, parents, cu, cu_host, None, k, v, lens, ctx).double().cpu()
    for i, seen in enumerate(([0], [0, 1], [0, 2], [0, 2, 3], [0, 1, 4])):
        want = (1000 + 256 * sum(j + 1 for j in seen)) / (ctx + len(seen))
        # weights of one and sums of whole numbers below 2^24, of which the last ones are rounded: 2^-24 each of up to ctx + 5 terms
        # where a wavefront's share of the keys is at most 2^16, so 2^-8 of it; the output's own rounding
        assert (out[i] - want).abs().max() <= want * (U[dtype] + 2.0**-8)
    assert torch.equal(v[4, 0, ctx : ctx + n, 0].cpu().double(), torch.arange(1, n + 1).double() * 256)
    tree_keep(torch.tensor([0, 0, 0, 0, 0b11001], device="cuda"), cu, cu_host, k[None], v[None], lens)
    assert lens.tolist() == [0, 0, 0, 0, ctx + 3] and v[4, 0, ctx : ctx + 3, 7].tolist() == [256.0, 1024.0, 1280.0]
    src = torch.tensor([0, 1, 2, 4, 4], dtype=torch.int32, device="cuda")
    kv_reorder(src, 5, k[None], v[None], lens, S, first=torch.full((5,), ctx - 3, dtype=torch.int32, device="cuda"))
    assert torch.equal(v[3, 0, ctx - 3 : ctx + 3], v[4, 0, ctx - 3 : ctx + 3]) and (v[3, 0, : ctx - 3] == 0).all() and lens.tolist()[3] == ctx + 3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(8, 8, 128), (39, 13, 64), (104, 13, 64), (208, 13, 64)], ids=lambda h: "%dx%dx%d" % h)
def test_lengths_in_any_order_and_outside_the_cache(heads, dtype):
    """Sequences that are taken by length, among them lengths that the device alone knows: negative, too long, past 31 bits."""
    r = random.Random(12)
    ctxs, nodes = [r.randrange(600) for _ in range(40)], [8 if b % 13 == 5 else 1 for b in range(40)]
    ctxs[20] = 599
    c = make(heads, dtype, ctxs, nodes, 12, max_seq=620)
    for b, n in ((1, -5), (3, 620), (7, 2**31 - 1), (8, -(2**31))):
        c["lens"][b] = n
    check(c, call(c, max_ctx=599), skipped=(1, 3, 7, 8))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_more_sequences_than_are_ordered(dtype):
    r = random.Random(13)
    n = 300
    c = make((2, 1, 64), dtype, [r.randrange(40) if b % 50 else 550 for b in range(n)], [r.randrange(3) for _ in range(n)], 13)
    check(c, call(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("what", ["qkv", "k", "v", "rope", "out"])
def test_buffers_off_16_bytes(what, dtype):
    """Views that start a row's alignment off: the kernels for every shape take them."""
    from paper_2502_09922_amd import tree_attention

    c = make((4, 2, 64), dtype, [20, 33], [5, 9], 14)
    d = {n: c[n].cuda() for n in ("qkv", "k", "v", "rope", "lens", "parents")}
    d["out"] = torch.zeros(14, 4 * 64, dtype=dtype, device="cuda")
    at = torch.zeros(d[what].numel() + 8, dtype=d[what].dtype, device="cuda")[2 : 2 + d[what].numel()].view(d[what].shape)
    at.copy_(d[what])
    d[what] = at
    assert at.data_ptr() % 16
    out = tree_attention(d["qkv"], d["parents"], torch.from_numpy(c["cu"]).cuda(), c["cu"], d["rope"], d["k"], d["v"], d["lens"], 33, out=d["out"])
    assert out is d["out"]
    check(c, (out.cpu(), d["k"].cpu(), d["v"].cpu()))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_scratch_of_any_size(dtype):
    """None, too little, enough: the same results but for the order of sums; a byte behind its end stays."""
    from paper_2502_09922_amd import binding as b

    c = make((6, 3, 128), dtype, [900, 3], [5, 1], 15)
    d = {n: c[n].cuda() for n in ("qkv", "rope", "lens", "parents")}
    cu, heads = torch.from_numpy(c["cu"]).cuda(), b.ls_heads(int(dtype == torch.bfloat16), 6, 3, 128, c["k"].shape[0], c["k"].shape[2])
    tree = b.ls_tree(d["parents"].data_ptr(), cu.data_ptr(), c["cu"].__array_interface__["data"][0])
    need = b.lib.ls_tree_attention_scratch_bytes(b.C.byref(heads), b.C.byref(tree), 2, 900)
    assert need > 0
    stream = torch.cuda.current_stream().cuda_stream
    for nb in (0, 16, need // 3, need - 1, need):
        out, k, v = torch.zeros(6, 6 * 128, dtype=dtype, device="cuda"), c["k"].cuda(), c["v"].cuda()
        scratch = torch.full((need + 64,), 77, dtype=torch.uint8, device="cuda")
        kv = b.ls_kv(k.data_ptr(), v.data_ptr(), d["lens"].data_ptr())
        assert b.lib.ls_tree_attention(b.C.byref(heads), b.C.byref(tree), 2, 900, d["qkv"].data_ptr(), d["rope"].data_ptr(), b.C.byref(kv), out.data_ptr(),
                                       scratch.data_ptr() if nb else None, nb, stream) == b.LS_OK
        check(c, (out.cpu(), k.cpu(), v.cpu()))
        assert (scratch[nb:] == 77).all()


@pytest.mark.parametrize("heads", [(4, 2, 128), (4, 4, 80)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("now", [[2, 0, 9], [0, 4, 3], [9, 9, 1], [3, 10, 2], [12, 3, 1]], ids=str)
def test_replayed_with_other_trees(heads, now):
    """A captured call whose bounds on the device change: smaller trees; trees that exceed its rows or its largest tree take no part."""
    from paper_2502_09922_amd import tree_accept, tree_attention, tree_keep

    most = [9, 8, 5]
    c = make(heads, torch.bfloat16, [40, 700, 3], now, 16, max_seq=740)
    rows = sum(most)
    qkv, parents = torch.zeros(rows, c["qkv"].shape[1], dtype=torch.bfloat16), torch.zeros(rows, dtype=torch.int32)
    qkv[: len(c["qkv"])], parents[: len(c["parents"])] = c["qkv"][:rows], c["parents"][:rows]
    host = np.cumsum([0] + most).astype(np.int32)
    d = {n: c[n].cuda() for n in ("k", "v", "rope", "lens")}
    qkv, parents, cu, tokens = qkv.cuda(), parents.cuda(), torch.from_numpy(host).cuda(), torch.zeros(rows, dtype=torch.int32).cuda()
    out = torch.full((rows, heads[0] * heads[2]), 7.0, dtype=torch.bfloat16, device="cuda")
    kept = torch.full((3,), -1, dtype=torch.int64, device="cuda")
    graph = torch.cuda.CUDAGraph()
    tree_attention(qkv, parents, cu, host, d["rope"], c["k"].cuda(), c["v"].cuda(), d["lens"], 700)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        tree_attention(qkv, parents, cu, host, d["rope"], d["k"], d["v"], d["lens"], 700, out=out)
        accepted = tree_accept(tokens, tokens, parents, cu, host)
        tree_keep(kept, cu, host, d["k"][None], d["v"][None], d["lens"])
    cu.copy_(torch.from_numpy(c["cu"]))
    graph.replay()
    torch.cuda.synchronize()
    part = [n if n <= max(most) and c["cu"][b + 1] <= rows else 0 for b, n in enumerate(now)]
    assert d["lens"][:3].tolist() == [ctx + n for ctx, n in zip(c["ctxs"], part)]
    deepest = [max(len(plain.path(t, i)) for i in range(len(t))) if n else 0 for t, n in zip(c["trees"], part)]
    assert accepted[1].tolist() == deepest
    there = torch.zeros(rows, dtype=torch.bool)
    for b, n in enumerate(part):
        there[c["cu"][b] : c["cu"][b] + n] = True
    got = out.cpu()
    assert (got[~there] == 7).all()
    k, v = d["k"].cpu(), d["v"].cpu()
    for b, n in enumerate(part):
        if n != now[b]:
            assert same(k[b], c["k"][b]) and same(v[b], c["v"][b])
    alone = dict(c, trees=[t if n else [] for t, n in zip(c["trees"], part)])
    full = torch.zeros(max(rows, int(c["cu"][-1])), got.shape[1], dtype=got.dtype)
    full[:rows] = got
    check(alone, (full, k, v))


def test_bounds_that_may_not_be_written():
    from paper_2502_09922_amd import tree_accept

    cu = np.array([0, 2, 3], np.int32)
    cu.flags.writeable = False
    t = torch.tensor([5, 7, 5], dtype=torch.int32).cuda()
    for host in (cu, [0, 2, 3], torch.tensor([0, 2, 3]).numpy(), np.array([0, 9, 2, 9, 3], np.int32)[::2]):
        kept, count, emitted, following = tree_accept(t, t, torch.tensor([-1, 0, -1], dtype=torch.int32).cuda(), torch.tensor([0, 2, 3], dtype=torch.int32).cuda(), host)
        assert kept.tolist() == [1, 1] and count.tolist() == [1, 1] and emitted[:, 0].tolist() == [5, 5] and following.tolist() == [5, 5]
