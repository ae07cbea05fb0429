"""Tree attention where its numbers are most exposed, against plain 64-bit arithmetic."""
import math

import pytest
import torch

import continuations_plain as plain
from test_gpu_tree import U, call, make

pytestmark = pytest.mark.gpu


def wanted(c, k, v):
    """Rows of c, which come turned, over the cache (k, v): (out, sums of weighted |v|, sizes of scores) in 64 bits."""
    hq, hkv, hd = c["heads"]
    parts = []
    for b, t in enumerate(c["trees"]):
        n, ctx, r = len(t), c["ctxs"][b], int(c["cu"][b])
        q = c["qkv"][r : r + n].double().view(n, -1, hd)[:, :hq]
        parts.append(plain.attend(q, k[b, :, : ctx + n].double(), v[b, :, : ctx + n].double(), ctx, t))
    return [torch.cat(p) for p in zip(*parts)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 2, 128), (4, 2, 64), (16, 1, 128), (3, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("ctx", [3, 40, 900])
def test_weights_keep_more_bits_than_the_output(heads, dtype, ctx):
    """Rows that come turned, so that queries are exact, over few keys and many.  An output is rounded once, a weight to no fewer than 15 bits (two
    bf16 parts, of which the second is rounded: 2^-7 2^-8 of the weight); scores are sums of hd products in 32 bits, sums of the weights have a
    term for each key.  A weight rounded to 8 bits is off by 2^-8."""
    c = make(heads, dtype, [ctx, ctx // 2], [9, 4], 20)
    out, k, v = call(c, turn=False)
    want, weighted, size = wanted(c, k, v)
    ds = (heads[2] + 10) * 2.0**-24 * size + 2.0**-23
    weights = (2.0**-15 if dtype == torch.bfloat16 else 0.0) + 2 * ds + (ctx + 9 + 16) * 2.0**-24
    err = (out.double().view(want.shape) - want).abs()
    bound = U[dtype] * want.abs() + 1.01 * weights * weighted
    assert float((err / bound).max()) <= 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 2, 128), (4, 2, 64), (16, 1, 128), (3, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("bad", [math.inf, -math.inf])
def test_infinite_cached_values_stay_what_they_are(heads, dtype, bad):
    """A positive weight times an infinite value, however many parts the weight has: all rows of the sequence see it."""
    hq, hkv, hd = heads
    for ctx, at in ((45, 44), (300, 7)):
        c = make(heads, dtype, [ctx, 50], [12, 5], 21)
        clean = call(c)[0].view(-1, hq, hd)
        c["v"][0, 0, at, 2] = bad
        out = call(c)[0].view(-1, hq, hd)
        assert (out[:12, : hq // hkv, 2] == bad).all()
        out[:12, : hq // hkv, 2] = clean[:12, : hq // hkv, 2]
        assert torch.equal(out, clean)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 2, 128), (4, 2, 64), (16, 1, 128), (3, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("turn", [False, True], ids=["as they come", "turned"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf])
def test_infinite_keys(heads, dtype, turn, bad):
    """A cached key with an infinite value: rows whose query is of the other sign there have it at a weight of zero, the others have no number."""
    hq, hkv, hd = heads
    c = make(heads, dtype, [40, 50], [12, 5], 22)
    c["k"][0, 0, 10, 2] = bad
    out, k, v = call(c, turn=turn)
    out = out.double().view(-1, hq, hd)
    rows = c["qkv"].double().view(17, -1, hd)[:, :hq]
    pos = [c["ctxs"][b] + len(plain.path(t, i)) - 1 for b, t in enumerate(c["trees"]) for i in range(len(t))]
    q = plain.turned(rows, c["rope"].double() if turn else None, pos)[:12]
    at = q[:, : hq // hkv, 2]  # what the infinite value is multiplied by
    assert (at.abs() > 1e-4).all() and ((at > 0) == (bad > 0)).any() and ((at > 0) != (bad > 0)).any()
    got = out[:12, : hq // hkv]
    assert (got.isnan().all(-1) == ((at > 0) == (bad > 0))).all()
    assert torch.isfinite(out[12:]).all() and torch.isfinite(out[:12, hq // hkv :]).all()
    want, weighted, size = plain.attend(q, k[0, :, :52].double(), v[0, :, :52].double(), 40, c["trees"][0])
    k[0, 0, 10, 2] = 0.0  # sizes of the other scores
    size = plain.attend(q, k[0, :, :52].double(), v[0, :, :52].double(), 40, c["trees"][0])[2][:, : hq // hkv]
    keep = ~got.isnan()
    # queries turned in 32 bits enter as two bf16 parts, of which the second is rounded: 2^-15 of them
    ds = (hd + 10) * 2.0**-24 * size + (2.0**-15 * size if dtype == torch.bfloat16 else 2.0**-21)
    weights = (2.0**-15 if dtype == torch.bfloat16 else 0.0) + 2 * ds + 70 * 2.0**-24
    err, want = (got - want[:, : hq // hkv]).abs(), want[:, : hq // hkv]
    assert float((err / (U[dtype] * want.abs() + 1.01 * weights * weighted[:, : hq // hkv]))[keep].max()) <= 1


@pytest.mark.parametrize("hd", [96, 128])
@pytest.mark.parametrize("ctx,s", [(40000, 1.0), (60000, 1.2), (60000, 2.0)])
def test_long_sums_of_equal_weights(hd, ctx, s):
    """One key above, all others equal, half of them of value one: added up one by one, each step rounds a weight the same way next to a long
    sum (4e-4 to 7e-4 of it).  Eight weights at a time, 64 times that, and those: 8 + 64 + ctx / 512 roundings of both sums; the
    matrix cores' kernel has shorter ones."""
    k, v = torch.zeros(1, 1, ctx + 1, hd), torch.zeros(1, 1, ctx + 1, hd)
    c = dict(heads=(1, 1, hd), ctxs=[ctx], trees=[[-1]], cu=torch.tensor([0, 1], dtype=torch.int32).numpy(), qkv=torch.zeros(1, 3 * hd), k=k, v=v,
             rope=torch.zeros(ctx + 1, hd // 2, 2), lens=torch.tensor([ctx], dtype=torch.int32), parents=torch.tensor([-1], dtype=torch.int32))
    c["qkv"][0, 0] = math.sqrt(hd)
    c["qkv"][0, hd] = -s
    k[0, 0, 1:ctx, 0] = -s
    v[0, 0, 1:ctx:2] = 1.0
    out, k, v = call(c, turn=False)
    want, weighted, size = wanted(c, k, v)
    weights = 2 * (8 + 64 + ctx / 512 + 16) * 2.0**-24 + 2 * ((hd + 8) * 2.0**-24 * size + 2.0**-21)
    err = (out.double().view(want.shape) - want).abs()
    assert float((err / (weights * weighted + U[torch.float32] * want)).max()) <= 1
