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
