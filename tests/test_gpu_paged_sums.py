"""Attention over pages: sums over long contexts, whose roundings must not all go the same way."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

PAGE = 64
TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


def call(heads, hd, dtype, lens, max_ctx, weighed):
    """Every 16th slot has a score of 0 and the others of a head one of their own below that, so that each tile brings the same sums; the new
    token's is 0 too.  Values are the same in all slots.  (out, weights or None, values, scores of the others, table)."""
    from paper_2502_09922_amd import PagedCache, paged_attention

    B, need = len(lens), [n // PAGE + 1 for n in lens]
    g = torch.Generator().manual_seed(heads + hd)
    order = torch.randperm(sum(need), generator=g).int()
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n], order = order[:n], order[n:]
    below = (-math.sqrt(hd) * (0.1 + 0.9 * torch.rand(heads, generator=g))).to(dtype)
    values = torch.randn(hd, generator=g).to(dtype)
    rows = torch.zeros(heads, PAGE, hd, dtype=dtype)
    rows[:, :, 0] = below[:, None]
    rows[:, ::16, 0] = 0
    size = (1, sum(need), heads, PAGE)
    k = rows.cuda().expand(size + (hd,)).contiguous()
    v = values.cuda().expand(size + (hd,)).contiguous()
    more = (torch.zeros(size, device="cuda"), torch.zeros(size, dtype=torch.int32, device="cuda")) if weighed else (None, None)
    at = torch.tensor(lens, dtype=torch.int32).cuda()
    cache = PagedCache(k, v, table.cuda(), at, at.clone(), *more)
    qkv = torch.zeros(B, 3, heads, hd, dtype=dtype)
    qkv[:, 0, :, 0] = 1
    qkv[:, 2] = values
    out = paged_attention(cache, qkv.view(B, -1).cuda(), None, max_ctx)
    return out.view(B, heads, hd).double().cpu(), None if more[0] is None else more[0][0].cpu(), values.double(), below.double() / math.sqrt(hd), table


def roundings(tiles, waves, pieces):
    """Of sums of weights and of weighted values, in half steps of the result, worst case: n terms that are added up one by one are off by at most
    (n + 1) / 2.  A tile of 16 keys brings 16 products to a value and four weights to a lane, in two steps; 16 tiles are added up,
    then those sums, then the wavefronts' and the pieces', with a factor each; lanes' weights in two steps."""
    far = (-(-tiles // 16) + 1) / 2 + 1
    joins = 2 * waves + 2 * pieces
    return 2 + 17 / 2 + far + 2 + joins, (16 * 16 + 1) / 2 + far + joins


@pytest.mark.parametrize("hd", [64, 128])
def test_outputs_of_one_workgroup(hd):
    """An understated bound: eight wavefronts have a whole context."""
    n = 262100
    out, _, values, _, _ = call(8, hd, torch.float32, [n], 40, False)
    bound = (sum(roundings(n // 16 // 8 + 1, 8, 1)) + 2) * 2.0**-24
    err = float(((out - values).abs() / values.abs()).max())
    print("outputs off by %.2e of them, %.2e allowed" % (err, bound))
    assert err <= bound


def test_outputs_of_contexts_that_are_dealt_out():
    """Two contexts of 256 heads, 1024 workgroups of four wavefronts: three pieces or four of a head of the long one."""
    n = 60000
    out, _, values, _, _ = call(256, 64, torch.float32, [n, 30], n, False)
    bound = (sum(roundings(n // 16 // 3 // 4 + 1, 4, 4)) + 2) * 2.0**-24
    err = float(((out - values).abs() / values.abs()).max())
    print("outputs off by %.2e of them, %.2e allowed" % (err, bound))
    assert err <= bound


@TYPES
def test_weights_of_long_contexts(dtype):
    """More heads than CUs, a workgroup of four wavefronts to each.  A weight: the exponent (the score, of which bf16's second part is 2^-23, the
    factor to base 2 in three roundings, the product) twice 2^-23 of the exponential, the reciprocal and the product, beside the sum
    of weights, whose terms are off by as much."""
    n, heads = 65519, 264
    out, weights, values, below, table = call(heads, 64, dtype, [n], n, True)
    slot = torch.arange(n + 1)
    got = weights[table[0].long()[slot // PAGE], :, slot % PAGE].double()  # [slots][heads]
    high = (slot % 16 == 0) | (slot == n)
    w = torch.where(high[:, None], 1.0, below.exp()[None])
    want = w / w.sum(0)
    bound = (roundings(n // 16 // 4 + 1, 4, 1)[0] + 3 + 2 * (4 + 6 * below.abs())) * 2.0**-24
    err = ((got - want).abs() / want).amax(0)
    print("weights off by %.2e of them, %.2e allowed" % (float(err.max()), float(bound.min())))
    assert (err <= bound).all()
    u = 2.0**-8 if dtype == torch.bfloat16 else sum(roundings(n // 16 // 4 + 1, 4, 1)) * 2.0**-24 + 2.0**-23
    assert ((out - values).abs() <= 1.01 * u * values.abs()).all()


def joined(pieces):
    """Roundings of a sum over pieces, eight at a time, sixteen times that, and those; a factor for each piece and each time."""
    return 9 / 2 + 1 + 17 / 2 + 1 + (-(-pieces // 128) + 1) / 2 + 1


MANY = pytest.mark.parametrize("hd,n,pieces", [(96, 523000, 4096), (64, 1000000, 256)], ids=["any shape", "matrix cores"])


def own_roundings(hd, n, pieces):
    """Of a piece's sums of weights and of weighted values.  The kernel for every shape adds eight keys up, and 64 times that; the other one has eight
    wavefronts in a piece."""
    if hd == 96:
        assert n / pieces <= 512
        return (9 / 2 + 65 / 2 + 1,) * 2
    return roundings(n // 16 // pieces // 8 + 1, 8, 0)


@MANY
def test_outputs_of_many_pieces(hd, n, pieces):
    out, _, values, _, _ = call(1, hd, torch.float32, [n], n, False)
    bound = (sum(own_roundings(hd, n, pieces)) + 2 * joined(pieces) + 2) * 2.0**-24
    err = float(((out - values).abs() / values.abs()).max())
    print("outputs off by %.2e of them, %.2e allowed" % (err, bound))
    assert err <= bound


@MANY
@TYPES
def test_weights_of_many_pieces(hd, n, pieces, dtype):
    out, weights, values, below, table = call(1, hd, dtype, [n], n, True)
    slot = torch.arange(n + 1)
    got = weights[table[0].long()[slot // PAGE], :, slot % PAGE].double()
    w = torch.where(((slot % 16 == 0) | (slot == n))[:, None], 1.0, below.exp()[None])
    want = w / w.sum(0)
    bound = (own_roundings(hd, n, pieces)[0] + joined(pieces) + 3 + 2 * (4 + 6 * below.abs())) * 2.0**-24
    err = float(((got - want).abs() / want).max())
    print("weights off by %.2e of them, %.2e allowed" % (err, float(bound.min())))
    assert err <= float(bound.min())
