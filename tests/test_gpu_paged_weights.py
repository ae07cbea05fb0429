"""The weights that slots get are fp32, as the softmax is that they come from: queries, turned in 32 bits, lose none on their way to the scores."""
import math

import pytest
import torch

import paged_plain as plain
from continuations_plain import turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (16, 1, 128), (20, 1, 128), (8, 2, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("lens", [[200, 7], [900, 3], [2500, 90]], ids=str)
def test_weights_of_large_scores(heads, dtype, lens):
    """Queries and keys of one pair of dims, turned, with scores of some 20: what a score is off by, a weight is off by, of itself.  A turned
    value has two roundings of its pair's size (2^-24 each); six products at most that are not zero are added up in 32 bits, however the matrix
    cores round (2^-23 each); the exponent is that of the maximum in a handful of roundings, its exponential off by 2^-21 at most; a sum of the
    weights has n terms, a slot's as many as there are query heads.  Parts of 16 bits would be off by up to 2^-16 of a score."""
    from paper_2502_09922_amd import paged_attention

    hq, hkv, hd = heads
    c = plain.Pages(heads, dtype, lens, 16, seed=hd + lens[0], weighed=True)
    rows = c.qkv.view(len(lens), hq + 2 * hkv, hd)
    rows[:, :, 2:] = 0
    rows[:, :hq] *= 10 * math.sqrt(hd / 64)
    c.k[..., 2:] = torch.where(c.k[..., 2:].isnan(), c.k[..., 2:], 0)
    c.weights = torch.where(c.weights.isnan(), c.weights, 0.0)
    rope, cache = plain.rope_table(max(lens) + 1, hd), c.on_gpu()
    paged_attention(cache, c.qkv[0].cuda(), rope.cuda(), max(lens))
    weights, keys = cache.weights.cpu(), cache.k.cpu()
    worst = 0.0
    for b, n in enumerate(lens):
        slot = torch.arange(n + 1)
        page, row = c.table[b].long()[slot // 16], slot % 16
        k = keys[0, page, :, row].double().permute(1, 0, 2)[..., :2]  # [hkv][slots][2]
        raw = rows[b].double()
        q = turned(raw[None, :hq], rope.double(), [n])[0].view(hkv, hq // hkv, hd)[..., :2]
        score = (q[:, :, None] * k[:, None]).sum(-1) / math.sqrt(hd)  # [hkv][heads of it][slots]
        size = (q[:, :, None] * k[:, None]).abs().sum(-1) / math.sqrt(hd)
        pair = raw[:hq].abs().sum(-1).view(hkv, -1, 1) * k.abs().sum(-1)[:, None] / math.sqrt(hd)
        p = torch.softmax(score, -1)
        ds = (2 * 2.0**-24 * pair + 6 * 2.0**-23 * size) * 1.01
        top = torch.where(p < 1e-30, 0.0, score).abs().amax(-1, keepdim=True)
        off = ds + (p * ds).sum(-1, keepdim=True) + 8 * 2.0**-24 * top + 2.0**-21 + (n + 17) * 2.0**-24
        want, bound = p.sum(1), (p * off).sum(1) * 1.01 + (hq // hkv + 2) * 2.0**-24 * p.sum(1)  # [hkv][slots]
        got = weights[0, page, :, row].double().T
        err = (got - want).abs()
        worst = max(worst, float((err / (bound + 1e-30)).max()))
    print("at most %.2f of what roundings make" % worst)
    assert worst <= 1
