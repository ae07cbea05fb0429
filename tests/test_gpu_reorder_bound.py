"""Reordering of caches whose lengths the host understates: the lengths on the device count."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_ctx", [0, 1, 17, 300, 700])
@pytest.mark.parametrize("heads,dtype", [((4, 64), torch.bfloat16), ((3, 128), torch.float32), ((2, 6), torch.bfloat16)],
                         ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else "")
@pytest.mark.parametrize("group", [2, 5, 9])
def test_an_understated_bound_costs_no_positions(group, heads, dtype, max_ctx):
    from paper_2502_09922_amd import kv_reorder

    (hkv, hd), S, B = heads, 700, 2 * group
    g = torch.Generator().manual_seed(group)
    k, v = (torch.randn(2, B, hkv, S, hd, generator=g).to(dtype) for _ in range(2))
    lens = torch.randint(500, S + 1, (B,), generator=g).int()
    lens[1], lens[group] = S + 40, 0  # past the cache's end, none
    src = (torch.arange(B) // group * group + (torch.arange(B) + 1) % group).int()
    for first in (None, torch.randint(0, 600, (B,), generator=g).int()):
        gk, gv, gl = k.cuda(), v.cuda(), lens.cuda()
        kv_reorder(src.cuda(), group, gk, gv, gl, max_ctx=max_ctx, first=None if first is None else first.cuda())
        wk, wv = k.clone(), v.clone()
        for b in range(B):
            at = slice(0 if first is None else int(first[b]), min(S, int(lens[src[b]])))
            if at.start < at.stop:
                wk[:, b, :, at], wv[:, b, :, at] = k[:, src[b], :, at], v[:, src[b], :, at]
        assert torch.equal(gk.cpu(), wk) and torch.equal(gv.cpu(), wv) and torch.equal(gl.cpu(), lens[src.long()])
