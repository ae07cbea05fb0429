"""Trees' bounds that the device alone knows: each sequence takes part or not by its own, whatever its neighbours' are."""
import numpy as np
import pytest
import torch

from test_gpu_tree import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("heads", [(4, 2, 128), (16, 2, 64), (3, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("ctx", [30, 2500])
@pytest.mark.parametrize("cu", [[0, 4, 40, 8, 12], [0, 4, -3, 8, 12], [0, 4, 2**31 - 1, 8, 12], [0, 4, 4, 8, 12]], ids=str)
def test_a_sequence_between_bounds_of_none(cu, ctx, heads, dtype):
    """Four trees of four nodes when the call was made; now the first and the last have theirs, and between them are bounds that no tree has (or
    rows of a tree that the third sequence takes).  Contexts of one workgroup and of several."""
    from paper_2502_09922_amd import tree_attention

    third = cu[2] == 4
    c = make(heads, dtype, [ctx, 20, ctx // 2, ctx - 7], [4, 0, 4 if third else 0, 4], 30)
    rows = 16
    qkv, parents = torch.zeros(rows, c["qkv"].shape[1], dtype=dtype), torch.zeros(rows, dtype=torch.int32)
    for b, n in ((0, 4), (2, 4), (3, 4)):
        if c["trees"][b]:
            qkv[cu[b] : cu[b] + n] = c["qkv"][c["cu"][b] : c["cu"][b] + n]
            parents[cu[b] : cu[b] + n] = c["parents"][c["cu"][b] : c["cu"][b] + n]
    c["qkv"], c["parents"], c["cu"] = qkv, parents, np.array(cu)
    d = {n: c[n].cuda() for n in ("qkv", "k", "v", "rope", "lens", "parents")}
    out = torch.full((rows, heads[0] * heads[2]), 7.0, dtype=dtype, device="cuda")
    tree_attention(d["qkv"], d["parents"], torch.tensor(cu, dtype=torch.int32).cuda(), np.arange(0, 20, 4, dtype=np.int32), d["rope"], d["k"], d["v"], d["lens"],
                   ctx, out=out)
    out = out.cpu()
    check(c, (out, d["k"].cpu(), d["v"].cpu()))
    none = [r for r in range(rows) if not (r < 4 or 8 <= r < 12 or (third and 4 <= r < 8))]
    assert (out[none] == 7).all()
