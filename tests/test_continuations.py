"""What ls_tree_attention, ls_tree_accept, ls_tree_keep, ls_beam_select and ls_kv_reorder refuse, before they touch a device."""
import ctypes as C

import numpy as np
import pytest

from paper_2502_09922_amd import binding as b

HERE = 4096  # an aligned address that no refused call looks at


def heads(**kw):
    v = dict(dtype=b.LS_DTYPE_BF16, n_q_heads=8, n_kv_heads=2, head_dim=128, max_batch=4, max_seq=100)
    v.update(kw)
    return b.ls_heads(*[v[n] for n, _ in b.ls_heads._fields_])


def tree(counts=(5, 0, 64), start=0, **kw):
    host = np.cumsum([start] + list(counts)).astype(np.int32)
    t = b.ls_tree(kw.get("parents", HERE), kw.get("cu", HERE), host.ctypes.data if kw.get("host", True) else None)
    t.keep = host
    return t


def attention(h=None, t=None, batch=3, max_ctx=36, qkv=HERE, rope=HERE, k=HERE, v=HERE, lens=HERE, out=HERE, kv=True):
    h, t = heads() if h is None else h, tree() if t is None else t
    layer = b.ls_kv(k, v, lens)
    return b.lib.ls_tree_attention(C.byref(h), C.byref(t), batch, max_ctx, qkv, rope, C.byref(layer) if kv else None, out, None, 0, None)


@pytest.mark.parametrize("wrong", [dict(dtype=2), dict(n_kv_heads=3), dict(n_kv_heads=0), dict(head_dim=0), dict(head_dim=65), dict(head_dim=258),
                                   dict(max_batch=0), dict(max_seq=0), dict(max_seq=(1 << 24) + 1)], ids=str)
def test_heads(wrong):
    assert attention(heads(**wrong)) == b.LS_ERR_INVALID_ARG
    assert b.lib.ls_tree_attention_scratch_bytes(C.byref(heads(**wrong)), C.byref(tree()), 3, 36) == 0


@pytest.mark.parametrize("counts,start", [((5, 65, 1), 0), ((5, -1, 3), 0), ((5, 1, 1), 1)])
def test_bounds_of_trees(counts, start):
    t = tree(counts, start)
    assert attention(t=t) == b.LS_ERR_INVALID_ARG
    assert b.lib.ls_tree_accept(C.byref(t), 3, *[HERE] * 6, None) == b.LS_ERR_INVALID_ARG
    kv = b.ls_kv(HERE, HERE, HERE)
    assert b.lib.ls_tree_keep(C.byref(heads()), 1, C.byref(t), 3, HERE, C.byref(kv), None) == b.LS_ERR_INVALID_ARG


@pytest.mark.parametrize("wrong", [dict(batch=0), dict(batch=5), dict(max_ctx=-1), dict(qkv=None), dict(out=None), dict(k=None), dict(v=None), dict(lens=None),
                                   dict(kv=False), dict(qkv=HERE + 1), dict(out=HERE + 1), dict(k=HERE + 1), dict(v=HERE + 1), dict(rope=HERE + 4)], ids=str)
def test_attention(wrong):
    assert attention(**wrong) == b.LS_ERR_INVALID_ARG
    assert b"ls_tree_attention" in b.lib.ls_last_error()


def test_attention_of_trees_that_do_not_fit():
    assert attention(max_ctx=96) == b.LS_ERR_KV_OVERFLOW  # the smallest tree of the call has 5 nodes
    for t in (tree(parents=None), tree(cu=None), tree(host=False)):
        assert attention(t=t) == b.LS_ERR_INVALID_ARG


def test_calls_without_nodes_do_nothing():
    t = tree((0, 0, 0), parents=None)
    assert attention(t=t, qkv=None, out=None) == b.LS_OK
    kv = b.ls_kv(HERE, HERE, HERE)
    assert b.lib.ls_tree_keep(C.byref(heads()), 1, C.byref(t), 3, HERE, C.byref(kv), None) == b.LS_OK


def test_accept_and_keep():
    t, h, kv = tree(), heads(), b.ls_kv(HERE, HERE, HERE)
    for i in range(6):
        args = [HERE] * 6
        args[i] = None
        assert b.lib.ls_tree_accept(C.byref(t), 3, *args, None) == b.LS_ERR_INVALID_ARG
    assert b.lib.ls_tree_accept(C.byref(t), 3, HERE, HERE, HERE + 4, HERE, HERE, HERE, None) == b.LS_ERR_INVALID_ARG
    assert b.lib.ls_tree_accept(None, 3, *[HERE] * 6, None) == b.LS_ERR_INVALID_ARG
    keep = lambda h=h, layers=2, t=t, batch=3, kept=HERE, kv=kv: b.lib.ls_tree_keep(  # noqa: E731
        C.byref(h), layers, C.byref(t), batch, kept, C.byref(kv), None)
    for wrong in (dict(layers=0), dict(layers=1 << 24), dict(batch=5), dict(kept=None), dict(kept=HERE + 4), dict(kv=b.ls_kv(None, HERE, HERE)),
                  dict(kv=b.ls_kv(HERE, HERE, None)), dict(kv=b.ls_kv(HERE + 2, HERE, HERE))):
        assert keep(**wrong) == b.LS_ERR_INVALID_ARG, wrong


def select(logits=HERE, scores=HERE, ended=None, groups=2, beams=3, vocab=10, k=4, eos=0, rows=HERE, tokens=HERE, best=HERE, scratch=HERE, nb=1 << 30):
    return b.lib.ls_beam_select(logits, scores, ended, groups, beams, vocab, k, eos, rows, tokens, best, scratch, nb, None)


@pytest.mark.parametrize("wrong", [dict(groups=0), dict(beams=0), dict(beams=65), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(k=0), dict(k=65), dict(k=31),
                                   dict(logits=None), dict(scores=None), dict(rows=None), dict(tokens=None), dict(best=None), dict(scratch=None),
                                   dict(scratch=HERE + 8), dict(logits=HERE + 2), dict(ended=HERE, eos=-1), dict(ended=HERE, eos=10)], ids=str)
def test_select(wrong):
    assert select(**wrong) == b.LS_ERR_INVALID_ARG
    assert b"ls_beam_select" in b.lib.ls_last_error()


def test_select_scratch():
    assert select(nb=b.lib.ls_beam_select_scratch_bytes(2, 3, 10, 4) - 1) == b.LS_ERR_OOM
    assert b.lib.ls_beam_select_scratch_bytes(0, 3, 10, 4) == 0 and b.lib.ls_beam_select_scratch_bytes(2, 3, 10, 31) == 0


@pytest.mark.parametrize("wrong", [dict(layers=0), dict(layers=1 << 20), dict(batch=0), dict(batch=6), dict(group=0), dict(group=65), dict(group=3), dict(max_ctx=-1),
                                   dict(max_ctx=101), dict(src=None), dict(kv=(None, HERE, HERE)), dict(kv=(HERE, HERE, None)), dict(kv=(HERE, HERE + 2, HERE))], ids=str)
def test_reorder(wrong):
    v = dict(layers=2, src=HERE, batch=4, group=2, max_ctx=50, kv=(HERE, HERE, HERE))
    v.update(wrong)
    kv = b.ls_kv(*v["kv"])
    assert b.lib.ls_kv_reorder(C.byref(heads()), v["layers"], v["src"], v["batch"], v["group"], None, v["max_ctx"], C.byref(kv), None) == b.LS_ERR_INVALID_ARG


def test_tensors_on_the_host_are_refused():
    import torch

    with pytest.raises(ValueError):
        b.beam_select(torch.zeros(4, 10), torch.zeros(4), beams=2, k=2)
    with pytest.raises(ValueError):
        b.tree_accept(*[torch.zeros(3, dtype=torch.int32)] * 3, torch.zeros(2, dtype=torch.int32), [0, 3])


@pytest.mark.parametrize("wrong", [dict(groups=1 << 22), dict(groups=1 << 20, beams=16)], ids=str)
def test_selections_that_no_launch_takes(wrong):
    assert select(**wrong) == b.LS_ERR_INVALID_ARG and b.lib.ls_beam_select_scratch_bytes(wrong["groups"], wrong.get("beams", 3), 10, 4) == 0


def test_batches_that_no_launch_takes():
    assert b.lib.ls_kv_reorder(C.byref(heads(max_batch=1 << 24)), 1, HERE, 4, 2, None, 50, C.byref(b.ls_kv(HERE, HERE, HERE)), None) == b.LS_ERR_INVALID_ARG
