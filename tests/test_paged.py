"""What ls_paged_attention, ls_paged_fill, ls_paged_evict and ls_stage_paged refuse, before they touch a device."""
import pytest
import torch

from paper_2502_09922_amd import binding as b

HERE = 4096  # an aligned address that no refused call looks at


def heads(**kw):
    v = dict(dtype=b.LS_DTYPE_BF16, n_q_heads=8, n_kv_heads=2, head_dim=128, max_batch=4, max_seq=100)
    v.update(kw)
    return b.ls_heads(*[v[n] for n, _ in b.ls_heads._fields_])


def pages(**kw):
    v = dict(k=HERE, v=HERE, weights=None, places=None, lens=HERE, positions=None, table=HERE, pages=50, page=16, columns=8)
    v.update(kw)
    return b.ls_pages(*[v[n] for n, _ in b.ls_pages._fields_])


WEIGHED = dict(weights=HERE, places=HERE, positions=HERE + 4096)


def attention(h=None, p=None, batch=3, max_ctx=36, qkv=HERE, rope=HERE, out=HERE + (1 << 20), scratch=None, nb=0):
    return b.lib.ls_paged_attention(h or heads(), p, batch, max_ctx, qkv, rope, out, scratch, nb, None)


def fill(h=None, layers=2, kv=(HERE, HERE, HERE + 8192), from_batch=3, from_seq=64, src=HERE, weights=None, max_len=64, p=None, batch=3):
    return b.lib.ls_paged_fill(h or heads(), layers, None if kv is None else b.ls_kv(*kv), from_batch, from_seq, src, weights, max_len, p, batch, None)


def evict(h=None, layers=2, p=None, batch=3, keep=40, first=2, recent=8, max_len=64, scratch=HERE, nb=1 << 40):
    return b.lib.ls_paged_evict(h or heads(), layers, p, batch, keep, first, recent, max_len, scratch, nb, None)


@pytest.mark.parametrize("wrong", [dict(dtype=2), dict(n_kv_heads=3), dict(n_kv_heads=0), dict(head_dim=0), dict(head_dim=65), dict(head_dim=258),
                                   dict(max_batch=0), dict(max_seq=0), dict(max_seq=(1 << 24) + 1)], ids=str)
def test_heads(wrong):
    h = heads(**wrong)
    assert attention(h, pages()) == fill(h, p=pages()) == evict(h, p=pages(**WEIGHED)) == b.LS_ERR_INVALID_ARG
    assert b.lib.ls_paged_attention_scratch_bytes(h, pages(**WEIGHED), 3, 36) == b.lib.ls_paged_evict_scratch_bytes(h, 2, 3, 40, 64) == 0


@pytest.mark.parametrize("wrong", [dict(k=None), dict(v=None), dict(lens=None), dict(table=None), dict(pages=0), dict(pages=(1 << 24) + 1), dict(page=0), dict(page=4),
                                   dict(page=24), dict(page=2048), dict(columns=0), dict(columns=(1 << 20) + 1), dict(weights=HERE), dict(places=HERE),
                                   dict(k=HERE + 1), dict(v=HERE + 1), dict(lens=HERE + 2), dict(table=HERE + 2), dict(positions=HERE + 2),
                                   dict(weights=HERE + 2, places=HERE), dict(weights=HERE, places=HERE + 2)], ids=str)
def test_pages(wrong):
    p = pages(**wrong)
    assert attention(p=p) == fill(p=p) == b.LS_ERR_INVALID_ARG
    assert b.lib.ls_paged_attention_scratch_bytes(heads(), p, 3, 36) == 0
    p = pages(**{**WEIGHED, **wrong})
    if wrong not in (dict(weights=HERE), dict(places=HERE)):
        assert evict(p=p) == b.LS_ERR_INVALID_ARG


@pytest.mark.parametrize("batch", [0, -1, 5])
def test_batches(batch):
    assert attention(p=pages(), batch=batch) == fill(p=pages(), batch=batch) == evict(p=pages(**WEIGHED), batch=batch) == b.LS_ERR_INVALID_ARG


def test_batches_that_no_launch_takes():
    h = heads(max_batch=1 << 20)
    assert attention(h, pages(), batch=65536) == fill(h, p=pages(), batch=65536) == evict(h, p=pages(**WEIGHED), batch=65536) == b.LS_ERR_INVALID_ARG


@pytest.mark.parametrize("wrong", [dict(max_ctx=-1), dict(qkv=None), dict(out=None), dict(qkv=HERE + 1), dict(out=HERE + (1 << 20) + 1), dict(rope=HERE + 4)], ids=str)
def test_attention(wrong):
    assert attention(p=pages(), **wrong) == b.LS_ERR_INVALID_ARG
    assert b"ls_paged_attention" in b.lib.ls_last_error()
    assert attention(p=None) == b.LS_ERR_INVALID_ARG


def test_contexts_that_do_not_fit():
    assert attention(p=pages(), max_ctx=128) == b.LS_ERR_KV_OVERFLOW  # 8 pages of 16 slots
    assert attention(p=pages(), max_ctx=100) == b.LS_ERR_KV_OVERFLOW  # 100 positions, the new token's would be the 101st
    assert attention(p=pages(positions=HERE + 4096), max_ctx=2**31 - 1) == b.LS_ERR_KV_OVERFLOW
    assert b.lib.ls_paged_attention_scratch_bytes(heads(), pages(**WEIGHED), 3, 128) == 0


def test_weighed_attention_wants_its_scratch():
    p = pages(**WEIGHED)
    need = b.lib.ls_paged_attention_scratch_bytes(heads(), p, 3, 36)
    assert need > 0
    assert attention(p=p) == attention(p=p, scratch=HERE, nb=need - 1) == b.LS_ERR_OOM
    assert attention(p=p, scratch=HERE + 8, nb=need) == b.LS_ERR_INVALID_ARG


@pytest.mark.parametrize("wrong", [dict(layers=0), dict(layers=1 << 24), dict(kv=None), dict(kv=(None, HERE, HERE + 8192)), dict(kv=(HERE, None, HERE + 8192)), dict(kv=(HERE, HERE, None)),
                                   dict(from_batch=0), dict(from_batch=1 << 24), dict(from_seq=0), dict(from_seq=(1 << 24) + 1), dict(src=None), dict(src=HERE + 2),
                                   dict(weights=HERE + 2), dict(max_len=-1), dict(kv=(HERE + 2, HERE, HERE + 8192)), dict(kv=(HERE, HERE + 2, HERE + 8192))], ids=str)
def test_fill(wrong):
    assert fill(p=pages(), **wrong) == b.LS_ERR_INVALID_ARG
    assert b"ls_paged_fill" in b.lib.ls_last_error()
    assert fill(p=pages(k=HERE + 2)) == b.LS_ERR_INVALID_ARG and fill(p=None) == b.LS_ERR_INVALID_ARG


@pytest.mark.parametrize("wrong", [dict(layers=0), dict(layers=1 << 24), dict(layers=1 << 20), dict(keep=0), dict(first=-1), dict(recent=-1), dict(first=20, recent=21),
                                   dict(first=2**31 - 1, recent=2**31 - 1), dict(max_len=-1), dict(max_len=(1 << 24) + 1), dict(scratch=HERE + 8)], ids=str)
def test_evict(wrong):
    assert evict(p=pages(**WEIGHED), **wrong) == b.LS_ERR_INVALID_ARG
    assert b"ls_paged_evict" in b.lib.ls_last_error()


def test_evict_scratch_and_weights():
    p, need = pages(**WEIGHED), b.lib.ls_paged_evict_scratch_bytes(heads(), 2, 3, 40, 64)
    assert need > 0
    assert evict(p=p, scratch=None) == evict(p=p, nb=need - 1) == b.LS_ERR_OOM
    assert evict(p=pages()) == b.LS_ERR_INVALID_ARG  # nothing to go by
    assert evict(p=pages(**WEIGHED, k=HERE + 2)) == b.LS_ERR_INVALID_ARG
    assert evict(p=p, keep=64) == evict(p=p, keep=2**31 - 1, first=0, recent=0) == b.LS_OK  # no sequence has more: nothing to do


def test_buffers_that_are_one():
    """What a call writes is not what it reads: lengths that are positions would count twice, lengths of a prompt's cache that are those of the
    pages would change under those who read them, and rows that are written would be queries of others."""
    twice = pages(**{**WEIGHED, "positions": HERE})
    near = pages(**{**WEIGHED, "positions": HERE + 4 * 3})  # max_batch entries of each
    for p in (twice, near):
        assert attention(p=p) == fill(p=p) == evict(p=p) == b.LS_ERR_INVALID_ARG
        assert b"one buffer" in b.lib.ls_last_error()
    p = pages(**WEIGHED)
    for lens in (HERE, HERE + 4 * 2, HERE - 4 * 2, HERE + 4096):
        assert fill(p=p, kv=(HERE, HERE, lens)) == b.LS_ERR_INVALID_ARG
        assert b"seq_lens overlaps" in b.lib.ls_last_error()
    h = heads()
    row = h.head_dim * (4 if h.dtype == b.LS_DTYPE_F32 else 2)
    far = HERE + (1 << 20)
    for out in (far, far + 3 * row * (h.n_q_heads + 2 * h.n_kv_heads) - 16, far - 3 * row * h.n_q_heads + 16):
        assert attention(p=pages(), qkv=far, out=out) == b.LS_ERR_INVALID_ARG
        assert b"out overlaps" in b.lib.ls_last_error()


def test_evictions_want_positions():
    """Without them the next token's would be its slot, which an eviction changes."""
    assert evict(p=pages(**{**WEIGHED, "positions": None})) == b.LS_ERR_INVALID_ARG
    assert b"positions" in b.lib.ls_last_error()


def test_weights_of_more_slots_than_a_launch_takes():
    h, p = heads(n_q_heads=512, n_kv_heads=512, max_seq=1 << 24), pages(**WEIGHED, page=1024, columns=1 << 14)
    assert b.lib.ls_paged_attention_scratch_bytes(h, p, 3, (1 << 24) - 1) == 0
    assert attention(h, p, max_ctx=(1 << 24) - 1, scratch=HERE, nb=1 << 60) == b.LS_ERR_INVALID_ARG
    assert b.lib.ls_paged_attention_scratch_bytes(h, p, 3, 1 << 22) > 0


def test_stage():
    assert b.lib.ls_stage_paged(None, HERE, 1, 0, pages(), HERE, None, None, 0, None) == b.LS_ERR_INVALID_ARG


def test_tensors_on_the_host_are_refused():
    k = torch.zeros(1, 4, 2, 8, 16)
    with pytest.raises(ValueError):
        b.PagedCache(k, k.clone(), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
