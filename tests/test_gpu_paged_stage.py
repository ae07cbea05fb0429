"""A stage's generation steps over a cache in pages (ls_stage_paged): what plain generation steps say, prompts filled in from the stage's
own cache, streams, graphs, refusals."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

import synth
from helpers import check_close, make_gpu, make_oracle, to_dev, to_host

pytestmark = pytest.mark.gpu

F32 = synth.CONFIGS["tiny_f32"]
BF16 = synth.StageShape("bf16", 2, 512, 8, 2, 128, 1408, 1000)
GENERIC = synth.StageShape("f32", 2, 96, 4, 2, 24, 160, 77)  # no kernel but those for every shape
WIDE = synth.StageShape("bf16", 2, 256, 2, 2, 64, 512, 301)  # logits of an odd width
SHAPES = pytest.mark.parametrize("shape", [F32, BF16, GENERIC, WIDE], ids=["f32", "bf16", "generic", "wide"])


def pools(st, lengths, room, page=8, weighed=False):
    """A PagedCache with pages for the sequences' lengths and `room` more, in a scattered order."""
    from paper_2502_09922_amd import PagedCache

    need = [-(-(n + room) // page) for n in lengths]
    order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(1)).int().tolist()
    table = torch.full((len(lengths), max(need)), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
    k, _ = st.caches()
    size = (k.shape[0], sum(need), k.shape[2], page, k.shape[4])
    nan = lambda: torch.full(size, math.nan, dtype=k.dtype, device="cuda")  # noqa: E731
    zeros = lambda: torch.zeros(len(lengths), dtype=torch.int32, device="cuda")  # noqa: E731
    more = (torch.zeros(size[:-1], device="cuda"), torch.zeros(size[:-1], dtype=torch.int32, device="cuda")) if weighed else (None, None)
    return PagedCache(nan(), nan(), table.cuda(), zeros(), zeros(), *more)


def ready(shape, lengths, room=12, weighed=False, seq=60):
    from paper_2502_09922_amd import paged_fill

    st = make_gpu(shape, 3, 0, 2, len(lengths), seq, 60)
    prompt = to_dev(shape, np.concatenate([synth.token_ids(20 + b, n, shape.vocab) for b, n in enumerate(lengths)]))
    said = st.prefill(prompt, lengths)
    cache = pools(st, lengths, room, weighed=weighed)
    paged_fill(cache, *st.caches(), st.seq_lens, torch.arange(len(lengths), dtype=torch.int32).cuda(), max(lengths))
    torch.cuda.synchronize()
    assert cache.lens.tolist() == cache.positions.tolist() == list(lengths)
    return st, cache, said


@SHAPES
@pytest.mark.parametrize("weighed", [False, True], ids=["", "weighed"])
@pytest.mark.parametrize("lengths", [[9], [9, 30, 14]], ids=str)
def test_steps_equal_those_over_the_stages_own_cache(shape, lengths, weighed):
    st, cache, said = ready(shape, lengths, weighed=weighed)
    B = len(lengths)
    ora = make_oracle(shape, 3, 0, 2, B, 60)
    said_o, _ = ora.prefill(np.concatenate([synth.token_ids(20 + b, n, shape.vocab) for b, n in enumerate(lengths)]), lengths)
    for step in range(10):
        feed = to_dev(shape, np.asarray(said_o, np.int32))
        got, logits = st.paged(feed, cache, max(lengths) + step, want_logits=True)
        said_o, want = ora.decode(np.asarray(said_o, np.int32))
        torch.cuda.synchronize()
        check_close(to_host(logits), want, shape.dtype, "paged %s step %d" % (shape.dtype, step))
        assert torch.equal(got, logits.argmax(1).int())
        if shape.dtype == "f32":
            assert got.tolist() == list(said_o)
        assert cache.lens.tolist() == cache.positions.tolist() == [n + step + 1 for n in lengths]
    if weighed:  # every step's new token gives each query head's weight of one away, in all layers
        total = float(cache.weights.double().sum())
        assert abs(total - 10 * B * 2 * shape.n_q_heads) <= 1e-4 * total
    st.close()


@SHAPES
def test_a_middle_stage(shape):
    """Hidden rows in and out, without embedding and head."""
    shape = shape.with_(vocab=0)
    from paper_2502_09922_amd import paged_fill

    lengths = [7, 20]
    st = make_gpu(shape, 5, 0, 2, 2, 40, 40)
    ora = make_oracle(shape, 5, 0, 2, 2, 40)
    x = synth.hidden_states(shape, 6, sum(lengths))
    st.prefill(to_dev(shape, x), lengths)
    ora.prefill(x, lengths)
    cache = pools(st, lengths, 8)
    paged_fill(cache, *st.caches(), st.seq_lens, torch.arange(2, dtype=torch.int32).cuda(), 20)
    for step in range(4):
        x = synth.hidden_states(shape, 7 + step, 2)
        got = st.paged(to_dev(shape, x), cache, 20 + step)
        want = ora.decode(x)
        want = want[0] if isinstance(want, tuple) else want
        check_close(to_host(got), want, shape.dtype, "paged middle %s step %d" % (shape.dtype, step))
    st.close()


@SHAPES
def test_sequences_without_room_and_without_part(shape):
    """One takes no part, one has no page for its next slot: both stay as they are, and the third is not touched by them."""
    lengths = [9, 16, 14]
    st, cache, _ = ready(shape, lengths, room=8)
    feed = to_dev(shape, synth.token_ids(50, 3, shape.vocab))
    alone = st.paged(feed, cache, 16, want_logits=True)[1]
    torch.cuda.synchronize()
    cache.lens.copy_(torch.tensor([-1, 16, 14], dtype=torch.int32))
    cache.positions.copy_(torch.tensor([9, 16, 14], dtype=torch.int32))
    cache.table[1, 2] = -1
    out, logits = st.paged(feed, cache, 16, want_logits=True)
    torch.cuda.synchronize()
    assert cache.lens.tolist() == [-1, 16, 15] and cache.positions.tolist() == [9, 16, 15]
    assert torch.equal(logits[2], alone[2])
    st.close()


def test_generation_at_a_budget():
    """Steps over a cache that is cut down all the time: positions go on, tokens far back fall out, the run is the same when replayed."""
    from paper_2502_09922_amd import paged_evict

    runs = []
    for _ in range(2):
        st, cache, said = ready(BF16, [30, 20], room=8, weighed=True, seq=100)
        tokens = []
        for step in range(40):
            said = st.paged(said, cache, 32)
            paged_evict(cache, keep=30, recent=8, first=2, max_len=33)
            tokens.append(said.tolist())
        torch.cuda.synchronize()
        assert cache.lens.tolist() == [30, 30] and cache.positions.tolist() == [70, 60]
        for b, pos in enumerate((70, 60)):
            slot = torch.arange(30)
            places = cache.places.cpu()[:, cache.table.cpu()[b].long()[slot // 8], :, slot % 8]  # [30][layers][heads]
            assert all(len(set(places[:, l, h].tolist())) == 30 for l in range(2) for h in range(2))
            assert ((places < 2).sum(0) == 2).all() and ((places >= pos - 8).sum(0) == 8).all()
        runs.append(tokens)
        st.close()
    assert runs[0] == runs[1]


@pytest.mark.parametrize("by_hand", [False, True], ids=["current", "given"])
def test_on_a_stream_of_its_own(by_hand):
    st, cache, _ = ready(F32, [9, 30])
    feeds = [to_dev(F32, synth.token_ids(60 + i, 2, F32.vocab)) for i in range(3)]
    want = [st.paged(f, cache, 30 + i).tolist() for i, f in enumerate(feeds)]
    cache.lens.copy_(torch.tensor([9, 30], dtype=torch.int32))
    cache.positions.copy_(cache.lens)
    side, feed = torch.cuda.Stream(), feeds[2].clone()
    torch.cuda.synchronize()
    for i in range(3):
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
            feed.copy_(feeds[i])
            said = st.paged(feed, cache, 30 + i, stream=side if by_hand else None)
        side.synchronize()
        assert said.tolist() == want[i]
    st.close()


@pytest.mark.parametrize("weighed", [False, True], ids=["", "weighed"])
def test_captured(weighed):
    """A captured step goes on generating: lengths grow on the device.  Eager steps of another cache between the replays."""
    st, cache, said = ready(BF16, [9, 20], weighed=weighed)
    other = pools(st, [9, 20], 12, weighed=weighed)
    from paper_2502_09922_amd import paged_fill

    paged_fill(other, *st.caches(), st.seq_lens, torch.arange(2, dtype=torch.int32).cuda(), 20)
    feed, eager = said.clone(), said.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = st.paged(feed, cache, 31)
        feed.copy_(out)
    for step in range(6):
        graph.replay()
        torch.cuda.synchronize()
        eager = st.paged(eager, other, 31)
        torch.cuda.synchronize()
        assert feed.tolist() == eager.tolist()
    assert cache.lens.tolist() == other.lens.tolist() == [15, 26]
    for n in ("k", "v", "weights", "places"):
        if getattr(cache, n) is not None:  # the same but for where the pages lie: slot by slot
            for b, m in enumerate((15, 26)):
                slot = torch.arange(m).cuda()
                a, e = (getattr(x, n)[:, x.table[b].long()[slot // 8], :, slot % 8] for x in (cache, other))
                assert torch.equal(a, e), n
    st.close()


def test_refusals():
    from paper_2502_09922_amd import LsError, PagedCache, binding as b

    st, cache, said = ready(F32, [9, 20])
    pages, h = cache._all, st.handle
    call = lambda s=h, x=said.data_ptr(), batch=2, ctx=20, p=pages, out=said.data_ptr(), scratch=None, nb=0: b.lib.ls_stage_paged(  # noqa: E731
        s, x, batch, ctx, p, out, None, scratch, nb, None)
    assert call(x=None) == call(out=None) == call(batch=0) == call(batch=3) == call(ctx=-1) == call(p=None) == b.LS_ERR_INVALID_ARG
    assert call(ctx=32) == b.LS_ERR_KV_OVERFLOW  # 4 pages of 8 slots
    no_positions = b.ls_pages(*[None if n == "positions" else getattr(pages, n) for n, _ in b.ls_pages._fields_])
    no_positions.columns = 100
    assert call(p=no_positions, ctx=60) == b.LS_ERR_KV_OVERFLOW  # the stage has 60 positions
    weighed = pools(st, [9, 20], 12, weighed=True)
    assert call(p=weighed._all) == b.LS_ERR_OOM
    middle = make_gpu(F32.with_(vocab=0), 5, 0, 2, 2, 40, 40, load=False)
    assert call(s=middle.handle) == b.LS_ERR_NOT_LOADED
    with pytest.raises(ValueError):
        st.paged(said.float(), cache, 20)
    with pytest.raises(ValueError):
        st.paged(said, pools(middle, [9, 20], 12).__class__(cache.k[:1].contiguous(), cache.v[:1].contiguous(), cache.table, cache.lens), 20)
    with pytest.raises(LsError):
        st.paged(said, cache, 32)
    with pytest.raises(ValueError):
        PagedCache(cache.k, cache.v, cache.table, cache.lens, weights=torch.zeros(1).cuda())
    torch.cuda.synchronize()
    assert cache.lens.tolist() == [9, 20]
    middle.close()
    st.close()
