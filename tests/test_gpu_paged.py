"""A cache in pages (ls_paged_attention, ls_paged_fill, ls_paged_evict) against plain 64-bit arithmetic."""
import copy
import math
import random

import pytest
import torch

import paged_plain as plain

pytestmark = pytest.mark.gpu

TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
WEIGHED = pytest.mark.parametrize("weighed", [False, True], ids=["", "weighed"])
HEADS = [(4, 4, 64), (4, 4, 128), (8, 2, 128), (8, 1, 128), (16, 2, 64), (32, 1, 64), (20, 1, 128), (3, 1, 128), (6, 2, 80), (2, 1, 256), (5, 5, 2)]


def attend(c, rope, layer=0, max_ctx=None, cache=None, **kw):
    """(the cache behind the call as Pages on the host, output rows)."""
    from paper_2502_09922_amd import paged_attention

    cache = c.on_gpu() if cache is None else cache
    out = paged_attention(cache, c.qkv[layer].cuda(), None if rope is None else rope.cuda(), max(0, int(c.lens.max())) if max_ctx is None else max_ctx, layer=layer, **kw)
    torch.cuda.synchronize()
    got = copy.copy(c)
    got.take(cache)
    return got, out.cpu()


def check(c, rope, layer=0, **kw):
    got, out = attend(c, rope, layer, **kw)
    plain.check_attention(c, layer, rope, got, out)
    return got, out


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%dx%dx%d" % h)
def test_ragged_sequences(heads, dtype, weighed):
    c = plain.Pages(heads, dtype, [0, 1, 15, 16, 17, 31, 33, 100, 7], 16, seed=1, weighed=weighed)
    check(c, plain.rope_table(128, heads[2]))


@TYPES
@WEIGHED
@pytest.mark.parametrize("page", [8, 16, 32, 64, 1024])
@pytest.mark.parametrize("heads", [(2, 2, 128), (8, 1, 64), (3, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
def test_pages_of_all_sizes(heads, page, dtype, weighed):
    c = plain.Pages(heads, dtype, [63, 0, 8, 130, 64, 7], page, seed=page, weighed=weighed)
    check(c, plain.rope_table(140, heads[2]))


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", [(2, 2, 128), (8, 1, 128), (4, 1, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("ctx", [600, 1023, 2500])
def test_long_contexts(heads, ctx, dtype, weighed):
    """Contexts that several workgroups share; without weights an understated bound of their length costs speed alone."""
    c = plain.Pages(heads, dtype, [ctx, 7, ctx // 2], 16, seed=ctx, weighed=weighed)
    rope = plain.rope_table(ctx + 5, heads[2])
    check(c, rope)
    if not weighed:
        check(c, rope, max_ctx=40)


@TYPES
@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 2, 80)], ids=lambda h: "%dx%dx%d" % h)
def test_sequences_beyond_the_bound_of_a_weighed_call(heads, dtype):
    c = plain.Pages(heads, dtype, [40, 41, 90, 3], 8, seed=3, weighed=True)
    got, out = attend(c, None, max_ctx=40)
    left = copy.deepcopy(c)
    left.lens[1] = left.lens[2] = -1  # as ones without room
    got.lens, got.positions = left.lens, left.positions
    plain.check_attention(left, 0, None, got, out)


@TYPES
@WEIGHED
def test_many_sequences(dtype, weighed):
    r = random.Random(4)
    c = plain.Pages((8, 2, 64), dtype, [r.choice([0, 1, 5, 30, 64, 200]) for _ in range(300)], 16, seed=4, weighed=weighed)
    check(c, plain.rope_table(210, 64))


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
def test_sequences_without_room(heads, dtype, weighed):
    """Negative lengths, lengths at and behind the table's end, a slot whose page is not named or lies outside the pool, positions that are
    negative or that the table of angles does not have."""
    c = plain.Pages(heads, dtype, [20, 30, 31, 32, 9, 12, 13, 14], 16, seed=5, weighed=weighed)
    c.lens[0] = -3
    c.lens[1], c.lens[2] = c.table.shape[1] * 16, 2**31 - 1
    c.table[3, 2] = c.k.shape[1]
    c.table[4, 0] = -2**31
    c.positions[5], c.positions[6] = -1, 60
    c.positions[1] = c.positions[2] = 5
    rope = plain.rope_table(60, heads[2])
    check(c, rope, max_ctx=c.table.shape[1] * 16 - 1)
    assert [c.room(b, 60) for b in range(8)] == [False] * 7 + [True]


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
def test_slots_without_a_page_are_not_there(heads, dtype, weighed):
    c = plain.Pages(heads, dtype, [100, 100, 40], 8, seed=6, weighed=weighed)
    c.table[0, 3], c.table[0, 0], c.table[1, 5:11], c.table[2, :5] = -1, c.k.shape[1], 2**31 - 1, -5
    check(c, plain.rope_table(110, heads[2]))


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
def test_positions_of_their_own_and_turned_rows(heads, dtype, weighed):
    c = plain.Pages(heads, dtype, [40, 3, 17], 8, seed=7, weighed=weighed)
    c.positions = torch.tensor([900, 3, 0], dtype=torch.int32)
    check(c, plain.rope_table(901, heads[2]))
    c.positions[0] = 2**31 - 1  # rows that come turned may stand anywhere
    check(c, None)


@TYPES
@pytest.mark.parametrize("heads", [(8, 2, 128), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
def test_without_positions(heads, dtype):
    from paper_2502_09922_amd import PagedCache, paged_attention

    c = plain.Pages(heads, dtype, [40, 0, 17], 8, seed=8)
    t = {n: x.cuda() for n, x in c.tensors().items() if x is not None and n != "positions"}
    cache, rope = PagedCache(**t), plain.rope_table(50, heads[2])
    out = paged_attention(cache, c.qkv[0].cuda(), rope.cuda(), 40).cpu()
    got = copy.copy(c)
    got.k, got.v, got.lens = cache.k.cpu(), cache.v.cpu(), cache.lens.cpu()
    plain.check_attention(c, 0, rope, got, out)


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", [(4, 2, 128), (8, 1, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_nonfinite_rows_stay_in_their_sequence(heads, dtype, weighed, bad):
    """A cached key, a cached value, a new row and a query that are no numbers, each in a sequence of its own beside a sound one; what a
    softmax over them gives.  (Keys infinite along every query: signs of single products do not matter.)"""
    c = plain.Pages(heads, dtype, [50, 50, 50, 50, 50], 16, seed=9, weighed=weighed)
    hq, hkv, hd = heads
    rows = c.qkv[0].view(5, hq + 2 * hkv, hd)
    rows[0, :hq, 0] = 1.0  # queries that see an infinite key all from one side, as rows come turned
    c.k[c.at(0, 0, 20)][:, 0] = bad
    c.v[c.at(0, 1, 20)][:, 5] = bad
    rows[2, hq + hkv :, 3] = bad
    rows[3, 1, 2] = math.nan
    got, out = attend(c, None)
    # sums against keys and values that are no numbers, in plain arithmetic
    plain.check_attention(c, 0, None, got, out)
    assert out[4].isfinite().all()


@TYPES
@WEIGHED
def test_scores_of_the_types_lowest_values(dtype, weighed):
    """Scores around the lowest finite ones and -inf for all but the new row: no weight, no NaN."""
    c = plain.Pages((4, 2, 128), dtype, [70, 33], 16, seed=10, weighed=weighed)
    c.qkv[0].view(2, 8, 128)[:, :6] = 0
    c.qkv[0].view(2, 8, 128)[:, :4, 0] = 1.0
    for i in range(60):
        c.k[c.at(0, 0, i)][:, 0] = torch.finfo(dtype).min if i % 2 else -math.inf
    for i in range(33):
        c.k[c.at(0, 1, i)][:, 0] = -math.inf
    got, out = check(c, None)
    assert out.isfinite().all()


@TYPES
@WEIGHED
def test_one_key_with_all_the_weight(dtype, weighed):
    """Large scores: the maximum moves late, and by far."""
    c = plain.Pages((4, 1, 128), dtype, [900, 64], 16, seed=11, weighed=weighed)
    c.k[c.at(0, 0, 700)] *= 30
    c.k[c.at(0, 1, 1)] *= 30
    check(c, None)


@TYPES
@WEIGHED
@pytest.mark.parametrize("what", ["qkv", "k", "v", "out", "rope"])
def test_buffers_off_16_bytes(what, dtype, weighed):
    from paper_2502_09922_amd import PagedCache, paged_attention

    def off(t):
        flat = torch.empty(t.numel() + 2, dtype=t.dtype, device="cuda")
        flat = flat[1 if t.dtype == torch.bfloat16 or what != "rope" else 2 :][: t.numel()].view(t.shape)
        return flat.copy_(t)

    c = plain.Pages((8, 2, 128), dtype, [40, 3, 170], 16, seed=12, weighed=weighed)
    rope, t = plain.rope_table(180, 128), {n: None if x is None else x.cuda() for n, x in c.tensors().items()}
    if what in t:
        t[what] = off(t[what])
    cache = PagedCache(**t)
    out = off(torch.empty(3, 8 * 128, dtype=dtype)) if what == "out" else None
    out = paged_attention(cache, off(c.qkv[0]) if what == "qkv" else c.qkv[0].cuda(), off(rope) if what == "rope" else rope.cuda(), 170, out=out)
    got = copy.copy(c)
    got.take(cache)
    plain.check_attention(c, 0, rope, got, out.cpu())


@TYPES
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
def test_scratch_of_any_size(heads, dtype):
    from paper_2502_09922_amd import binding as b

    c = plain.Pages(heads, dtype, [1500, 90], 16, seed=13)
    rope, hq = plain.rope_table(1510, heads[2]).cuda(), heads[0]
    cache = c.on_gpu()
    h, pages = cache.heads(hq, 1510), cache._layers[0]
    need = b.lib.ls_paged_attention_scratch_bytes(h, pages, 2, 1500)
    scratch = torch.empty(need + 64, dtype=torch.uint8, device="cuda")
    qkv = c.qkv[0].cuda()
    for nb in (0, 16, need // 3, need - 1, need, need + 64):
        for at in (0, 4):
            out = torch.full((2, hq * heads[2]), math.nan, dtype=dtype, device="cuda")
            scratch.fill_(255)  # NaN
            assert b.lib.ls_paged_attention(h, pages, 2, 1500, qkv.data_ptr(), rope.data_ptr(), out.data_ptr(), scratch.data_ptr() + at if nb else None,
                                            min(nb, need + 64 - at), 0) == 0
            torch.cuda.synchronize()
            got = copy.copy(c)
            got.take(cache)
            plain.check_attention(c, 0, rope.cpu(), got, out.cpu())
    assert (scratch[need:] == 255).all()


@TYPES
@WEIGHED
def test_layers_of_one_cache(dtype, weighed):
    c = plain.Pages((4, 2, 64), dtype, [50, 9], 8, layers=3, seed=14, weighed=weighed)
    rope, cache = plain.rope_table(60, 64), c.on_gpu()
    for layer in (2, 0, 1):
        got, out = attend(c, rope, layer, cache=cache)
        plain.check_attention(c, layer, rope, got, out)
        c.take(cache)


@TYPES
def test_shared_pages(dtype):
    """Two sequences whose tables begin with the same pages."""
    c = plain.Pages((8, 2, 128), dtype, [48, 50, 20], 16, seed=15)
    c.table[1, :3] = c.table[0, :3]
    for layer in range(1):
        for i in range(48, 50):
            at = c.at(layer, 1, i)
            c.k[at] = c.v[at] = torch.randn(2, 128).to(dtype)
    got, out = attend(c, None)
    for b in (0, 1, 2):  # one after the other in the plain form
        alone = copy.deepcopy(c)
        alone.lens = torch.where(torch.arange(3) == b, c.lens, torch.tensor(-1, dtype=torch.int32))
        g = copy.copy(alone)
        at = c.at(0, b, int(c.lens[b]))
        g.k, g.v = c.k.clone(), c.v.clone()
        g.k[at], g.v[at] = got.k[at], got.v[at]
        masked = torch.zeros_like(out)
        masked[b] = out[b]
        plain.check_attention(alone, 0, None, g, masked)


@TYPES
def test_offsets_beyond_32_bits(dtype):
    """A pool of more than 4 GiB of keys, a sequence in its last pages."""
    from paper_2502_09922_amd import PagedCache, paged_attention

    hq, hkv, hd, page = 8, 8, 128, 64
    pages = (1 << 32) // (hkv * page * hd * dtype.itemsize) + 5
    c = plain.Pages((hq, hkv, hd), dtype, [150], page, seed=16, weighed=True, spare=0)
    own = c.k.shape[1]
    k, v = (torch.empty(1, pages, hkv, page, hd, dtype=dtype, device="cuda") for _ in range(2))
    w, p = torch.zeros(1, pages, hkv, page, device="cuda"), torch.zeros(1, pages, hkv, page, dtype=torch.int32, device="cuda")
    k[:, -own:], v[:, -own:], w[:, -own:], p[:, -own:] = c.k.cuda(), c.v.cuda(), c.weights.cuda(), c.places.cuda()
    table = torch.where(c.table < 0, c.table, c.table + (pages - own)).int().cuda()
    cache = PagedCache(k, v, table, c.lens.cuda(), c.positions.cuda(), w, p)
    out = paged_attention(cache, c.qkv[0].cuda(), None, 150).cpu()
    got = copy.copy(c)
    got.k, got.v, got.weights, got.places = (x[:, -own:].cpu() for x in (k, v, w, p))
    plain.check_attention(c, 0, None, got, out)


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (2, 1, 96)], ids=lambda h: "%dx%dx%d" % h)
def test_replayed_while_sequences_grow(heads, dtype, weighed):
    """A captured step, replayed with the lengths of later steps, eager work and other scratch between the replays."""
    from paper_2502_09922_amd import paged_attention

    c = plain.Pages(heads, dtype, [30, 0, 121], 16, seed=17, weighed=weighed, room=8)
    rope, cache, qkv = plain.rope_table(140, heads[2]), c.on_gpu(), c.qkv[0].cuda()
    turn = rope.cuda()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = paged_attention(cache, qkv, turn, 128)
    for step in range(4):
        qkv.normal_(generator=torch.Generator("cuda").manual_seed(step))
        c.qkv[0] = qkv.cpu()
        graph.replay()
        torch.cuda.synchronize()
        got = copy.copy(c)
        got.take(cache)
        plain.check_attention(c, 0, rope, got, out.cpu())
        c.take(cache)
        cache.lens.add_(1)
        cache.positions.add_(1)
        c.lens, c.positions = cache.lens.cpu(), cache.positions.cpu()
        torch.empty(1 << 22, device="cuda").fill_(math.nan)


def test_streams():
    """Inputs that arrive late on a stream of the caller's; two calls at once on two streams."""
    from paper_2502_09922_amd import paged_attention

    cs = [plain.Pages((8, 2, 128), torch.bfloat16, [700, 30 + i], 16, seed=18 + i, weighed=True) for i in range(2)]
    caches, streams = [c.on_gpu() for c in cs], [torch.cuda.Stream() for _ in cs]
    late = [c.qkv[0].cuda() for c in cs]
    feeds = [torch.full_like(q, math.nan) for q in late]
    torch.cuda.synchronize()
    outs = []
    for cache, feed, q, st in zip(caches, feeds, late, streams):
        with torch.cuda.stream(st):
            torch.cuda._sleep(20_000_000)
            feed.copy_(q)
            outs.append(paged_attention(cache, feed, None, 701))
    torch.cuda.synchronize()
    for c, cache, out in zip(cs, caches, outs):
        got = copy.copy(c)
        got.take(cache)
        plain.check_attention(c, 0, None, got, out.cpu())


# ---- filling -----------------------------------------------------------------------------------------------------------------
def prompts(c, from_batch, from_seq, lens, seed):
    g = torch.Generator().manual_seed(seed)
    hkv, hd = c.heads[1:]
    k, v = (torch.randn(c.layers, from_batch, hkv, from_seq, hd, generator=g).to(c.k.dtype) for _ in range(2))
    return k, v, torch.tensor(lens, dtype=torch.int32), torch.rand(c.layers, from_batch, hkv, from_seq, generator=g)


def equal(c, cache):
    for n, t in c.tensors().items():
        if t is not None:
            assert plain.same(getattr(cache, n).cpu(), t), n


@TYPES
@pytest.mark.parametrize("weighed", ["", "zeros", "weighed"])
@pytest.mark.parametrize("heads", [(2, 2, 128), (8, 4, 64), (3, 3, 6), (5, 1, 90)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("page", [8, 64])
def test_fill(heads, page, dtype, weighed):
    from paper_2502_09922_amd import paged_fill

    c = plain.Pages(heads, dtype, [3, 50, 200, 0, 90, 64, 33, 8], page, layers=2, seed=21, weighed=bool(weighed), spare=1)
    c.table[4, 1] = -1
    k, v, lens, w = prompts(c, 9, 199, [50, 1, 64, 0, 199, 65, 200, -4, 130], 22)
    src = [1, 0, 4, 3, 8, 2, 9, 5]  # one that is none, and prompts longer than the sequence's pages
    for max_len in (199, 20):
        cache = c.on_gpu()
        paged_fill(cache, k.cuda(), v.cuda(), lens.cuda(), torch.tensor(src, dtype=torch.int32).cuda(), max_len, w.cuda() if weighed == "weighed" else None)
        want = copy.deepcopy(c)
        plain.fill(want, k, v, lens, src, w if weighed == "weighed" else None)
        equal(want, cache)
    cache = c.on_gpu()  # nobody: entries outside, and lengths that are none
    paged_fill(cache, k.cuda(), v.cuda(), lens.cuda(), torch.tensor([-1, 6, 7, 9, 2**31 - 1, -2**31, 6, 7], dtype=torch.int32).cuda(), 199)
    equal(c, cache)


# ---- eviction ----------------------------------------------------------------------------------------------------------------
def cut(c, keep, first, recent, max_len):
    from paper_2502_09922_amd import paged_evict

    cache = c.on_gpu()
    paged_evict(cache, keep=keep, recent=recent, first=first, max_len=max_len)
    want = copy.deepcopy(c)
    plain.evict(want, keep, first, recent, max_len)
    equal(want, cache)
    return want


@TYPES
@pytest.mark.parametrize("heads", [(2, 2, 128), (8, 4, 64), (3, 3, 6), (5, 1, 90)], ids=lambda h: "%dx%dx%d" % h)
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 0), (1, 0, 1), (16, 4, 4), (33, 0, 33), (40, 40, 0), (64, 0, 0), (199, 1, 5), (250, 0, 0)])
def test_evict(heads, dtype, keep, first, recent):
    c = plain.Pages(heads, dtype, [200, 33, 34, 1, 0, 65, 201, -1], 8, layers=2, seed=keep, weighed=True)
    cut(c, keep, first, recent, 201)
    cut(c, keep, first, recent, 200)  # a sequence of 201 is left alone


@pytest.mark.parametrize("weights", ["zeros", "few values", "signed", "not numbers", "infinite", "one bit"])
@pytest.mark.parametrize("n", [65, 300, 1025])
def test_equal_and_odd_weights(weights, n):
    """Ties go by the lower slot; a weight that is no number is below all others, -0 is 0."""
    c = plain.Pages((3, 3, 2), torch.float32, [n, n - 1], 16, seed=n, weighed=True)
    g = torch.Generator().manual_seed(n)
    w = torch.rand(c.weights.shape, generator=g)
    if weights == "zeros":
        w = torch.where(w < 0.5, 0.0, -0.0)
    elif weights == "few values":
        w = (w * 4).floor()
    elif weights == "signed":
        w = w - 0.5
    elif weights == "not numbers":
        w = torch.where(w < 0.4, math.nan, w)
        w = torch.where(w > 0.9, -math.nan, w)
    elif weights == "infinite":
        w = torch.where(w < 0.3, -math.inf, torch.where(w > 0.7, math.inf, w))
    else:  # neighbours among the numbers
        w = (torch.ones(w.shape).view(torch.int32) + (w * 3).int()).view(torch.float32)
    c.weights = w
    for keep, first, recent in ((1, 0, 0), (n // 2, 3, 5), (n - 2, 0, 0), (n - 1, 0, 1)):
        cut(c, keep, first, recent, n)


def test_places_in_any_order():
    """Positions of their own for each kv head, more of them protected than stay, and tokens that stand at odd positions."""
    c = plain.Pages((4, 4, 8), torch.float32, [120, 90, 100, 110], 8, layers=2, seed=31, weighed=True)
    g = torch.Generator().manual_seed(31)
    c.places = torch.randint(0, 500, c.places.shape, generator=g).int()
    c.positions = torch.tensor([500, 0, 2**31 - 1, -5], dtype=torch.int32)
    for keep, first, recent in ((20, 0, 20), (60, 30, 30), (10, 10, 0)):
        cut(c, keep, first, recent, 120)


def test_sequences_with_a_page_that_is_none_are_left_alone():
    c = plain.Pages((2, 2, 64), torch.bfloat16, [50, 50, 50, 50], 16, seed=32, weighed=True)
    c.table[0, 0], c.table[1, 3], c.table[2, 3] = -1, c.k.shape[1], c.table[2, 3]
    c.table[3, 4:] = 2**31 - 1  # behind its slots: not looked at
    want = cut(c, 20, 0, 4, 50)
    assert want.lens.tolist() == [50, 50, 20, 20]


@pytest.mark.parametrize("n,keep", [(3000, 512), (9001, 2000), (40000, 39990), (70001, 300)])
def test_long_sequences(n, keep):
    """Slots beyond what a workgroup's registers hold."""
    heads, page = (1, 2, 2), 64
    c = plain.Pages(heads, torch.float32, [1], page, seed=33, weighed=True)
    pages = (n + page - 1) // page
    r = random.Random(n)
    order = list(range(pages))
    r.shuffle(order)
    g = torch.Generator().manual_seed(n)
    c.table, c.lens, c.positions = torch.tensor([order], dtype=torch.int32), torch.tensor([n], dtype=torch.int32), torch.tensor([n], dtype=torch.int32)
    c.k, c.v = (torch.randn(1, pages, 2, page, 2, generator=g) for _ in range(2))
    c.weights = (torch.rand(1, pages, 2, page, generator=g) * 5000).floor()
    slot = torch.arange(pages * page).view(pages, page).int()
    c.places = torch.zeros(1, pages, 2, page, dtype=torch.int32)
    for i, p in enumerate(order):
        c.places[0, p] = slot[i]
    cut(c, keep, 4, keep // 4, n)


def test_many_sequences_are_cut_down():
    r = random.Random(5)
    c = plain.Pages((2, 2, 16), torch.bfloat16, [r.choice([0, 1, 20, 40, 41, 64, 90]) for _ in range(300)], 8, seed=34, weighed=True)
    cut(c, 40, 2, 8, 90)


def test_evictions_replayed():
    """A captured eviction, replayed over lengths and weights of its own each time."""
    from paper_2502_09922_amd import paged_evict

    c = plain.Pages((4, 2, 64), torch.bfloat16, [70, 40, 99], 16, layers=2, seed=35, weighed=True)
    cache, graph = c.on_gpu(), torch.cuda.CUDAGraph()
    full = cache.lens.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        paged_evict(cache, keep=41, recent=5, max_len=100)
    for step in range(4):
        cache.lens.copy_(full if step != 2 else full - 20)
        cache.weights.uniform_(generator=torch.Generator("cuda").manual_seed(step))
        c.take(cache)
        graph.replay()
        torch.cuda.synchronize()
        plain.evict(c, 41, 0, 5, 100)
        equal(c, cache)
        torch.empty(1 << 22, device="cuda").fill_(math.nan)


# ---- together ----------------------------------------------------------------------------------------------------------------
@TYPES
@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64), (6, 2, 80)], ids=lambda h: "%dx%dx%d" % h)
def test_a_run_at_a_budget(heads, dtype):
    """Prompts into pages, cut down, then steps that attend in every layer, add weights up, and evict one slot each: every call
    against the plain form of what it found."""
    from paper_2502_09922_amd import paged_evict, paged_fill

    layers, keep, page = 2, 40, 16
    c = plain.Pages(heads, dtype, [100, 64, 20], page, layers=layers, seed=41, weighed=True)
    k, v, lens, w = prompts(c, 3, 100, [20, 100, 64], 42)
    src, rope = [1, 2, 0], plain.rope_table(140, heads[2])
    cache = c.on_gpu()
    paged_fill(cache, k.cuda(), v.cuda(), lens.cuda(), torch.tensor(src, dtype=torch.int32).cuda(), 100, w.cuda())
    plain.fill(c, k, v, lens, src, w)
    equal(c, cache)
    g = torch.Generator().manual_seed(43)
    for step in range(25):
        paged_evict(cache, keep=keep, recent=8, first=2, max_len=100 if step == 0 else keep + 1)
        plain.evict(c, keep, 2, 8, 100)
        equal(c, cache)
        c.qkv = torch.randn(c.qkv.shape, generator=g).to(dtype)
        for layer in range(layers):
            got, out = attend(c, rope, layer, max_ctx=keep, cache=cache)
            plain.check_attention(c, layer, rope, got, out)
            c.take(cache)
        cache.lens.add_(1)
        cache.positions.add_(1)
        c.take(cache)
    # the third has pages for 32 slots: behind them its rows are zeros, and it is not cut down
    assert c.lens.tolist() == [keep + 1, keep + 1, 45] and c.positions.tolist() == [125, 89, 45]


# ---- contexts that are dealt out by their lengths ----------------------------------------------------------------------------
DEALT = pytest.mark.parametrize("heads", [(8, 2, 128), (20, 1, 64), (4, 4, 64), (34, 2, 128)], ids=lambda h: "%dx%dx%d" % h)


@TYPES
@WEIGHED
@DEALT
def test_long_and_short_contexts(heads, dtype, weighed):
    """One long sequence among short ones, some of which take no part, have no room or lack a page."""
    c = plain.Pages(heads, dtype, [40, 6200, 0, 300, 8, 3100, 16, 17, 90], 16, seed=51, weighed=weighed)
    c.lens[4], c.table[6, 1], c.table[5, 7], c.table[1, 100:105] = -1, c.k.shape[1], -1, 2**31 - 1
    c.positions[8] = 6300
    check(c, plain.rope_table(6300, heads[2]))


@TYPES
@WEIGHED
@pytest.mark.parametrize("batch", [2, 64, 65, 256, 300, 1025])
def test_one_long_context_among_many(batch, dtype, weighed):
    """As many sequences as one register, four and sixteen of a wavefront hold the lengths of, and more."""
    r = random.Random(batch)
    lens = [r.choice([0, 1, 5, 15, 16, 40]) for _ in range(batch)]
    lens[batch // 3] = 6200
    c = plain.Pages((2, 1, 64), dtype, lens, 32, seed=52, weighed=weighed)
    check(c, plain.rope_table(6201, 64))


@TYPES
@WEIGHED
def test_all_long_contexts(dtype, weighed):
    """More pieces than workgroups could take with one each, and none long enough to be cut."""
    c = plain.Pages((4, 4, 128), dtype, [3400 + 7 * i for i in range(6)], 64, seed=53, weighed=weighed)
    check(c, None)


@TYPES
@DEALT
def test_dealt_with_scratch_of_any_size(heads, dtype):
    from paper_2502_09922_amd import binding as b

    c = plain.Pages(heads, dtype, [6200, 20, 700], 64, seed=54)
    rope, hq = plain.rope_table(6210, heads[2]).cuda(), heads[0]
    cache, qkv = c.on_gpu(), c.qkv[0].cuda()
    h, pages = cache.heads(hq, 6210), cache._layers[0]
    need = b.lib.ls_paged_attention_scratch_bytes(h, pages, 3, 6200)
    scratch = torch.empty(need + 64, dtype=torch.uint8, device="cuda")
    for nb in (0, 16, 4096, need // 40, need // 3, need - 1, need):
        out = torch.full((3, hq * heads[2]), math.nan, dtype=dtype, device="cuda")
        scratch.fill_(255)  # NaN
        assert b.lib.ls_paged_attention(h, pages, 3, 6200, qkv.data_ptr(), rope.data_ptr(), out.data_ptr(), scratch.data_ptr(), nb, 0) == 0
        torch.cuda.synchronize()
        assert (scratch[nb:] == 255).all()
        got = copy.copy(c)
        got.take(cache)
        plain.check_attention(c, 0, rope.cpu(), got, out.cpu())


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", [(20, 1, 128), (40, 2, 64), (16, 16, 64)], ids=lambda h: "%dx%dx%d" % h)
def test_pieces_of_more_heads_than_a_block(heads, dtype, weighed):
    c = plain.Pages(heads, dtype, [2500, 1300], 16, seed=55, weighed=weighed)
    check(c, plain.rope_table(2501, heads[2]))


@TYPES
@WEIGHED
@pytest.mark.parametrize("heads", [(4, 2, 128), (40, 2, 128)], ids=lambda h: "%dx%dx%d" % h)
def test_a_workgroup_to_a_sequence(heads, dtype, weighed):
    """More sequences than CUs, of which one is longer than the others by far but for being dealt out."""
    lens = [5] * 140
    lens[70], lens[71] = 1400 if dtype == torch.float32 else 2800, 1025
    c = plain.Pages(heads, dtype, lens, 16, seed=56, weighed=weighed)
    check(c, plain.rope_table(2801, heads[2]))


@pytest.mark.parametrize("weighed", [False, True], ids=["", "weighed"])
def test_dealt_anew_by_each_replay(weighed):
    """A captured call whose sequences' lengths become others."""
    from paper_2502_09922_amd import paged_attention

    c = plain.Pages((8, 2, 128), torch.bfloat16, [3900, 3900, 3900], 64, seed=57, weighed=weighed)
    cache, qkv, graph = c.on_gpu(), c.qkv[0].cuda(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = paged_attention(cache, qkv, None, 3900)
    for lens in ([3900, 3, 100], [0, 0, 0], [-1, 3899, 2000], [3900, 3900, 3900]):
        cache.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.take(cache)
        graph.replay()
        torch.cuda.synchronize()
        got = copy.copy(c)
        got.take(cache)
        plain.check_attention(c, 0, None, got, out.cpu())
        c.take(cache)
        torch.empty(1 << 22, device="cuda").fill_(math.nan)


# ---- eviction, further ---------------------------------------------------------------------------------------------------------
LENGTHS = [(600, 570, 3), (1500, 1469, 20), (3000, 2999, 1), (5000, 4990, 9), (9000, 8968, 0), (12000, 4000, 64), (20000, 19995, 4), (31000, 30970, 100),
           (32768, 5, 5), (32769, 32768, 1)]


@pytest.mark.parametrize("batch,n,keep,recent", [(1,) + x for x in LENGTHS] + [(1100,) + x for x in LENGTHS[:3]])
def test_all_lengths_of_sequences_that_are_cut_down(batch, n, keep, recent):
    """Few moves and many, by one wavefront to sixteen; beside sequences that stay as they are where there are many."""
    page, hkv = 64, 2
    pages = (n + page - 1) // page
    c = plain.Pages((2, hkv, 2), torch.float32, [1], page, seed=61, weighed=True)
    g, order = torch.Generator().manual_seed(n), list(range(pages))
    random.Random(n).shuffle(order)
    c.table = torch.full((batch, pages), 7, dtype=torch.int32)
    c.table[batch // 2] = torch.tensor(order, dtype=torch.int32)
    c.lens = torch.full((batch,), min(5, keep), dtype=torch.int32)
    c.lens[batch // 2] = n
    c.positions = c.lens.clone()
    c.k, c.v = (torch.randn(1, pages, hkv, page, 2, generator=g) for _ in range(2))
    c.weights = torch.randn(1, pages, hkv, page, generator=g).exp() * (torch.rand(1, pages, hkv, page, generator=g) < 0.9)
    c.places = torch.randint(0, n, (1, pages, hkv, page), generator=g).int()
    want = cut(c, keep, 0, recent, n)
    assert int(want.lens[batch // 2]) == keep


@pytest.mark.parametrize("keep,recent,values", [(400, 30, 7), (70000, 0, 1 << 20), (65536, 65536, 3), (20, 20, 1 << 20)])
def test_sequences_beyond_registers_beside_short_ones(keep, recent, values):
    """Long and short ones of a call, equal weights or few, lengths of the bound and below, a sequence that is left alone."""
    page, hkv, lens = 1024, 2, [70000, 500, 131073, 65537, 1, -1]
    c = plain.Pages((2, hkv, 2), torch.float32, [1], page, seed=63, weighed=True)
    need = [max(0, n + page - 1) // page for n in lens]
    g, order = torch.Generator().manual_seed(keep), list(range(sum(need)))
    random.Random(keep).shuffle(order)
    c.table = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        for i in range(n):
            c.table[b, i] = order.pop()
    c.lens = torch.tensor(lens, dtype=torch.int32)
    c.positions = c.lens.clone()
    size = (1, sum(need), hkv, page)
    c.k, c.v = (torch.randn(size + (2,), generator=g) for _ in range(2))
    c.weights = torch.randint(0, values, size, generator=g).float()
    c.places = torch.randint(0, 140000, size, generator=g).int()
    want = cut(c, keep, 0, recent, 131073)
    assert want.lens.tolist() == [min(n, keep) for n in lens]


def test_evictions_beyond_32_bits():
    """More rows of a layer than 32-bit offsets of their weights reach: a sequence in the last pages, in the second layer."""
    from paper_2502_09922_amd import paged_evict

    hkv, page, n, keep = 8, 1024, 3000, 1000
    pages = (1 << 29) // (hkv * page) + 3
    c = plain.Pages((8, hkv, 2), torch.bfloat16, [1], page, seed=62, weighed=True)
    own, g = 3, torch.Generator().manual_seed(62)
    c.k, c.v = (torch.randn(1, own, hkv, page, 2, generator=g).bfloat16() for _ in range(2))
    c.weights, c.places = torch.rand(1, own, hkv, page, generator=g), torch.randint(0, n, (1, own, hkv, page), generator=g).int()
    c.table, c.lens, c.positions = torch.tensor([[2, 0, 1]], dtype=torch.int32), torch.tensor([n], dtype=torch.int32), torch.tensor([n], dtype=torch.int32)
    big = [torch.zeros((2, pages) + t.shape[2:], dtype=t.dtype, device="cuda") for t in (c.k, c.v, c.weights, c.places)]
    for t, x in zip((c.k, c.v, c.weights, c.places), big):
        x[1, -own:] = t[0].cuda()
        x[0, -own:] = t[0].cuda()
    from paper_2502_09922_amd import PagedCache

    table = (c.table + (pages - own)).int().cuda()
    cache = PagedCache(big[0], big[1], table, c.lens.cuda(), c.positions.cuda(), big[2], big[3])
    paged_evict(cache, keep=keep, recent=10, max_len=n)
    plain.evict(c, keep, 0, 10, n)
    for t, x in zip((c.k, c.v, c.weights, c.places), big):
        for layer in (0, 1):
            assert plain.same(x[layer, -own:].cpu(), t[0])
    assert cache.lens.tolist() == [keep]


@TYPES
@pytest.mark.parametrize("heads,slots", [((1, 1, 128), 3311), ((1, 1, 128), 3313), ((8, 1, 128), 411), ((8, 1, 128), 413), ((16, 1, 64), 190), ((2, 2, 64), 500)],
                         ids=lambda x: str(x).replace(" ", ""))
@pytest.mark.parametrize("batch", [1, 270])
def test_scores_around_what_stays_on_the_chip(heads, slots, dtype, batch):
    """Weights of sequences whose scores just fit beside the tiles, and of ones whose scores do not; few workgroups and many."""
    lens = [2] * batch
    lens[0], lens[-1] = slots // 2, slots
    c = plain.Pages(heads, dtype, lens, 16, seed=71, weighed=True, room=2)
    check(c, None, max_ctx=slots)
    check(c, None, max_ctx=slots + 1)
