"""A cache in pages in plain 64-bit arithmetic, sequence by sequence, for the tests of its calls."""
import math
import random

import torch

from continuations_plain import turned

U = {torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}  # half a step of a stored value, relative


def bits(t):
    return t.view({8: torch.int64, 4: torch.int32, 2: torch.int16}[t.element_size()])


def same(a, b):
    return torch.equal(bits(a), bits(b))


class Pages:
    """Pools and tables on the host: sequences of `lens` slots in pages anywhere in the pool, everything else NaN."""

    def __init__(self, heads, dtype, lens, page, layers=1, seed=0, weighed=False, room=1, spare=3):
        hq, hkv, hd = heads
        r, g = random.Random(seed), torch.Generator().manual_seed(seed)
        need = [(max(n, 0) + room + page - 1) // page for n in lens]
        pages = sum(need) + spare
        order = list(range(pages))
        r.shuffle(order)
        columns = max(need) + 1
        self.table = torch.full((len(lens), columns), -1, dtype=torch.int32)
        for b, n in enumerate(need):
            for i in range(n):
                self.table[b, i] = order.pop()
        size = (layers, pages, hkv, page, hd)
        self.k, self.v = (torch.full(size, math.nan, dtype=dtype) for _ in range(2))
        self.weights = torch.full(size[:-1], math.nan) if weighed else None
        self.places = torch.full(size[:-1], -7, dtype=torch.int32) if weighed else None
        self.heads, self.page, self.layers = heads, page, layers
        self.lens = torch.tensor(lens, dtype=torch.int32)
        self.positions = self.lens.clone()
        for b, n in enumerate(lens):
            for layer in range(layers):
                for i in range(max(n, 0)):
                    at = self.at(layer, b, i)
                    self.k[at], self.v[at] = (torch.randn(hkv, hd, generator=g).to(dtype) for _ in range(2))
                    if weighed:
                        self.weights[at], self.places[at] = torch.rand(hkv, generator=g), i
        self.qkv = torch.randn(layers, len(lens), (hq + 2 * hkv) * hd, generator=g).to(dtype)

    def at(self, layer, b, i):
        """Index of slot i of a sequence in the pools, all kv heads."""
        return layer, int(self.table[b, i // self.page]), slice(None), i % self.page

    def named(self, b, i):
        return 0 <= i // self.page < self.table.shape[1] and 0 <= int(self.table[b, i // self.page]) < self.k.shape[1]

    def room(self, b, positions):
        n, pos = int(self.lens[b]), int(self.positions[b])
        return n >= 0 and self.named(b, n) and 0 <= pos < positions

    def tensors(self):
        return dict(k=self.k, v=self.v, table=self.table, lens=self.lens, positions=self.positions, weights=self.weights, places=self.places)

    def on_gpu(self):
        """A PagedCache of copies of the tensors."""
        from paper_2502_09922_amd import PagedCache

        return PagedCache(**{n: None if t is None else t.cuda() for n, t in self.tensors().items()})

    def take(self, cache):
        """The tensors as they are on the GPU now."""
        for n, t in self.tensors().items():
            if t is not None:
                setattr(self, n, getattr(cache, n).cpu())


def rope_table(positions, hd):
    at = torch.arange(positions, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)
    return torch.stack([at.cos(), at.sin()], -1).float()


def check_attention(c, layer, rope, got, out):
    """A call's pools `got` (Pages) and output rows against those before it (`c`).  The new key: turned in 32 bits (two products and a sum
    of values of at most the pair's size: 3 2^-24 of it, twice that for a rounding border crossed) and rounded once.  Attention over
    the rows that the cache then holds: queries turned in 32 bits and, for matrix products, split into two bf16 parts (2^-15 left
    out), hd products summed in 32 bits: a score is off by its ds, and its weight by that and the mean of all ds; exponents are of products
    with the maximum (rounded, a few times 2^-24 of it); weights of bf16 products have two parts (2^-15); sums of m terms in 32 bits
    are off by m 2^-24 of their sizes."""
    hq, hkv, hd = c.heads
    dtype, u = c.k.dtype, U[c.k.dtype]
    left = {n: getattr(got, n).clone() for n in ("k", "v", "weights", "places") if getattr(got, n) is not None}
    for b in range(len(c.lens)):
        row = out[b].double().view(hq, hd)
        if not c.room(b, 1 << 31 if rope is None else rope.shape[0]):
            assert (out[b] == 0).all(), b
            continue
        n, at = int(c.lens[b]), c.at(layer, b, int(c.lens[b]))
        raw = c.qkv[layer, b].double().view(1, hq + 2 * hkv, hd)
        qk = turned(raw[:, : hq + hkv], None if rope is None else rope.double(), [int(c.positions[b])])[0]
        assert same(got.v[at], c.qkv[layer, b].view(hq + 2 * hkv, hd)[hq + hkv :].contiguous()), b
        want = qk[hq:]
        pair = raw[0, hq : hq + hkv].abs().view(hkv, -1, 2).sum(-1).repeat_interleave(2, -1)
        finite = want.isfinite()
        assert ((got.k[at].double() - want).abs() <= u * want.abs() + 2 * 3 * 2.0**-24 * pair)[finite].all(), b
        for name, before in (("k", c.k), ("v", c.v)):
            left[name][at] = before[at]
        slots = [i for i in range(n + 1) if c.named(b, i)]
        keys, vals = (torch.stack([pool[c.at(layer, b, i)].double() for i in slots], 1) for pool in (got.k, got.v))  # [hkv][slots][hd]
        q = qk[:hq].view(hkv, hq // hkv, hd)
        score = q @ keys.transpose(1, 2) / math.sqrt(hd)
        p = torch.softmax(score, -1)
        exact = (p @ vals).reshape(hq, hd)
        size = (q.abs() @ keys.abs().transpose(1, 2) / math.sqrt(hd)).masked_fill(score == -math.inf, 0.0)  # of scores that count
        ds = (hd + 8) * 2.0**-24 * size + (2.0**-15 * size if dtype == torch.bfloat16 else 0.0)
        top = score.masked_fill(p < 1e-30, 0.0).abs().amax(-1, keepdim=True)
        factor = ds + (p * ds).sum(-1, keepdim=True) + 8 * 2.0**-24 * top + 2.0**-21 + (n + 17) * 2.0**-24
        bound = u * exact.abs() + ((p * (factor + (2.0**-15 if dtype == torch.bfloat16 else 0.0))) @ vals.abs()).reshape(hq, hd) * 1.01 + 1e-30
        finite = exact.isfinite()
        assert torch.equal(finite, row.isfinite()) and torch.equal(exact.isnan(), row.isnan()), b
        err = (row - exact).abs()
        assert (err <= bound)[finite].all(), (b, n, float((err / bound)[finite].max()))
        if c.weights is None:
            continue
        gain, off = p.sum(1), (p * factor).sum(1) * 1.01  # [hkv][slots]
        for j, i in enumerate(slots):
            to = c.at(layer, b, i)
            had = c.weights[to].double() if i < n else torch.zeros(hkv)
            w, g = had + gain[:, j], got.weights[to].double()
            assert ((g - w).abs() <= off[:, j] + (2 * u_sum(hq // hkv)) * w.abs() + 1e-30).logical_or(w.isnan() & g.isnan()).all(), (b, i, g, w)
            left["weights"][to] = c.weights[to]
        assert (got.places[at] == c.positions[b]).all()
        left["places"][at] = c.places[at]
    for name, t in left.items():  # nothing else was written
        assert same(t, getattr(c, name)), name
    assert torch.equal(got.lens, c.lens) and torch.equal(got.positions, c.positions)


def u_sum(terms):
    """Rounding of a 32-bit sum of so many terms and one more, relative to a sum of positive ones."""
    return (terms + 1) * 2.0**-24


def fill(c, from_k, from_v, from_lens, src, weights):
    """What ls_paged_fill makes of the pools, in place."""
    for b, s in enumerate(src):
        if not 0 <= s < from_k.shape[1]:
            continue
        n = int(from_lens[s])
        if not 0 <= n <= min(from_k.shape[3], c.table.shape[1] * c.page):
            continue
        for i in range(n):
            if not c.named(b, i):
                continue
            for layer in range(c.layers):
                at = c.at(layer, b, i)
                c.k[at], c.v[at] = from_k[layer, s, :, i], from_v[layer, s, :, i]
                if c.weights is not None:
                    c.weights[at], c.places[at] = 0.0 if weights is None else weights[layer, s, :, i], i
        c.lens[b] = c.positions[b] = n


def evict(c, keep, first, recent, max_len):
    """What ls_paged_evict makes of the pools, in place."""
    hkv = c.heads[1]
    for b in range(len(c.lens)):
        n, pos = int(c.lens[b]), int(c.positions[b])
        if n <= keep or n > max_len or n > c.table.shape[1] * c.page or not all(c.named(b, i) for i in range(n)):
            continue
        for layer in range(c.layers):
            for h in range(hkv):
                at = [(layer, int(c.table[b, i // c.page]), h, i % c.page) for i in range(n)]

                def key(i):
                    w, place = float(c.weights[at[i]]), int(c.places[at[i]])
                    if place < first or place >= pos - recent:
                        return (0, 0.0, i)
                    return (2, 0.0, i) if math.isnan(w) else (1, -w, i)

                kept = set(sorted(range(n), key=key)[:keep])
                to = [i for i in range(keep) if i not in kept]
                frm = [i for i in range(keep, n) if i in kept]
                assert len(to) == len(frm)
                for x, y in zip(to, frm):
                    for pool in (c.k, c.v, c.weights, c.places):
                        pool[at[x]] = pool[at[y]]
        c.lens[b] = keep
