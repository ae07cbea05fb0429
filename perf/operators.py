"""The operators of several continuations of a sequence over one cache, as data: attention of a
tree of drafted tokens over a cache, what is kept of such a tree, beam search's selection and the
reordering of its caches; each in its plain form (`own` false) and by this package's calls.

Keys of a case
  kind    "tree" (attention of drafted tokens, with rotation and cache append), "keep" (acceptance
          of the drafts against what the model says, and the cache's compaction), "select" (the k best
          of beams x vocabulary), "reorder" (sequences' caches from their beams' parents)
  heads   a key of HEADS;  dtype: type of queries and caches;  layers of the caches ("keep", "reorder")
  batch   sequences;  lo, hi: cached positions are spread over [lo, hi], the first sequence has hi
  few, many: drafted tokens of a sequence, spread over [few, many], the first sequence has `many`
  groups, beams, vocab, k, done: requests, their beams, tokens of the vocabulary, chosen ones of a
          request, whether some beams have ended ("select")
  group   beams of a request, neighbours in the batch;  shared: positions that all of them share ("reorder")
"""
import math
import random

import numpy as np
import torch

own = False

# heads of queries, heads of keys and values, head size: this package's configurations (synth.CONFIGS)
HEADS = {"tiny": (4, 4, 64), "7b": (32, 32, 128), "13b": (40, 40, 128), "70b": (64, 8, 128)}
ROPE_BASE = 10000.0
MOST_NODES = 64


def listed():
    return [
        # the smallest call: one sequence of the tiny fp32 model checks a root and four drafts; latency alone
        dict(name="tree_tiny_f32", kind="tree", heads="tiny", dtype="f32", batch=1, lo=40, hi=40, few=5, many=5),
        # one interactive sequence with a long context and a draft tree of a usual size
        dict(name="tree_7b_1x26", kind="tree", heads="7b", dtype="bf16", batch=1, lo=3000, hi=3000, few=26, many=26),
        # a batch of requests that each check sixteen tokens, contexts of the 13B-shaped benchmark
        dict(name="tree_13b_32x16", kind="tree", heads="13b", dtype="bf16", batch=32, lo=1024, hi=1087, few=16, many=16),
        # the largest: grouped queries, contexts of the 70B-shaped benchmark, trees of different sizes
        dict(name="tree_70b_64_ragged", kind="tree", heads="70b", dtype="bf16", batch=64, lo=128, hi=2287, few=4, many=16),
        # fp32 caches at real head sizes, as one checks a bf16 deployment against them
        dict(name="tree_7b_f32_4x12", kind="tree", heads="7b", dtype="f32", batch=4, lo=131, hi=700, few=7, many=12),
        # the end of an interactive sequence's step: a quarter of the 7B model's layers
        dict(name="keep_7b_1x26", kind="keep", heads="7b", dtype="bf16", layers=8, batch=1, lo=3000, hi=3000, few=26, many=26),
        # the same for a batch, a tenth of the 13B model's layers
        dict(name="keep_13b_32x16", kind="keep", heads="13b", dtype="bf16", layers=4, batch=32, lo=1024, hi=1087, few=16, many=16),
        # beam search of one request
        dict(name="select_1x4", kind="select", groups=1, beams=4, vocab=32000, k=4, done=False),
        # sixteen requests of eight beams, some of them ended; twice as many candidates as beams
        dict(name="select_16x8_done", kind="select", groups=16, beams=8, vocab=32000, k=16, done=True),
        # many requests over a vocabulary of odd size: rows that start anywhere
        dict(name="select_64x5_odd", kind="select", groups=64, beams=5, vocab=50257, k=10, done=False),
        # beams of one request behind a shared prompt: a quarter of the 7B model's layers
        dict(name="reorder_7b_1x4", kind="reorder", heads="7b", dtype="bf16", layers=8, batch=4, lo=600, hi=600, group=4, shared=512),
        # beams without a shared prefix, a tenth of the 13B model's layers
        dict(name="reorder_13b_8x4", kind="reorder", heads="13b", dtype="bf16", layers=4, batch=32, lo=700, hi=1087, group=4, shared=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tree"] * 4 + ["keep", "select", "select", "reorder"])
    if kind == "select":
        groups, beams = _log_int(rng, 1, 64), rng.randint(1, 16)
        vocab = _log_int(rng, 500, max(501, min(130000, 16_000_000 // (groups * beams))))
        return dict(kind=kind, groups=groups, beams=beams, vocab=vocab, k=rng.randint(1, 2 * beams), done=rng.random() < 0.3)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    heads = rng.choice(["tiny", "7b", "13b", "70b"])
    if kind == "tree":
        hi = _log_int(rng, 16, 4096)
        # caches of 34k positions of 40 heads at most, and products as in the largest listed case at most
        hq, hkv, hd = HEADS[heads]
        wide = 2 if dtype == "f32" else 1
        batch = _log_int(rng, 1, max(1, min(64, 34000 * 40 // (hkv * wide) // (hi + MOST_NODES))))
        many = _log_int(rng, 1, max(1, min(MOST_NODES, int(2.7e10 / wide / (4.0 * hq * hd * batch * hi)))))
        return dict(kind=kind, heads=heads, dtype=dtype, batch=batch, lo=max(1, int(hi * rng.choice([1.0, rng.uniform(0.1, 1.0)]))),
                    hi=hi, few=max(1, int(many * rng.choice([1.0, rng.uniform(0.2, 1.0)]))), many=many)
    layers, hi = rng.randint(1, 8), _log_int(rng, 32, 2048)
    room = 4 * 36000 * 40 // (HEADS[heads][1] * (2 if dtype == "f32" else 1))
    batch = _log_int(rng, 1, max(1, min(64, room // (layers * (hi + MOST_NODES)))))
    if kind == "keep":
        many = _log_int(rng, 2, MOST_NODES)
        return dict(kind=kind, heads=heads, dtype=dtype, layers=layers, batch=batch, lo=max(1, hi // rng.randint(1, 4)), hi=hi,
                    few=max(1, many // rng.randint(1, 3)), many=many)
    group = rng.randint(2, 8)
    return dict(kind=kind, heads=heads, dtype=dtype, layers=layers, batch=group * max(1, batch // group), lo=max(1, hi // rng.randint(1, 2)),
                hi=hi, group=group, shared=int(hi * rng.choice([0.0, rng.uniform(0.2, 0.9)])))


# ---- what a case is made of: lengths, trees and parents go by the case, all values by the seed ----------------------------
def _rng(case, what):
    return random.Random("%s %r" % (what, sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    """Cached positions of the sequences; beams of a request have the same."""
    r, group = _rng(case, "lengths"), case.get("group", 1)
    lens = [case["hi"]] + [r.randint(case["lo"], case["hi"]) for _ in range(case["batch"] // group - 1)]
    return [n for n in lens for _ in range(group)]


def _trees(case):
    """Parents of each sequence's nodes, a parent in front of its children: node i hangs under one of the nodes in front of it,
    mostly under one that is a third of the way, which makes trees of a few levels as drafting programs make them."""
    r, out = _rng(case, "trees"), []
    for b in range(case["batch"]):
        n = case["many"] if b == 0 else r.randint(case["few"], case["many"])
        out.append([-1] + [max(0, min(i - 1, int((i - 1) * r.uniform(0.2, 0.7)))) if r.random() < 0.9 else r.randrange(i) for i in range(1, n)])
    return out


def _path(parents, i):
    """Nodes from the root to node i."""
    return (_path(parents, parents[i]) if i else []) + [i]


def _accepted(case):
    """The node of each tree that the model's own tokens lead to."""
    r = _rng(case, "accepted")
    return [r.randrange(len(p) // 3, len(p)) for p in _trees(case)]


def _sources(case):
    r, g = _rng(case, "sources"), case["group"]
    return [b // g * g + r.randrange(g) for b in range(case["batch"])]


def _ended(case):
    r = _rng(case, "ended")
    return [int(case["done"] and r.random() < 0.25) for _ in range(case["groups"] * case["beams"])]


def _max_seq(case):
    return (case["hi"] + case.get("many", 1) + 31) // 32 * 32


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gen(seed, *key):
    return torch.Generator(device="cuda").manual_seed(random.Random("%d %r" % (seed, key)).randrange(1 << 62))


def _normal(seed, key, size, dtype, std):
    return torch.empty(size, dtype=dtype, device="cuda").normal_(0.0, std, generator=_gen(seed, key))


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


# Queries, keys and values are sums of `hidden` products of a normalised row and N(0, 0.02) weights.
def _inputs(case, seed):
    s = {"case": case}
    if case["kind"] == "select":
        rows = case["groups"] * case["beams"]
        s["logits"] = _normal(seed, "logits", (rows, case["vocab"]), torch.float32, 2.5)
        s["scores"] = -_normal(seed, "scores", (rows,), torch.float32, 3.0).abs()
        s["ended"] = _ints(_ended(case)) if case["done"] else None
        return s
    hq, hkv, hd = HEADS[case["heads"]]
    lens = _lengths(case)
    std = 0.02 * math.sqrt(hq * hd)
    size = (case["batch"], hkv, _max_seq(case), hd)
    if case["kind"] != "tree":
        size = (case["layers"],) + size
    s["k"], s["v"] = _normal(seed, "k", size, _dtype(case), std), _normal(seed, "v", size, _dtype(case), std)
    s["lens"], s["seq_lens"] = _ints(lens), _ints(lens)
    if case["kind"] == "reorder":
        s["src"] = _ints(_sources(case))
        s["first"] = _ints([min(case["shared"], n) for n in lens])
        return s
    trees = _trees(case)
    s["cu_host"] = np.cumsum([0] + [len(p) for p in trees]).astype(np.int32)
    s["cu"], s["parents"] = _ints(s["cu_host"].tolist()), _ints([p for t in trees for p in t])
    rows = int(s["cu_host"][-1])
    if case["kind"] == "tree":
        s["qkv"] = _normal(seed, "qkv", (rows, (hq + 2 * hkv) * hd), _dtype(case), std)
        at = torch.arange(size[-2], dtype=torch.float64, device="cuda")[:, None] * ROPE_BASE ** (
            -2.0 * torch.arange(hd // 2, dtype=torch.float64, device="cuda") / hd)
        s["rope"] = torch.stack([at.cos(), at.sin()], -1).float()
        return s
    # what the model says at every node, and drafts that agree with it along one path
    said = torch.randint(0, 32000, (rows,), dtype=torch.int32, device="cuda", generator=_gen(seed, "said"))
    agree = torch.tensor([i in set(_path(t, a)) for t, a in zip(trees, _accepted(case)) for i in range(len(t))], device="cuda")
    under = _ints([int(s["cu_host"][b]) + max(p, 0) for b, t in enumerate(trees) for p in t], torch.int64)
    s["said"], s["tokens"] = said, torch.where(agree, said[under], (said[under] + 1) % 32000)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    torch.cuda.synchronize()
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if kind == "tree":
        return _tree(s)
    if kind == "keep":
        s["seq_lens"].copy_(s["lens"])  # the scheduler names the cached length of every slot
        return _keep(s)
    return _select(s) if kind == "select" else _reorder(s)


def _tree(s):
    hi = s["case"]["hi"]
    if own:
        from paper_2502_09922_amd import tree_attention

        out = tree_attention(s["qkv"], s["parents"], s["cu"], s["cu_host"], s["rope"], s["k"], s["v"], s["seq_lens"], max_ctx=hi)
        return {"out": out, "k": s["k"], "v": s["v"]}
    (B, hkv, _, hd), rows = s["k"].shape, s["qkv"].shape[0]
    hq = s["qkv"].shape[1] // hd - 2 * hkv
    seq, node, sees, lens = _nodes(s)
    N = sees.shape[1]
    at = lens[seq] + sees.sum(-1)[seq, node] - 1
    turn = s["rope"][at][:, None]
    heads = s["qkv"].float().view(rows, hq + 2 * hkv, hd)
    u, w = heads[:, : hq + hkv, 0::2], heads[:, : hq + hkv, 1::2]
    qk = torch.stack([u * turn[..., 0] - w * turn[..., 1], u * turn[..., 1] + w * turn[..., 0]], -1).view(rows, hq + hkv, hd)
    s["k"][seq, :, lens[seq] + node] = qk[:, hq:].to(s["k"].dtype)
    s["v"][seq, :, lens[seq] + node] = heads[:, hq + hkv :].to(s["v"].dtype)
    S = hi + N
    q = torch.zeros(B, N, hq, hd, device="cuda")
    q[seq, node] = qk[:, :hq]
    q = q.view(B, N, hkv, hq // hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, hkv, N * (hq // hkv), hd)
    score = q @ s["k"][:, :, :S].float().transpose(2, 3) / math.sqrt(hd)
    behind = torch.arange(S, device="cuda")[None] - lens[:, None]  # of the context: the tree's slots
    seen = sees.gather(2, behind.clamp(0, N - 1)[:, None].expand(B, N, S)) & (behind < N)[:, None] | (behind < 0)[:, None]
    score = score.view(B, hkv, N, -1, S).masked_fill(~seen[:, None, :, None], -math.inf).view(B, hkv, -1, S)
    p = (score - score.amax(-1, keepdim=True)).exp()
    o = (p @ s["v"][:, :, :S].float()) / p.sum(-1, keepdim=True)
    o = o.view(B, hkv, N, hq // hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, N, hq * hd)[seq, node]
    return {"out": o.to(s["qkv"].dtype), "k": s["k"], "v": s["v"]}


def _nodes(s):
    """Sequence and node of each row, [sequence][node][node] which nodes a node sees (its path from the root), cached lengths."""
    cu = s["cu"].long()
    rows, B, N = int(s["cu_host"][-1]), len(s["cu_host"]) - 1, int(np.diff(s["cu_host"]).max())
    seq = torch.searchsorted(cu[1:], torch.arange(rows, device="cuda"), right=True)
    node = torch.arange(rows, device="cuda") - cu[seq]
    step = torch.eye(N, dtype=torch.float64, device="cuda").repeat(B, 1, 1)
    step[seq, node, s["parents"].clamp(min=0).long()] = 1.0
    return seq, node, torch.linalg.matrix_power(step, MOST_NODES) > 0, s["seq_lens"].long()


def _keep(s):
    if own:
        from paper_2502_09922_amd import tree_accept, tree_keep

        kept, count, emitted, following = tree_accept(s["tokens"], s["said"], s["parents"], s["cu"], s["cu_host"])
        tree_keep(kept, s["cu"], s["cu_host"], s["k"], s["v"], s["seq_lens"])
        return {"kept": kept, "count": count, "emitted": emitted, "next": following, "k": s["k"], "v": s["v"], "seq_lens": s["seq_lens"]}
    seq, node, sees, lens = _nodes(s)
    B, N = sees.shape[:2]
    agrees = torch.zeros(B, N, dtype=torch.bool, device="cuda")
    said = torch.zeros(B, N, dtype=torch.int64, device="cuda")
    agrees[seq, node] = (s["tokens"] == s["said"][(s["cu"].long()[seq] + s["parents"].clamp(min=0))]) | (node == 0)
    said[seq, node] = s["said"].long()
    on = (~sees | agrees[:, None]).all(-1)
    order = torch.arange(N, device="cuda")
    best = torch.where(on & agrees, sees.sum(-1) * MOST_NODES - order, -1).argmax(-1)
    path = sees[torch.arange(B, device="cuda"), best]
    count = path.sum(-1)
    kept = (path.long() << order).sum(-1)
    nodes = torch.where(path, order, N).sort(-1).values
    there = order < count[:, None]
    emitted = torch.full((B, MOST_NODES), -1, dtype=torch.int32, device="cuda")
    emitted[:, :N] = torch.where(there, said.gather(1, nodes.clamp(max=N - 1)), -1).int()
    following = said.gather(1, best[:, None])[:, 0].int()
    # all rows are fetched before any is written; slots behind the kept ones get what they hold
    b, to = torch.arange(B, device="cuda")[:, None], lens[:, None] + order
    fetch = torch.where(there, lens[:, None] + nodes, to)
    s["k"][:, b, :, to] = s["k"][:, b, :, fetch]
    s["v"][:, b, :, to] = s["v"][:, b, :, fetch]
    s["seq_lens"].add_(count)
    return {"kept": kept, "count": count.int(), "emitted": emitted, "next": following, "k": s["k"], "v": s["v"], "seq_lens": s["seq_lens"]}


def _select(s):
    case = s["case"]
    G, W, V, K = case["groups"], case["beams"], case["vocab"], case["k"]
    if own:
        from paper_2502_09922_amd import beam_select

        rows, tokens, scores = beam_select(s["logits"], s["scores"], beams=W, k=K, ended=s["ended"], eos=2)
        return {"rows": rows, "tokens": tokens, "scores": scores}
    # in 64 bits: two candidates of different beams may lie next to each other
    x = s["logits"].double()
    top = x.amax(-1, keepdim=True)
    score = x - (top + (x - top).exp().sum(-1, keepdim=True).log()) + s["scores"].double()[:, None]
    if s["ended"] is not None:
        stays = torch.full_like(score, -math.inf)
        stays[:, 2] = s["scores"].double()
        score = torch.where(s["ended"][:, None] != 0, stays, score)
    score = score.masked_fill(score.isnan(), -math.inf).view(G, W * V)
    score, at = score.sort(dim=-1, descending=True, stable=True)
    at = at[:, :K]
    return {"rows": (at // V + torch.arange(G, device="cuda")[:, None] * W).int(), "tokens": (at % V).int(), "scores": score[:, :K].float()}


def _reorder(s):
    case = s["case"]
    if own:
        from paper_2502_09922_amd import kv_reorder

        kv_reorder(s["src"], case["group"], s["k"], s["v"], s["seq_lens"], max_ctx=case["hi"], first=s["first"])
        return {"k": s["k"], "v": s["v"], "seq_lens": s["seq_lens"]}
    src, at = s["src"].long(), torch.arange(s["k"].shape[3], device="cuda")
    moved = (at >= s["first"][:, None]) & (at < s["seq_lens"][src][:, None])
    s["k"].copy_(torch.where(moved[None, :, None, :, None], s["k"][:, src], s["k"]))
    s["v"].copy_(torch.where(moved[None, :, None, :, None], s["v"][:, src], s["v"]))
    s["seq_lens"].copy_(s["seq_lens"][src])
    return {"k": s["k"], "v": s["v"], "seq_lens": s["seq_lens"]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "select":
        live = sum(1 - e for e in _ended(case))
        return {"bytes": 4.0 * live * case["vocab"] + 4.0 * case["groups"] * (case["beams"] + 3 * case["k"]), "flops": 4.0 * live * case["vocab"]}
    hq, hkv, hd = HEADS[case["heads"]]
    e, lens = _dtype(case).itemsize, _lengths(case)
    row = 2.0 * hkv * hd * e  # key and value of one position of one layer
    if case["kind"] == "reorder":
        moved = [n - min(case["shared"], n) for b, (n, src) in enumerate(zip(lens, _sources(case))) if src != b]
        return {"bytes": 2.0 * case["layers"] * row * sum(moved) + 12.0 * len(lens), "flops": 0.0}
    trees = _trees(case)
    rows = sum(len(t) for t in trees)
    if case["kind"] == "keep":
        moved = sum(1 for t, a in zip(trees, _accepted(case)) for j, i in enumerate(_path(t, a)) if i != j)
        return {"bytes": 2.0 * case["layers"] * row * moved + 12.0 * rows + 4.0 * len(trees) * (MOST_NODES + 5), "flops": 0.0}
    pairs = sum(len(t) * n + sum(len(_path(t, i)) for i in range(len(t))) for t, n in zip(trees, lens))
    return {"bytes": row * (sum(lens) + 2 * rows) + 2.0 * rows * hq * hd * e + 4.0 * rows, "flops": 4.0 * hq * hd * pairs}


# ---- the same in 64 bits, sequence by sequence ------------------------------------------------------------------------------
def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "select":
        rows, tokens, scores = [], [], []
        for g in range(case["groups"]):
            rs = range(g * case["beams"], (g + 1) * case["beams"])
            each = [torch.log_softmax(s["logits"][r].double(), -1) + s["scores"][r].double() for r in rs]
            for i, r in enumerate(rs):
                if s["ended"] is not None and int(s["ended"][r]):
                    each[i] = torch.full_like(each[i], -math.inf)
                    each[i][2] = s["scores"][r].double()
            val, at = torch.cat(each).topk(case["k"])
            rows.append(g * case["beams"] + at // case["vocab"])
            tokens.append(at % case["vocab"])
            scores.append(val)
        return {"rows": torch.stack(rows).int(), "tokens": torch.stack(tokens).int(), "scores": torch.stack(scores)}
    lens, k, v = _lengths(case), s["k"], s["v"]
    if case["kind"] == "reorder":
        k2, v2 = k.clone(), v.clone()
        for b, src in enumerate(_sources(case)):
            at = slice(min(case["shared"], lens[b]), lens[src])
            k2[:, b, :, at], v2[:, b, :, at] = k[:, src, :, at], v[:, src, :, at]
        return {"k": k2, "v": v2, "seq_lens": _ints([lens[i] for i in _sources(case)])}
    trees = _trees(case)
    if case["kind"] == "keep":
        said, kept, count, emitted, following = s["said"].tolist(), [], [], [], []
        k2, v2 = k.clone(), v.clone()
        for b, (t, a) in enumerate(zip(trees, _accepted(case))):
            path, r = _path(t, a), int(s["cu_host"][b])
            bits = sum(1 << i for i in path)
            kept.append(bits - (1 << 64) if bits >> 63 else bits)
            count.append(len(path))
            emitted.append([said[r + i] for i in path] + [-1] * (MOST_NODES - len(path)))
            following.append(said[r + a])
            for j, i in enumerate(path):
                k2[:, b, :, lens[b] + j], v2[:, b, :, lens[b] + j] = k[:, b, :, lens[b] + i], v[:, b, :, lens[b] + i]
        return {"kept": _ints(kept, torch.int64), "count": _ints(count), "emitted": _ints(emitted), "next": _ints(following), "k": k2, "v": v2,
                "seq_lens": _ints([n + c for n, c in zip(lens, count)])}
    hq, hkv, hd = HEADS[case["heads"]]
    k2, v2, out = k.double(), v.double(), []
    for b, t in enumerate(trees):
        r, n, c = int(s["cu_host"][b]), len(t), lens[b]
        rows = s["qkv"][r : r + n].double().view(n, hq + 2 * hkv, hd)
        paths = [_path(t, i) for i in range(n)]
        turn = s["rope"].double()[torch.tensor([c + len(p) - 1 for p in paths], device="cuda")]
        z = torch.view_as_complex(rows[:, : hq + hkv].contiguous().view(n, hq + hkv, hd // 2, 2)) * torch.view_as_complex(turn)[:, None]
        qk = torch.view_as_real(z).reshape(n, hq + hkv, hd)
        k2[b, :, c : c + n], v2[b, :, c : c + n] = qk[:, hq:].transpose(0, 1), rows[:, hq + hkv :].transpose(0, 1)
        # attention is over the rows that the cache holds, in its type
        keys = torch.cat([k[b, :, :c].double(), qk[:, hq:].transpose(0, 1).to(k.dtype).double()], 1)
        vals = v2[b, :, : c + n]
        seen = torch.ones(n, c + n, dtype=torch.bool, device="cuda")
        seen[:, c:] = torch.tensor([[i in p for i in range(n)] for p in paths], device="cuda")
        q = qk[:, :hq].view(n, hkv, hq // hkv, hd).permute(1, 2, 0, 3)
        sc = torch.matmul(q, keys[:, None].transpose(2, 3)) / math.sqrt(hd)
        p = torch.softmax(sc.masked_fill(~seen, -math.inf), -1)
        out.append(torch.matmul(p, vals[:, None]).permute(2, 0, 1, 3).reshape(n, hq * hd))
    return {"out": torch.cat(out), "k": k2, "v": v2}
