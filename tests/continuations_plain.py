"""Draft trees, beams and their caches in plain 64-bit arithmetic on the CPU, node by node: what the kernels are compared with."""
import math

import torch


def path(parents, i):
    """Nodes from the root to node i."""
    out = [i]
    while out[0] > 0 and 0 <= parents[out[0]] < out[0]:
        out.insert(0, parents[out[0]])
    return out


def random_tree(rng, n):
    return [-1] + [rng.randrange(max(0, i - 6), i) for i in range(1, n)]


def turned(rows, rope, positions):
    """rows [n, heads, hd] with pairs (2i, 2i + 1) turned by rope [max_seq, hd/2, 2] at their positions."""
    if rope is None:
        return rows.clone()
    c, s = rope[positions][:, None, :, 0], rope[positions][:, None, :, 1]
    u, w = rows[..., 0::2], rows[..., 1::2]
    return torch.stack([u * c - w * s, u * s + w * c], -1).reshape(rows.shape)


def attend(q, keys, vals, ctx, parents):
    """q [n, hq, hd], keys and vals [hkv, ctx + n, hd], float64.  Returns out [n, hq, hd], the sums of weighted |v| and the largest
    sum of |q k| / sqrt(hd) that a row has among its keys, from which rounding errors are bounded."""
    n, hq, hd = q.shape
    hkv = keys.shape[0]
    out, weighted, size = torch.empty_like(q), torch.empty_like(q), torch.empty(n, hq, 1, dtype=q.dtype)
    for i in range(n):
        seen = list(range(ctx)) + [ctx + j for j in path(parents, i)]
        for h in range(hq):
            k, v = keys[h // (hq // hkv)][seen], vals[h // (hq // hkv)][seen]
            p = torch.softmax(k @ q[i, h] / math.sqrt(hd), 0)
            out[i, h], weighted[i, h] = p @ v, p @ v.abs()
            size[i, h] = (k.abs() @ q[i, h].abs()).max() / math.sqrt(hd)
    return out, weighted, size


def accepted(parents, tokens, said):
    """Path that is kept: the deepest accepted node's, of equals that of the lowest index."""
    on = [True] + [False] * (len(parents) - 1)
    for i in range(1, len(parents)):
        p = parents[i]
        on[i] = 0 <= p < i and on[p] and tokens[i] == said[p]
    paths = [path(parents, i) for i in range(len(parents)) if on[i]]
    return max(paths, key=len)  # the first of the longest


def select(logits, scores, ended, beams, k, eos):
    """(rows, tokens, scores) of the k best candidates of every request, best first, equal ones by index."""
    x = logits.double()
    x = x - x.amax(1, keepdim=True)  # apart: next to a logit of the type's lowest value the rest would be lost in 64 bits too
    s = x - x.exp().sum(1, keepdim=True).log() + scores.double()[:, None]
    for r in range(x.shape[0]):
        if ended is not None and ended[r]:
            s[r] = -math.inf
            s[r, eos] = scores[r]
    s = torch.where(s.isnan(), -math.inf, s).view(-1, beams * x.shape[1])
    s, at = s.sort(dim=1, descending=True, stable=True)
    at = at[:, :k]
    return at // x.shape[1] + torch.arange(s.shape[0])[:, None] * beams, at % x.shape[1], s[:, :k]
