"""Plain 64-bit forms of the operators of a step of several new tokens per sequence, on the CPU, one sequence, head and
node at a time, and the inputs that the tests share."""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts(v):
    return [0] + [int(x) for x in np.cumsum(v)]


def random_parents(rng, n, spread=5, forest=False):
    """Parents of a tree whose nodes follow one of the `spread` before them; with `forest` some follow the cache."""
    up = [-1] + [max(0, j - 1 - int(rng.integers(0, spread))) for j in range(1, n)]
    if forest:
        up = [-1 if j > 0 and rng.random() < 0.15 else p for j, p in enumerate(up)]
    return up[:n]


def ancestors(parent):
    """(bool [n, n]: row i has node i and its ancestors, depth of every node)."""
    n = len(parent)
    seen, depth = np.zeros((n, n), dtype=bool), []
    for i in range(n):
        a, d = i, -1
        while a >= 0:
            seen[i, a] = True
            a, d = parent[a], d + 1
        depth.append(d)
    return seen, depth


def pack_mask(seen_per_seq, words):
    """Mask rows of all sequences, int32 bit patterns [tokens, words]."""
    rows = []
    for seen in seen_per_seq:
        for r in seen:
            w = [0] * words
            for j in np.flatnonzero(r):
                w[j // 32] |= 1 << (j % 32)
            rows.append([x - (1 << 32) if x >= 1 << 31 else x for x in w])
    return torch.tensor(rows, dtype=torch.int32).view(-1, words)


def rope_reference(x, weight, eps, pos, inv_freq, interleaved):
    """(value, how large the terms of each rotated sum are) of rows x [tokens, heads, D], 64 bits."""
    x = x.double().cpu()
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + float(np.float32(eps))) * weight.double().cpu()
    y, size = x.clone(), x.abs()
    if inv_freq is not None:
        f = inv_freq.double().cpu()
        half = f.numel()
        a = pos.double().cpu()[:, None] * f[None]
        cos, sin = torch.cos(a)[:, None], torch.sin(a)[:, None]
        lo, hi = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        p, q = x[..., lo], x[..., hi]
        y[..., lo], y[..., hi] = p * cos - q * sin, p * sin + q * cos
        size[..., lo] = size[..., hi] = p.abs() + q.abs()
    return y, size


def tree_reference(q, Kp, Vp, Kn, Vn, seen, scale):
    """One sequence and KV head: q [n, G, D], prefix [L, D], nodes [n, D], seen bool [n, n].  64 bits; returns out
    [n, G, D], the same of |V| (how large the weighted sums are), lse [n, G]."""
    n, G, _ = q.shape
    q, Kp, Vp, Kn, Vn = (x.double() for x in (q.reshape(n * G, D), Kp, Vp, Kn, Vn))
    hidden = torch.from_numpy(~seen).to(q.device).repeat_interleave(G, 0)
    z = torch.cat([q @ Kp.t().contiguous(), (q @ Kn.t().contiguous()).masked_fill(hidden, -math.inf)], 1) * scale
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse.masked_fill(lse == -math.inf, 0.0)[:, None])     # rows that see nothing: 0
    V = torch.cat([Vp, Vn])
    return (p @ V).view(n, G, D), (p @ V.abs()).view(n, G, D), lse.view(n, G)


def accept_reference(parent, draft, target, most):
    """(path, next id) of one sequence."""
    n, path, cur, nxt = len(parent), [], 0, -1
    while n and cur is not None and len(path) < most:
        path.append(cur)
        nxt = target[cur]
        cur = next((j for j in range(cur + 1, n) if parent[j] == cur and draft[j] == target[cur]), None)
    return path, nxt
