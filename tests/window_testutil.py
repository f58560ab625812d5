"""Plain 64-bit forms of the calls on caches in 8 bits and with a sliding window, and the inputs that their tests share."""
from __future__ import annotations

import math

import torch

D = 128
E_MIN, E_MAX = -100, 120


def pow2(e):
    return torch.exp2(e.double())


def e4m3(x):
    """The nearest e4m3 value of |x| <= 448 in 64 bits, ties to the even one."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def half_step(x):
    """Half the distance of the e4m3 values around x."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 4)


def exponent(x):
    """The least e with |x| <= 448 * 2^e for every finite x of a block, within the range of the scales."""
    m = x.abs()
    m = torch.where(torch.isfinite(m), m, 0.0).max().item() if m.numel() else 0.0
    if m == 0.0:
        return E_MIN
    f, e = math.frexp(m)
    return min(max(e - 9 + (f > 0.875), E_MIN), E_MAX)


def quantise(X, block):
    """(codes e4m3, scales e8m0) of X [H, rows, D], blocks from row 0 on."""
    H, n, _ = X.shape
    nb = -(-n // block)
    pad = torch.zeros(H, nb * block, D, dtype=torch.float64, device=X.device)
    pad[:, :n] = X.double()
    pad = pad.view(H, nb, block, D)
    e = torch.tensor([[exponent(pad[h, b]) for b in range(nb)] for h in range(H)], device=X.device).view(H, nb)
    codes = e4m3(pad / pow2(e)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(H, nb * block, D)[:, :n]
    return codes.contiguous().view(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def as_bytes(x):
    return x.view(torch.uint8)


def values(codes, scale, block, dtype=torch.float64):
    """The numbers that a cache in 8 bits stands for, [H, rows, D]."""
    x = as_bytes(codes).contiguous().view(torch.float8_e4m3fn).to(dtype)
    s = pow2(as_bytes(scale).long() - 127).to(dtype)
    return x * s.repeat_interleave(block, 1)[:, : x.shape[1], None]


def attend(q, K, V, seen, scale=None):
    """q [R, D], K / V [T, D], seen bool [R, T]: (out, the same of |V|, lse, the largest sum of a logit's terms' sizes) in 64 bits;
    0, 0, -inf and 0 where nothing is seen."""
    q, K, V = q.double(), K.double(), V.double()
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    if K.shape[0] == 0:
        none = torch.full(q.shape[:1], -math.inf, dtype=torch.float64, device=q.device)
        return torch.zeros_like(q), torch.zeros_like(q), none, torch.zeros_like(none)
    z = ((q @ K.t().contiguous()) * scale).masked_fill(~seen, -math.inf)
    terms = ((q.abs() @ K.abs().t().contiguous()) * scale).masked_fill(~seen, 0.0).amax(1)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse.masked_fill(lse == -math.inf, 0.0)[:, None])
    return p @ V, p @ V.abs(), lse, terms


# Weights below 2^-126 of the largest are 0: of fewer than 2^20 keys whose values are below 2^6, 2^-100 of the sum at most.
TINY = 2.0 ** -100


def f32_bar(terms):
    """How far a result in 32 bits may be off, relative to `size` = sum p |V| / sum p.  A logit's 128 exact products are added up in
    eight matrix instructions: roundings of 2^-24 of a sum that grows to `terms` and is half of it in the mean, 2^-22 of it in all.
    That counts twice, in a weight and in their sum, and the exponent's own roundings (product with the scale, 2^-24, and the
    scale's, 2^-24) add as much again: 2^-20.  Exponentials and the sums over the keys are off by units of 2^-24: 1e-5 covers them."""
    return 1e-5 + 2.0 ** -20 * terms
