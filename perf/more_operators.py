"""The measured cases of attention over a cache in 8 bits and with a sliding window, and the same in elementary torch
operations.

A case is one pass through one of three operators, head dim 128:

  append  dsk_kv8_append: new tokens' keys normed, rotated and put with the values into a cache of 8-bit codes (e4m3) with
          one power-of-two scale for each block of rows and head; the queries normed and rotated in the same pass
  window  dsk_window_attn: causal attention of the new tokens (one of a decoding step to a whole prompt) over a cache in
          bf16 or in 8 bits; a token sees the `window` last tokens, itself among them, and the first `sinks`
  sparse  dsk_window_sparse_decode_attn: one new token per sequence sees the selected slots, the `window` last tokens and
          the first `sinks`, each token once

Head counts and lengths are those of the library's own workloads (one head at 4K tokens; 32 query / 8 KV heads up to
128K tokens; 40 heads without grouping at 128K tokens; eight ragged sequences of 16K to 64K tokens); `draw` gives
anything between.  K and V are Gaussian with four outlier channels per KV head scaled by 8, queries are Gaussian.
Where `own` is true, `prepare` also makes the argument structs and workspaces that a serving program keeps.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128                  # head dim of the library
THETA = 500000.0         # base of the rotation's frequencies
EPS = 1e-6
EVERY = 0x7FFFFFFF       # a window that hides nothing
E_MIN, E_MAX = -100, 120  # exponents of the scales

DEFAULTS = dict(B=1, ragged=0.0, Hq=32, Hkv=8, tokens=32768, new=1, window=EVERY, sinks=0, bits=8, block=32, layout="hnd",
                out="bf16", budget=0, b=16, shared=False, rot=128, inter=False, norm=True)


def _case(kind, **kw):
    c = dict(DEFAULTS, kind=kind)
    c.update(kw)
    return c


def listed():
    return [
        # one decoding step of a small batch: latency and nothing else
        _case("append", name="append_decode_b8", B=8, ragged=0.6, tokens=65521),
        # a long prompt, written into an empty cache in one pass
        _case("append", name="append_prompt_32k", tokens=0, new=32768),
        # ragged prompts of a model without grouped heads that go on in the middle of a block, a quarter of the channels
        # rotated in neighbouring pairs, no norm, larger blocks, token-major cache
        _case("append", name="append_mha_ragged", B=5, ragged=0.7, Hq=40, Hkv=40, tokens=333, new=4099, block=64, rot=32,
              inter=True, norm=False, layout="nhd"),
        # a small draft model on one short request, in 32 bits (its logits are compared)
        _case("window", name="window_1head_4k", Hq=1, Hkv=1, tokens=4095, bits=16, out="f32"),
        # a decoding step of a batch whose layer sees a window and a few first tokens only, cache in bf16
        _case("window", name="window_decode_b16_sinks", B=16, ragged=0.5, tokens=32768, window=4096, sinks=4, bits=16),
        # a decoding step at the longest context of a grouped-query model, the whole cache in 8 bits
        _case("window", name="window_decode8_128k", tokens=131071),
        # a serving batch of ragged contexts in 8 bits, four new tokens each, token-major cache, larger blocks
        _case("window", name="window_step8_b8_ragged", B=8, ragged=0.75, tokens=65521, new=4, layout="nhd", block=64),
        # a whole prompt, plain causal attention
        _case("window", name="window_prompt_8k", tokens=0, new=8191, bits=16),
        # a piece of a long prompt over what the cache holds of it in 8 bits, a window and a few first tokens
        _case("window", name="window_piece8_sinks", tokens=30011, new=2048, window=4096, sinks=4),
        # a model without grouped heads at the longest context: the most K and V
        _case("window", name="window_mha8_128k", Hq=40, Hkv=40, tokens=131071),
        # the headline configuration's selection per query head, from a cache in 8 bits, with what is near
        _case("sparse", name="sparse8_128k", tokens=131072, budget=4096, b=32, window=128, sinks=4),
        # a serving batch of ragged contexts, one selection per KV head, the newest tokens not yet in the tables
        _case("sparse", name="sparse8_b8_shared", B=8, ragged=0.75, tokens=65521, budget=4096, b=16, window=1024, sinks=16,
              shared=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    kind = rng.choice(["window"] * 5 + ["sparse"] * 3 + ["append"] * 3)
    Hq, Hkv = rng.choice([(1, 1), (8, 8), (16, 2), (28, 4), (32, 8), (32, 8), (40, 8), (64, 8), (40, 40)])
    B = rng.choice([1, 1, 2, 3, 5, 8, 16])
    c = dict(Hq=Hq, Hkv=Hkv, B=B, ragged=round(rng.uniform(0.0, 0.9), 3) if B > 1 else 0.0, block=rng.choice([32, 32, 64, 128]),
             layout=rng.choice(["hnd", "hnd", "nhd"]))
    if kind == "append":
        c.update(new=_log_int(rng, 1, 32768 * 48 // (B * (Hq + 2 * Hkv))), tokens=_log_int(rng, 1, 131072),
                 rot=rng.choice([128, 128, 128, 96, 64, 32, 16]), inter=rng.random() < 0.3, norm=rng.random() < 0.7)
        return _case(kind, **c)
    c.update(bits=rng.choice([8, 8, 8, 16]), out=rng.choice(["bf16", "bf16", "bf16", "f32"]), sinks=rng.choice([0, 0, 1, 4, 16, 64]))
    if kind == "sparse":
        b = rng.choice([8, 16, 32, 64])
        most = min(131072, 40 * 131072 // (Hkv * B * (c["bits"] // 8)))
        c.update(b=b, budget=_log_int(rng, b, 8192) // b * b, tokens=_log_int(rng, 1, most), shared=rng.random() < 0.5,
                 window=rng.choice([0, _log_int(rng, 1, 4096)]))
        return _case(kind, **c)
    new = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 8192)])
    # no more rows of K and V, products or logits than the listed
    flops = work(_case("window", tokens=0, new=8191))["flops"]
    hi = min(131072, 40 * 131072 // (Hkv * B * (c["bits"] // 8)), flops / (4.0 * D * Hq * new * B), 2e9 / (Hq * new * B))
    hi = max(int(hi) - new, 1)
    if 4.0 * D * Hq * B * new * new > flops:
        new = max(1, int(math.sqrt(flops / (4.0 * D * Hq * B))))
    c.update(new=new, tokens=_log_int(rng, 1, hi), window=rng.choice([EVERY, _log_int(rng, 1, 8192)]))
    return _case(kind, **c)


# ---- geometry that follows from a case alone ---------------------------------------------------
def _less(c, most, least):
    """`most` of the first sequence, the others lose up to `ragged` of it."""
    return [max(least, int(most * (1.0 - c["ragged"] * ((0.6180339887 * i) % 1.0)))) for i in range(c["B"])]


def _lens(c):
    return _less(c, c["tokens"], min(c["tokens"], 1))


def _news(c):
    return _less(c, c["new"], 1)


def _slots(c):
    """Selected slots of a sequence, of b tokens each but for the last."""
    return [min(c["budget"] // c["b"], -(-L // c["b"])) for L in _lens(c)]


def _visible(c, L, n):
    """Tokens that the n new ones behind L see in all, and the sum of what each of them sees."""
    W, F = c["window"], c["sinks"]
    first = max(0, L - W + 1)                                   # of the first new token's window
    any_ = L + n - first + min(F, first)
    p = range(L, L + n) if n <= 64 else range(L, L + n, 16)
    each = [min(W, x + 1) + min(F, max(0, x + 1 - W)) for x in p]
    return any_, sum(each) * (n / len(each))


def work(case):
    c = case
    lens, new, row = _lens(c), _news(c), D * c["bits"] // 8
    N = sum(new)
    if c["kind"] == "append":
        return {"bytes": N * (4 * c["Hq"] * D + 6 * c["Hkv"] * D) + 2 * N * c["Hkv"] // c["block"] + 4 * N, "flops": 0}
    out = 4 if c["out"] == "f32" else 2
    if c["kind"] == "sparse":
        near = [min(L, c["window"]) + min(c["sinks"], max(0, L - c["window"])) for L in lens]
        far = [0.75 * n * c["b"] for n in _slots(c)]            # slots are b/2 to b tokens long
        heads = c["Hkv"] if c["shared"] else c["Hq"]
        return {"bytes": 2 * row * (c["Hkv"] * sum(near) + heads * sum(far)) + c["B"] * c["Hq"] * (D * (2 + out) + 4),
                "flops": 4.0 * D * c["Hq"] * (sum(near) + sum(far))}
    seen = [_visible(c, L, n) for L, n in zip(lens, new)]
    return {"bytes": 2 * row * c["Hkv"] * sum(x for x, _ in seen) + N * c["Hq"] * (D * (2 + out) + 4),
            "flops": 4.0 * D * c["Hq"] * sum(x for _, x in seen)}


# ---- inputs ------------------------------------------------------------------------------------
def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _starts(v):
    out = [0]
    for x in v:
        out.append(out[-1] + int(x))
    return out


def _pow2(e):
    """2^e in 32 bits, e from -126 to 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _exponent(largest):
    """The least e with largest <= 448 * 2^e (448 = 0.875 * 2^9 is the largest e4m3 value)."""
    m, x = torch.frexp(largest.float())
    return (x - 9 + (m > 0.875).int()).masked_fill(largest == 0, E_MIN).clamp(E_MIN, E_MAX)


def _cache(c, g, rows, empty=False):
    """K or V of all heads as (rows [Hkv, rows, D] in the case's layout, scales [Hkv, rows / block] or None): Gaussian,
    four channels of each head scaled by 8."""
    H, S = c["Hkv"], c["block"]
    dtype = torch.bfloat16 if c["bits"] == 16 else torch.uint8
    X = torch.empty((rows, H, D) if c["layout"] == "nhd" else (H, rows, D), dtype=dtype, device="cuda")
    X = X.transpose(0, 1) if c["layout"] == "nhd" else X
    scale = torch.empty(H, -(-rows // S), dtype=torch.uint8, device="cuda") if c["bits"] == 8 else None
    loud = torch.ones(H, 1, D, device="cuda")
    loud.scatter_(2, torch.rand(H, 1, D, generator=g, device="cuda").argsort(-1)[..., :4], 8.0)
    for h in range(H):
        x = torch.randn(rows, D, generator=g, device="cuda") * loud[h]
        if empty:
            x.zero_()
        if c["bits"] == 16:
            X[h] = x
        else:
            x = x.bfloat16().float().view(-1, S, D)
            e = _exponent(x.abs().amax((1, 2)))
            X[h] = (x * _pow2(-e)[:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(rows, D)
            scale[h] = (e + 127).byte()
    if c["bits"] == 8:
        X, scale = X.view(torch.float8_e4m3fn), scale.view(torch.float8_e8m0fnu)
    return X, scale


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    lens, new, S = _lens(c), _news(c), c["block"]
    s = dict(c=c, new=new, most=max(new), n_new=_i32(new), cu=_i32(_starts(new)), N=sum(new))
    if c["kind"] == "append":
        # the step writes far into long sequences: the cache itself holds the end of each, a block begun among it
        far = _i32([max(0, L - 1024) for L in lens])
        lens = [L if L <= 1024 else 32 + L % 97 for L in lens]
    room = [-(-(L + n + 16) // S) * S for L, n in zip(lens, new)]      # regions begin with a block
    s.update(lens=lens, rows=sum(room), row0=_i32(_starts(room)[:-1]), len=_i32(lens))
    s["K"], s["k_scale"] = _cache(c, g, s["rows"], empty=c["kind"] == "append" and not c["tokens"])
    s["V"], s["v_scale"] = _cache(c, g, s["rows"], empty=c["kind"] == "append" and not c["tokens"])
    if c["kind"] == "append":
        x = torch.randn(s["N"], c["Hq"] + 2 * c["Hkv"], D, generator=g, device="cuda")   # one fused projection's output
        x = x.mul_(torch.exp(torch.randn(s["N"], 1, 1, generator=g, device="cuda"))).bfloat16()
        s["q"], s["k"], s["v"] = x[:, : c["Hq"]], x[:, c["Hq"]: c["Hq"] + c["Hkv"]], x[:, c["Hq"] + c["Hkv"]:]
        seq, i = _tokens(s)
        s["pos"] = (s["len"] + far)[seq] + i.int()
        s["inv_freq"] = (THETA ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda") / c["rot"])).float()
        s["wq"] = s["wk"] = None
        if c["norm"]:
            s["wq"] = 1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")
            s["wk"] = 1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")
        s["q_out"] = torch.zeros(s["N"], c["Hq"], D, dtype=torch.bfloat16, device="cuda")
        return s
    n = c["B"] if c["kind"] == "sparse" else s["N"]
    s["q"] = torch.randn(n, c["Hq"], D, generator=g, device="cuda").bfloat16()
    if c["kind"] == "sparse":
        heads, k = c["Hkv"] if c["shared"] else c["Hq"], c["budget"] // c["b"]
        start = torch.zeros(c["B"], heads, k, dtype=torch.int32, device="cuda")
        length, count = torch.zeros_like(start), torch.zeros(c["B"], heads, dtype=torch.int32, device="cuda")
        for i, (L, r0) in enumerate(zip(lens, _starts(room))):
            slots = -(-L // c["b"])
            n = min(k, slots)
            pick = torch.rand(heads, slots, generator=g, device="cuda").argsort(-1)[:, :n].sort(-1).values
            full = torch.randint((c["b"] + 1) // 2, c["b"] + 1, pick.shape, generator=g, device="cuda")
            start[i, :, :n] = (r0 + pick * c["b"]).int()
            length[i, :, :n] = torch.minimum(full, L - pick * c["b"]).int()
            count[i] = n
        s["sel"] = (start, length, count)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        s["call"] = _handle(s)
    return s


# ---- the plain forms ---------------------------------------------------------------------------
def _tokens(s):
    """Sequence and place in it of every new token."""
    t = torch.arange(s["N"], device="cuda")
    seq = torch.searchsorted(s["cu"][1:].long(), t, right=True)
    return seq, t - s["cu"].long()[seq]


def _turn(x, w, s):
    """Norm over the channels, then the rotation; x [N, heads, D] in 32 bits."""
    c = s["c"]
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
    angle = s["pos"].double()[:, None] * s["inv_freq"].double()               # 64 bits: positions go far
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    rot, rest = x[..., : c["rot"]], x[..., c["rot"]:]
    a, b = (rot[..., 0::2], rot[..., 1::2]) if c["inter"] else rot.chunk(2, -1)
    a, b = a * cos - b * sin, a * sin + b * cos
    rot = torch.stack([a, b], -1).flatten(-2) if c["inter"] else torch.cat([a, b], -1)
    return torch.cat([rot, rest], -1)


def _put(X, scale, x, s):
    """x [N, Hkv, D] in 32 bits into the blocks of X, where a block's scale may have to grow for them."""
    S, seq, i = s["c"]["block"], *_tokens(s)
    codes, scale = X.view(torch.uint8), scale.view(torch.uint8)
    end = (s["row0"] + s["len"]).long()                                       # first new row of every sequence
    row = end[seq] + i
    largest = torch.zeros(scale.shape, device="cuda").index_reduce_(1, row // S, x.abs().amax(-1).t(), "amax")
    need = _exponent(largest)
    # blocks that are begun keep their scale, or take the larger one and their rows with it
    first = end // S                                                          # [B]
    begun = end % S > 0
    before = scale[:, first].int() - 127                                      # [Hkv, B]
    grown = torch.where(begun, torch.maximum(need[:, first], before), need[:, first])
    old = first[:, None] * S + torch.arange(S, device="cuda")
    y = codes[:, old].view(torch.float8_e4m3fn).float() * torch.pow(2.0, (before - grown).float())[..., None, None]
    y = y.to(torch.float8_e4m3fn).view(torch.uint8)
    codes[:, old] = torch.where((old < end[:, None])[..., None], y, codes[:, old])
    need[:, first] = grown
    touched = torch.zeros(scale.shape[1], dtype=torch.bool, device="cuda")
    touched[row // S] = True
    scale.copy_(torch.where(touched, (need + 127).byte(), scale))
    codes[:, row] = (x.transpose(0, 1) * _pow2(-need[:, row // S])[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)


def _append(s):
    s["q_out"].copy_(_turn(s["q"].float(), s["wq"], s))
    _put(s["K"], s["k_scale"], _turn(s["k"].float(), s["wk"], s), s)
    _put(s["V"], s["v_scale"], s["v"].float(), s)
    return {"q": s["q_out"], "K": s["K"], "V": s["V"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _rows(X, scale, heads, row, S):
    """The rows of the cache in 32 bits: heads and row index its first two axes."""
    if scale is None:
        return X[heads, row].float()
    x = X.view(torch.uint8)[heads, row].view(torch.float8_e4m3fn).float()
    return x * _pow2(scale.view(torch.uint8)[heads, row // S].int() - 127)[..., None]


def _attend(z, seen, values):
    """Softmax of the logits that are seen, times the values; z [..., queries, keys]."""
    z = z.masked_fill_(~seen, -math.inf)
    top = z.amax(-1)
    top = torch.where(top == -math.inf, 0.0, top)[..., None]
    z = z.sub_(top).exp_()
    den = z.sum(-1)
    out = torch.matmul(z, values) / torch.where(den > 0, den, 1.0)[..., None]
    return out, torch.log(den) + top[..., 0]


def _window(s):
    c = s["c"]
    B, Hkv, G, M, F = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], s["most"], c["sinks"]
    # the tokens that a sequence's new ones see: a few first ones, and from the first one's window on
    lo = [max(0, L - c["window"] + 1) for L in s["lens"]]
    most = max(L + n - f for L, n, f in zip(s["lens"], s["new"], lo))
    lo = _i32(lo).long()
    few = torch.arange(F, device="cuda").expand(B, F)
    t = torch.cat([few, lo[:, None] + torch.arange(most, device="cuda")], 1)   # [B, keys]: positions
    there = torch.cat([few < lo[:, None], torch.ones(B, most, dtype=torch.bool, device="cuda")], 1)
    there &= t < (s["len"] + s["n_new"])[:, None]
    row = torch.where(there, s["row0"].long()[:, None] + t, 0)[:, None]
    heads = torch.arange(Hkv, device="cuda")[:, None]
    i = torch.arange(M, device="cuda")
    real = i < s["n_new"][:, None]                                             # [B, M]
    at = torch.where(real, s["cu"].long()[:-1, None] + i, 0)                   # token of every query
    q = s["q"][at].float().view(B, M, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, M * G, D)
    p = (s["len"].long()[:, None] + i)[..., None]                              # its position
    t = t[:, None]
    seen = there[:, None] & (t <= p) & ((t > p - c["window"]) | (t < F))       # [B, M, keys]
    seen = seen[:, :, None].expand(-1, -1, G, -1).flatten(1, 2)[:, None]
    z = torch.matmul(q, _rows(s["K"], s["k_scale"], heads, row, c["block"]).transpose(-1, -2)) * (1.0 / math.sqrt(D))
    out, lse = _attend(z, seen, _rows(s["V"], s["v_scale"], heads, row, c["block"]))
    seq, i = _tokens(s)
    out = out.view(B, Hkv, M, G, D).permute(0, 2, 1, 3, 4)[seq, i].reshape(s["N"], c["Hq"], D)
    lse = lse.view(B, Hkv, M, G).permute(0, 2, 1, 3)[seq, i].reshape(s["N"], c["Hq"])
    return {"out": out if c["out"] == "f32" else out.bfloat16(), "lse": lse}


def _sparse(s):
    c = s["c"]
    start, length, count = s["sel"]
    B, H, F, W = c["B"], start.shape[1], c["sinks"], c["window"]
    R = c["Hq"] // H                                                           # queries of a selection
    row0, end = s["row0"].long()[:, None], (s["row0"] + s["len"]).long()[:, None]
    near = torch.maximum(end - W, row0)                                        # first row of the window
    off = torch.arange(c["b"], device="cuda")
    far = (start.long()[..., None] + off).flatten(2)                           # [B, H, keys]
    there = (off < length[..., None]) & (torch.arange(start.shape[2], device="cuda")[:, None] < count[..., None, None])
    there = there.flatten(2) & (far >= (row0 + F)[..., None]) & (far < near[..., None])
    few = row0 + torch.arange(F, device="cuda")
    win = near + torch.arange(min(W, max(s["lens"])), device="cuda")
    extra = torch.cat([few, win], 1)                                           # [B, keys]
    here = torch.cat([few < near, win < end], 1)
    row = torch.cat([far, extra[:, None].expand(-1, H, -1)], 2)
    there = torch.cat([there, here[:, None].expand(-1, H, -1)], 2)
    row = torch.where(there, row, 0)
    heads = (torch.arange(H, device="cuda") // (H // c["Hkv"]))[:, None]
    q = s["q"].float().view(B, H, R, D)
    z = torch.matmul(q, _rows(s["K"], s["k_scale"], heads, row, c["block"]).transpose(-1, -2)) * (1.0 / math.sqrt(D))
    out, lse = _attend(z, there[:, :, None], _rows(s["V"], s["v_scale"], heads, row, c["block"]))
    out, lse = out.view(B, c["Hq"], D), lse.view(B, c["Hq"])
    return {"out": out if c["out"] == "f32" else out.bfloat16(), "lse": lse}


# ---- the framework's calls ---------------------------------------------------------------------
def _handle(s):
    """What a serving program keeps for the call: outputs, argument struct, workspace."""
    import paper_2602_03184_amd as dsk
    c = s["c"]
    if c["kind"] == "append":
        return dsk.make_kv8_appender(s["k"], s["v"], s["K"], s["V"], s["k_scale"], s["v_scale"], scale_block=c["block"],
                                     seq_row0=s["row0"], seq_len=s["len"], cu_new=s["cu"], max_new=s["most"], q=s["q"],
                                     q_out=s["q_out"], pos=s["pos"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS,
                                     inv_freq=s["inv_freq"], interleaved=c["inter"])
    kw = dict(seq_row0=s["row0"], seq_len=s["len"], window=c["window"], n_sink=c["sinks"], k_scale=s["k_scale"],
              v_scale=s["v_scale"], scale_block=c["block"], want_f32=c["out"] == "f32", want_bf16=c["out"] != "f32")
    if c["kind"] == "sparse":
        start, length, count = s["sel"]
        return dsk.make_window_sparse_args(s["q"], s["K"], s["V"], sel_start=start, sel_len=length, sel_count=count, b=c["b"],
                                           **kw)
    return dsk.make_window_attn_args(s["q"], s["K"], s["V"], cu_new=s["cu"], max_new=s["most"], max_seqlen=max(s["lens"]), **kw)


def _call(s):
    import paper_2602_03184_amd as dsk
    h, kind = s["call"], s["c"]["kind"]
    if kind == "append":
        dsk.dsk_kv8_append(h.args)
        return {"q": s["q_out"], "K": s["K"], "V": s["V"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if kind == "sparse":
        dsk.dsk_window_sparse_decode_attn(h.args)
    else:
        dsk.dsk_window_attn(h.args)
    return {"out": h.out if s["c"]["out"] == "f32" else h.out_bf16, "lse": h.lse}


def run(state):
    if own:
        return _call(state)
    return {"append": _append, "window": _window, "sparse": _sparse}[state["c"]["kind"]](state)


# ---- the same from the definitions, in 64 bits -------------------------------------------------
def _exact_turn(x, w, s):
    """Rows of every token [N, heads, D], 64 bits, as complex numbers turned by their angles."""
    c = s["c"]
    if w is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
    half = c["rot"] // 2
    z = torch.view_as_complex(x[..., : c["rot"]].unflatten(-1, (half, 2) if c["inter"] else (2, half)).transpose(
        -1, -1 if c["inter"] else -2).contiguous())
    t = torch.outer(s["pos"].double(), s["inv_freq"].double())
    z = z * torch.polar(torch.ones_like(t), t)[:, None]
    y = x.clone()
    y[..., : c["rot"]] = torch.view_as_real(z).transpose(-1, -1 if c["inter"] else -2).flatten(-2)
    return y


def _e4m3(x):
    """The nearest e4m3 value, ties to the even one: steps of an eighth of the power of two below, 2^-9 at least."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_put(X, scale, x, s):
    S, H = s["c"]["block"], s["c"]["Hkv"]
    codes = X.view(torch.uint8).view(torch.float8_e4m3fn).double()
    scale = (scale.view(torch.uint8).double() - 127).exp2()
    row0, cu = s["row0"].tolist(), s["cu"].tolist()
    for b, (L, n) in enumerate(zip(s["lens"], s["new"])):
        first = (row0[b] + L) // S * S                                         # of the first block that is written
        last = -(-(row0[b] + L + n) // S) * S
        got = row0[b] + L - first                                              # rows that it has already
        y = torch.zeros(H, last - first, D, dtype=torch.float64, device="cuda")
        y[:, got: got + n] = x[cu[b]: cu[b + 1]].transpose(0, 1)
        y = y.view(H, -1, S, D)
        least = torch.ceil(torch.log2(y.abs().amax((2, 3)) / 448.0)).clamp(E_MIN, E_MAX)
        old = codes[:, first: first + got].clone()
        if got:
            was = scale[:, first // S].log2()
            least[:, 0] = torch.maximum(least[:, 0], was)
            old = _e4m3(old * (was - least[:, 0]).exp2()[:, None, None])
        scale[:, first // S: last // S] = least.exp2()
        y = _e4m3(y / least.exp2()[:, :, None, None]).view(H, -1, D)
        codes[:, first: first + got] = old
        codes[:, first + got: first + got + n] = y[:, got: got + n]
    return codes, scale


def _exact_rows(X, scale, h, rows, S):
    if scale is None:
        return X[h][rows].double()
    x = X[h].view(torch.uint8)[rows].view(torch.float8_e4m3fn).double()
    return x * (scale[h].view(torch.uint8)[rows // S].double() - 127).exp2()[:, None]


def _exact_attend(q, k, v, seen):
    z = (q @ k.t().contiguous() / math.sqrt(D)).masked_fill(~seen, -math.inf)
    return torch.softmax(z, 1).nan_to_num(0.0) @ v, torch.logsumexp(z, 1)


def exact(case, seed):
    s = _inputs(case, seed)
    c, S = s["c"], s["c"]["block"]
    if c["kind"] == "append":
        K, ks = _exact_put(s["K"], s["k_scale"], _exact_turn(s["k"].double(), s["wk"], s), s)
        V, vs = _exact_put(s["V"], s["v_scale"], s["v"].double(), s)
        return {"q": _exact_turn(s["q"].double(), s["wq"], s), "K": K, "V": V, "k_scale": ks, "v_scale": vs}
    G, F, W = c["Hq"] // c["Hkv"], c["sinks"], c["window"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    row0, cu = s["row0"].tolist(), s["cu"].tolist()
    for b, (L, n) in enumerate(zip(s["lens"], s["new"])):
        if c["kind"] == "sparse":
            start, length, count = (x[b].tolist() for x in s["sel"])
            for h in range(c["Hq"]):
                j = h // G if c["shared"] else h
                pick = [torch.arange(x, x + y, device="cuda") for x, y in zip(start[j][:count[j]], length[j])]
                near = [torch.arange(row0[b], row0[b] + min(F, L), device="cuda"),
                        torch.arange(row0[b] + max(0, L - W), row0[b] + L, device="cuda")]
                rows = torch.unique(torch.cat(pick + near))
                k, v = (_exact_rows(X, y, h // G, rows, S) for X, y in ((s["K"], s["k_scale"]), (s["V"], s["v_scale"])))
                all_ = torch.ones(1, len(rows), dtype=torch.bool, device="cuda")
                o, l = _exact_attend(s["q"][b, h: h + 1].double(), k, v, all_)
                out[b, h], lse[b, h] = o[0], l[0]
            continue
        t = torch.arange(L + n, device="cuda")
        p = t[L:, None]
        seen = (t <= p) & ((p - t < W) | (t < F))
        keep = seen.any(0).nonzero()[:, 0]
        seen = seen[:, keep].repeat_interleave(G, 0)
        for h in range(c["Hkv"]):
            k, v = (_exact_rows(X, y, h, row0[b] + keep, S) for X, y in ((s["K"], s["k_scale"]), (s["V"], s["v_scale"])))
            mine = slice(cu[b], cu[b + 1]), slice(h * G, (h + 1) * G)
            o, l = _exact_attend(s["q"][mine].double().reshape(n * G, D), k, v, seen)
            out[mine], lse[mine] = o.view(n, G, D), l.view(n, G)
    return {"out": out, "lse": lse}
