"""dsk_window_attn against the definition in 64 bits, on the numbers that the cache stands for (codes * scale without rounding).
Bars: f32_bar() of size = sum p |V| / sum p.  bf16 outputs: weights of two terms are off by 2^-16, single ones by half a step, 2^-8 of
each and so of the size, the result once more, 2^-8 of it."""
import math

import pytest
import torch

from step_testutil import i32, starts
from window_testutil import D, TINY, as_bytes, attend, f32_bar, quantise, values

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8
ALL = 0x7FFFFFFF


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


class Case:
    """A batch with a region per sequence, K and V with outlier channels, and its reference."""

    def __init__(self, lens, new, Hq, Hkv, *, bits=8, block=32, window=ALL, sinks=0, nhd=False, seed=0, spare=3, pad=0, sharp=1.0,
                 aligned=True):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.lens, self.new, self.Hq, self.Hkv, self.bits, self.block = lens, new, Hq, Hkv, bits, block
        self.window, self.sinks = window, sinks
        room = [a + b + spare for a, b in zip(lens, new)]
        if bits == 8 and aligned:
            room = [-(-x // block) * block for x in room]
        self.row0 = starts(room)
        self.cu, self.rows = starts(new), self.row0[-1]
        self.N = self.cu[-1] + pad

        def cache():
            X = torch.randn(Hkv, max(self.rows, 1), D, generator=g, device="cuda")
            X[..., 7::31] *= 4.0
            X *= torch.exp(torch.randn(Hkv, max(self.rows, 1), 1, generator=g, device="cuda"))
            X, scale = (X.bfloat16(), None) if bits == 16 else quantise(X, block)
            if nhd:
                wide = torch.zeros(X.shape[1], Hkv, D + 32, dtype=torch.bfloat16 if bits == 16 else torch.uint8, device="cuda")
                view = wide[..., :D].transpose(0, 1)
                view.copy_(X if bits == 16 else as_bytes(X))
                X = view if bits == 16 else view.view(torch.float8_e4m3fn)
            return X, scale
        (self.K, self.ks), (self.V, self.vs) = cache(), cache()
        self.q = (torch.randn(max(self.N, 1), Hq, D, generator=g, device="cuda") * sharp).bfloat16()[: self.N]

    def numbers(self):
        if self.bits == 16:
            return self.K.double(), self.V.double()
        return values(self.K, self.ks, self.block), values(self.V, self.vs, self.block)

    def kwargs(self, **over):
        kw = dict(seq_row0=i32(self.row0[:-1]), seq_len=i32(self.lens), cu_new=i32(self.cu), max_new=max(max(self.new), 1),
                  max_seqlen=max(self.lens), window=self.window, n_sink=self.sinks, k_scale=self.ks, v_scale=self.vs,
                  scale_block=self.block)
        kw.update(over)
        return kw

    def run(self, **over):
        r = _dsk().make_window_attn_args(self.q, self.K, self.V, **self.kwargs(**over))
        for t in (r.out, r.out_bf16, r.lse):
            if t is not None:
                t.fill_(9.0)
        r.step()
        torch.cuda.synchronize()
        return r

    def seen(self, s):
        L, n = self.lens[s], self.new[s]
        t = torch.arange(L + n, device="cuda")
        p = t[L:, None]
        return (t <= p) & ((p - t < self.window) | (t < self.sinks))

    def reference(self, scale=None):
        G = self.Hq // self.Hkv
        K, V = self.numbers()
        out, size = (torch.zeros(self.cu[-1], self.Hq, D, dtype=torch.float64, device="cuda") for _ in range(2))
        lse, bar = (torch.zeros(self.cu[-1], self.Hq, dtype=torch.float64, device="cuda") for _ in range(2))
        for s, n in enumerate(self.new):
            t, seen = slice(self.cu[s], self.cu[s + 1]), self.seen(s).repeat_interleave(G, 0)
            for h in range(self.Hkv):
                hs, rows = slice(h * G, (h + 1) * G), slice(self.row0[s], self.row0[s] + self.lens[s] + n)
                o, z, l, terms = attend(self.q[t, hs].reshape(n * G, D), K[h, rows], V[h, rows], seen, scale)
                out[t, hs], size[t, hs], lse[t, hs] = o.view(n, G, D), z.view(n, G, D), l.view(n, G)
                bar[t, hs] = f32_bar(terms).view(n, G)
        return out, size, lse, bar

    def check(self, scale=None, want=None):
        out, size, lse, bar = self.reference(scale) if want is None else want
        n = self.cu[-1]
        sc = 0.0 if scale is None else scale
        a = self.run(scale=sc)
        b = self.run(scale=sc, want_f32=False, want_bf16=True)
        c = self.run(scale=sc, want_bf16=True)
        weights = 2.0 ** -16 if max(self.new) * self.Hq // self.Hkv <= 64 else BF16
        assert bool(((a.out[:n].double() - out).abs() <= bar[..., None] * size + TINY).all())
        assert bool(((b.out_bf16[:n].double() - out).abs() <= BF16 * (1 + BF16) * out.abs() + (weights * (1 + BF16) + bar[..., None]) * size + TINY).all())
        assert torch.equal(c.out[:n], a.out[:n]) and torch.equal(c.out_bf16[:n], a.out[:n].bfloat16())
        fine = torch.isfinite(lse)
        for r in (a, b, c):
            got = r.lse[:n].double()
            assert torch.equal(got[~fine], lse[~fine])
            assert bool(((got - lse)[fine].abs() <= bar[fine] + 1e-5 * lse[fine].abs()).all())
            for t in (r.out, r.out_bf16, r.lse):                 # rows behind the last sequence stay as they were
                assert t is None or bool((t[n:] == 9.0).all())
        return a


LENS = [0, 1, 31, 32, 33, 64, 127, 129, 700, 1025]


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (8, 8), (8, 2), (6, 2), (5, 1), (16, 2), (14, 2), (40, 1)])
@pytest.mark.parametrize("new", [1, 2, 7, 16, 33])
def test_group_widths_and_ragged_lengths(Hq, Hkv, new, bits):
    n = [max(0, new - (s % 3)) for s in range(len(LENS))]
    Case(LENS, n, Hq, Hkv, bits=bits, seed=new, nhd=new == 7, block=(32, 64, 128)[new % 3], pad=2).check()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("window, sinks", [(1, 0), (1, 1), (5, 0), (31, 4), (32, 32), (33, 33), (64, 1), (100, 64), (100, 500), (640, 4), (5000, 4),
                                           (ALL, 7), (ALL, ALL), (7, ALL)])
@pytest.mark.parametrize("new", [1, 12, 150])
def test_windows_and_first_tokens(window, sinks, new, bits):
    Case([0, 3, 37, 300, 1000], [new, new, max(new - 1, 1), 0, new], 8, 2, bits=bits, window=window, sinks=sinks, seed=window % 97 + new).check()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("Hq, Hkv, new", [(4, 4, 300), (8, 2, 257), (8, 1, 130), (3, 1, 1000)])
def test_prompts(Hq, Hkv, new, bits):
    Case([0, 45, 600], [new, new // 3, new], Hq, Hkv, bits=bits, seed=new, nhd=new == 257).check()
    Case([0, 45, 600], [new, new // 3, new], Hq, Hkv, bits=bits, seed=new, window=70, sinks=3).check()


@pytest.mark.parametrize("bits", [8, 16])
def test_long_contexts_split_over_many_workgroups(bits):
    Case([20011, 40000, 3], [1, 1, 1], 8, 2, bits=bits, seed=8).check()
    Case([20011, 40000, 3], [4, 1, 4], 8, 2, bits=bits, seed=8, window=30000, sinks=40).check()
    Case([33333], [16], 4, 4, bits=bits, seed=9, nhd=True, block=128).check()
    Case([9000], [128], 8, 1, bits=bits, seed=10).check()
    Case([70001], [3], 1, 1, bits=bits, seed=11).check()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("end", [4095, 4096, 4097, 4127, 4159, 4223, 4351])
def test_the_cache_ends_in_any_place_of_a_tile(end, bits):
    Case([end], [1], 8, 2, bits=bits, seed=end, spare=0).check()
    Case([end - 40], [40], 8, 2, bits=bits, seed=end, spare=0, window=999).check()


def test_sequences_that_begin_within_a_block_of_scales():
    c = Case([50, 300], [9, 70], 8, 2, seed=5, aligned=False, spare=1)
    assert c.row0[1] % 32
    c.check()


def test_scale_and_sharp_logits():
    for bits in (8, 16):
        c = Case([300, 40], [9, 9], 8, 2, seed=6, bits=bits)
        c.check(scale=0.03)
    # one key takes nearly all the weight
    Case([300, 40], [9, 9], 8, 2, seed=7, sharp=8.0).check()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("new, window, sinks", [(1, 40, 3), (9, 40, 3), (9, ALL, 0), (150, 40, 35), (150, ALL, 0)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_seen_may_hold_anything(what, new, window, sinks, bits):
    """Rows that have left the window, rows of later tokens, the room behind every sequence and other sequences' rows."""
    if bits == 8:
        what = float("nan")                                      # there are no infinities
    c = Case([70, 0, 333], [new, new, 3], 8, 2, bits=bits, window=window, sinks=sinks, seed=13, spare=20)
    clean = [c.run(), c.run(want_f32=False, want_bf16=True)]

    def put(X, rows, value):
        if bits == 16:
            X[:, rows] = value
        else:
            as_bytes(X)[:, rows] = 0x7F if not isinstance(value, torch.Tensor) else value
    for s in range(3):
        for X in (c.K, c.V):                                     # the room
            put(X, slice(c.row0[s] + c.lens[s] + c.new[s], c.row0[s + 1]), what)
    for s in range(3):
        seen = c.seen(s)
        for t in {0, 5, max(c.lens[s] - 41, 0), c.lens[s], c.lens[s] + c.new[s] // 2, c.lens[s] + c.new[s] - 1}:
            if t >= c.lens[s] + c.new[s]:
                continue
            old = [(X if bits == 16 else as_bytes(X))[:, c.row0[s] + t].clone() for X in (c.K, c.V)]
            for X in (c.K, c.V):
                put(X, c.row0[s] + t, what)
            tok = torch.arange(c.cu[s], c.cu[s + 1], device="cuda")
            for r0, kw in zip(clean, ({}, dict(want_f32=False, want_bf16=True))):
                r = c.run(**kw)
                a, b = (x.out if x.out is not None else x.out_bf16 for x in (r, r0))
                blind, others = tok[~seen[:, t]], torch.cat([torch.arange(0, c.cu[s]), torch.arange(c.cu[s + 1], c.cu[-1])]).cuda()
                assert torch.equal(a[blind], b[blind]) and torch.equal(r.lse[blind], r0.lse[blind])
                assert torch.equal(a[others], b[others])
                assert not bool(torch.isfinite(a[tok[seen[:, t]]]).all(-1).any()) or not bool(seen[:, t].any())
            for X, o in zip((c.K, c.V), old):
                put(X, c.row0[s] + t, o)


@pytest.mark.parametrize("byte", [255, 254])
@pytest.mark.parametrize("new, window, sinks", [(1, 40, 3), (9, 45, 3), (9, ALL, 0), (150, 70, 35)])
def test_scales_of_blocks_that_are_not_seen_may_hold_anything(new, window, sinks, byte):
    """Also 255, which stands for no number; where it is seen, the result is none."""
    c = Case([170, 0, 333], [new, new, 3], 8, 2, window=window, sinks=sinks, seed=14, spare=7, aligned=False)
    clean = [c.run(), c.run(want_f32=False, want_bf16=True)]
    seen = torch.zeros(c.ks.shape[1] * 32, dtype=torch.bool, device="cuda")
    for s in range(3):
        seen[c.row0[s]: c.row0[s] + c.lens[s] + c.new[s]] = c.seen(s).any(0)
    unseen = ~seen.view(-1, 32).any(1)
    assert bool(unseen.any()) or window == ALL
    for X in (c.ks, c.vs):
        as_bytes(X)[:, unseen] = byte
    for r0, kw in zip(clean, ({}, dict(want_f32=False, want_bf16=True))):
        r = c.run(**kw)
        a, b = (x.out if x.out is not None else x.out_bf16 for x in (r, r0))
        assert torch.equal(a, b) and torch.equal(r.lse, r0.lse)
        if byte == 254:
            continue
        for blk in (0, (c.row0[0] + c.lens[0] + new // 2) // 32, (c.row0[2] + 300) // 32):
            old = as_bytes(c.vs)[:, blk].clone()
            as_bytes(c.vs)[:, blk] = 255
            r = c.run(**kw)
            a = r.out if r.out is not None else r.out_bf16
            meets = torch.cat([c.seen(s)[:, [t for t in range(c.lens[s] + c.new[s]) if (c.row0[s] + t) // 32 == blk]].any(1) for s in range(3)])
            assert torch.equal(a[~meets], b[~meets]) and torch.equal(r.lse[~meets], r0.lse[~meets])
            assert not bool(torch.isfinite(a[meets]).all(-1).any()) or not bool(meets.any())
            as_bytes(c.vs)[:, blk] = old


def test_an_infinity_that_is_seen_gives_that_infinity():
    for new, kw in ((1, {}), (9, {}), (150, dict(window=90, sinks=40))):
        c = Case([60], [new], 8, 2, bits=16, seed=14, **kw)
        seen = c.seen(0)
        c.V[:, 33, 5] = float("inf")
        c.V[:, 60 + new - 1, 6] = -float("inf")
        for out in (c.run().out, c.run(want_f32=False, want_bf16=True).out_bf16):
            assert torch.equal(out[..., 5] == float("inf"), seen[:, 33, None].expand(-1, 8))
            assert torch.equal(out[..., 6] == -float("inf"), seen[:, 60 + new - 1, None].expand(-1, 8))
            fine = [i for i in range(D) if i not in (5, 6)]
            assert bool(torch.isfinite(out[..., fine]).all())


@pytest.mark.parametrize("bits", [8, 16])
def test_a_nan_in_a_query_is_its_rows_alone(bits):
    for new in (1, 9, 150):
        c = Case([5000, 20], [new, new], 8, 2, bits=bits, seed=15)
        a = c.run()
        c.q[new // 2, 3, 17] = float("nan")
        b = c.run()
        assert bool(torch.isnan(b.out[new // 2, 3]).all()) and bool(torch.isnan(b.lse[new // 2, 3]))
        keep = torch.ones(2 * new, 8, dtype=torch.bool, device="cuda")
        keep[new // 2, 3] = False
        assert torch.equal(a.out[keep], b.out[keep]) and torch.equal(a.lse[keep], b.lse[keep])


@pytest.mark.parametrize("bits", [8, 16])
def test_malformed_tables_are_cut(bits):
    c = Case([64, 64], [8, 8], 4, 2, bits=bits, seed=14, spare=0, aligned=False)
    base = c.run()
    r = c.run(cu_new=i32([0, 8, 400]))                           # more tokens than there are rows and max_new
    assert torch.equal(r.out, base.out)
    r = c.run(cu_new=i32([0, 8, 3]))
    assert torch.equal(r.out[:8], base.out[:8]) and bool((r.out[8:] == 9.0).all())
    r = c.run(cu_new=i32([-1, 8, 16]))
    assert bool((r.out[:8] == 9.0).all()) and torch.equal(r.out[8:], base.out[8:])
    r = c.run(seq_len=i32([10 ** 9, 64]))                        # cut to max_seqlen = 64
    assert torch.equal(r.out, base.out)
    for kw in (dict(seq_row0=i32([-5, c.row0[1]])), dict(seq_len=i32([-5, 64])), dict(seq_row0=i32([2 ** 31 - 1, c.row0[1]])),
               dict(seq_row0=i32([c.rows, c.row0[1]]))):
        for more in ({}, dict(window=3, n_sink=2)):
            r = c.run(**kw, **more)
            assert bool((r.out[:8] == 0.0).all()) and bool((r.lse[:8] == -math.inf).all())
            assert more or torch.equal(r.out[8:], base.out[8:])
    r = c.run(seq_row0=i32([c.rows - 1, c.row0[1]]))             # one row is left: all tokens see it alone
    v = c.numbers()[1][:, -1].repeat_interleave(2, 0)
    assert bool(((r.out[:8].double() - v).abs() <= 1e-5 * v.abs()).all()) and torch.equal(r.out[8:], base.out[8:])
    r = c.run(seq_row0=i32([c.rows - 1, c.row0[1]]), window=3, n_sink=0)
    assert bool((r.out[:8] == 0.0).all()) and bool((r.lse[:8] == -math.inf).all())


def test_bit_identical_from_call_to_call_on_another_stream_and_in_a_graph():
    for bits in (8, 16):
        for new in ([1, 1], [20, 9], [300, 2]):
            c = Case([5000, 700], new, 8, 2, bits=bits, seed=15)
            a, b = c.run(), c.run()
            st = torch.cuda.Stream()
            r = _dsk().make_window_attn_args(c.q, c.K, c.V, **c.kwargs())
            torch.cuda.synchronize()
            r.step(st)
            st.synchronize()
            for x in (b, r):
                assert torch.equal(a.out, x.out) and torch.equal(a.lse, x.lse)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                r.step(st)
            for _ in range(3):
                r.out.zero_()
                c.run()
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(a.out, r.out) and torch.equal(a.lse, r.lse)


def test_one_token_equals_the_decode_attention():
    dsk = _dsk()
    c = Case([3000], [1], 32, 8, bits=16, seed=16, spare=0)
    den = dsk.dense_decode_attn(c.q, c.K, c.V, i32([0, c.rows]), c.rows)
    r = c.run()
    torch.cuda.synchronize()
    _, size, lse, bar = c.reference()                            # either is off by as much from the definition
    assert bool(((r.out - den.out).double().abs() <= 2 * bar[..., None] * size).all())
    assert bool(((r.lse - den.lse).double().abs() <= 2 * (bar + 1e-5 * lse.abs())).all())


@pytest.mark.parametrize("bits", [8, 16])
def test_pieces_of_a_prompt_give_what_the_whole_gives(bits):
    c = Case([0], [700], 8, 2, bits=bits, window=200, sinks=5, seed=17)
    whole = c.run()
    _, size, lse, bar = c.reference()
    at = 0
    for n in (1, 40, 300, 3, 356):
        kw = c.kwargs(seq_len=i32([at]), cu_new=i32([0, n]), max_new=n, max_seqlen=at)
        r = _dsk().window_attn(c.q[at: at + n].contiguous(), c.K, c.V, **kw)
        torch.cuda.synchronize()
        t = slice(at, at + n)                                    # either is off by as much from the definition
        assert bool(((r.out - whole.out[t]).double().abs() <= 2 * bar[t, :, None] * size[t] + TINY).all())
        assert bool(((r.lse - whole.lse[t]).double().abs() <= 2 * (bar[t] + 1e-5 * lse[t].abs())).all())
        at += n


def test_a_workspace_for_the_longest_cache_serves_shorter_ones():
    c = Case([9000, 100], [2, 2], 8, 2, seed=18)
    r = _dsk().make_window_attn_args(c.q, c.K, c.V, **c.kwargs(max_seqlen=120_000))
    for most in (120_000, 40_000, 9000):
        r.args.max_seqlen = most
        r.out.fill_(9.0)
        r.step()
        torch.cuda.synchronize()
        out, size, _, bar = c.reference()
        assert bool(((r.out.double() - out).abs() <= bar[..., None] * size + TINY).all())


def test_large_caches():
    """A cache whose rows lie beyond 2^32 bytes of a head's first, in both types."""
    for bits in (8, 16):
        width = bits // 8
        rows = (1 << 32) // (2 * D * width) + 128
        X = torch.zeros(rows, 2, D, dtype=torch.uint8 if bits == 8 else torch.bfloat16, device="cuda")
        c = Case([40], [9], 4, 1, bits=bits, seed=19, spare=0, aligned=False)
        row0 = (rows - 100) // 32 * 32
        K, V = (X[:, h:h + 1].transpose(0, 1) for h in range(2))
        for big, small in ((K, c.K), (V, c.V)):
            big[:, row0: row0 + 49] = small if bits == 16 else as_bytes(small)
        over = dict(seq_row0=i32([row0]))
        if bits == 8:
            K, V = K.view(torch.float8_e4m3fn), V.view(torch.float8_e4m3fn)
            for name, small in (("k_scale", c.ks), ("v_scale", c.vs)):
                s = torch.full((1, -(-rows // 32)), 127, dtype=torch.uint8, device="cuda")
                s[:, row0 // 32: row0 // 32 + 2] = as_bytes(small)
                over[name] = s.view(torch.float8_e8m0fnu)
        want = c.run()
        r = _dsk().window_attn(c.q, K, V, **c.kwargs(**over))
        torch.cuda.synchronize()
        assert torch.equal(r.out, want.out) and torch.equal(r.lse, want.lse)
        del X, K, V


def test_sequences_that_share_their_rows():
    """More tokens in all than the cache has rows, of different lengths: every part of every sequence is taken."""
    for bits in (8, 16):
        c = Case([30000, 29000, 5], [2, 2, 2], 8, 2, bits=bits, seed=20, spare=0)
        c.row0 = [0, 0, 0, c.row0[3]]
        c.lens = [30000, 21000, 29999]
        c.check()
        c = Case([9000] + [5] * 9, [2] * 10, 8, 2, bits=bits, seed=21, spare=0)
        c.row0 = [0] * 10 + [c.row0[10]]
        c.lens = [9000 - 31 * s for s in range(10)]
        c.check()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("new", [1, 150])
def test_large_caches_with_few_and_many_tokens(new, bits):
    """As above for the kernels of few and of many rows, whose result is in bf16."""
    rows = (1 << 32) // (2 * D * (bits // 8)) + 512
    X = torch.zeros(rows, 2, D, dtype=torch.uint8 if bits == 8 else torch.bfloat16, device="cuda")
    c = Case([140], [new], 4, 1, bits=bits, window=100, sinks=5, seed=20, spare=0, aligned=False)
    row0, n = (rows - 300) // 32 * 32, 140 + new
    K, V = (X[:, h:h + 1].transpose(0, 1) for h in range(2))
    for big, small in ((K, c.K), (V, c.V)):
        big[:, row0: row0 + n] = small if bits == 16 else as_bytes(small)
    over = dict(seq_row0=i32([row0]))
    if bits == 8:
        K, V = K.view(torch.float8_e4m3fn), V.view(torch.float8_e4m3fn)
        for name, small in (("k_scale", c.ks), ("v_scale", c.vs)):
            s = torch.full((1, -(-rows // 32)), 127, dtype=torch.uint8, device="cuda")
            s[:, row0 // 32: row0 // 32 + small.shape[1]] = as_bytes(small)
            over[name] = s.view(torch.float8_e8m0fnu)
    kw = dict(want_f32=False, want_bf16=True)
    want = c.run(**kw)
    r = _dsk().window_attn(c.q, K, V, **c.kwargs(**over, **kw))
    torch.cuda.synchronize()
    assert torch.equal(r.out_bf16, want.out_bf16) and torch.equal(r.lse, want.lse)


@pytest.mark.parametrize("bits", [8, 16])
def test_long_prompts_with_steps_in_the_middle_of_their_runs(bits):
    """Runs of many tiles of which all but the ends are seen by every row, from the first token, from a window, and split."""
    for new, lens, kw in ((2100, [0, 700], {}), (700, [3000, 64], dict(window=2500, sinks=40)), (70, [9000], dict(sinks=3))):
        Case(lens, [new] * len(lens), 8, 1, bits=bits, seed=new, nhd=new == 700, **kw).check()


@pytest.mark.parametrize("new", [1, 16, 150])
def test_an_infinity_in_the_middle_of_a_run_stays_when_larger_logits_follow(new):
    """In a tile that every row sees, and in the next one a key that a row weighs far more than all before, yet not so much that the
    infinity's weight falls below 2^-80 of the largest."""
    c = Case([900], [new], 8, 2, bits=16, seed=22, sharp=0.2)    # logits of 12 at most, 34 between two keys
    for kw in ({}, dict(want_f32=False, want_bf16=True)):
        clean = c.run(**kw)
        for row, key in ((100, 140), (300, 333), (511, 512), (896, 897)):
            oldV, oldK = c.V[:, row].clone(), c.K[:, key].clone()
            for h in range(2):
                q = c.q[new // 2, 4 * h + 1].double()            # a logit of 22 for this row
                c.K[h, key] = (22.0 * math.sqrt(D) / (q @ q) * q).bfloat16()
            c.V[:, row, 5], c.V[0, row, 6] = float("inf"), -float("inf")
            r = c.run(**kw)
            out = r.out if r.out is not None else r.out_bf16
            assert bool((out[..., 5] == float("inf")).all()) and bool((out[:, :4, 6] == -float("inf")).all())
            assert bool(torch.isfinite(out[:, 4:, 6]).all()) and bool(torch.isfinite(r.lse).all())
            fine = [i for i in range(D) if i not in (5, 6)]
            assert bool(torch.isfinite(out[..., fine]).all())
            c.V[:, row], c.K[:, key] = oldV, oldK
        again = c.run(**kw)
        assert torch.equal(again.lse, clean.lse)


@pytest.mark.parametrize("byte", [246, 247, 250, 254])
@pytest.mark.parametrize("new, Hq, Hkv", [(1, 4, 4), (3, 8, 2), (8, 8, 2), (16, 8, 2), (30, 8, 2), (70, 8, 2)])
def test_a_row_that_is_not_seen_may_be_too_large_for_its_scale(new, Hq, Hkv, byte):
    """A block whose scale puts the largest codes beyond the finite numbers.  Rows of it that are seen hold zeros; the row that is not
    seen, of a later token or past the window, holds the largest codes."""
    lens, window = 100, ALL
    if new == 1:
        window = 90                                              # positions 0 to 10 are gone, block 0 has 11 to 31 that are seen
    c = Case([lens], [new], Hq, Hkv, window=window, seed=23)
    row = 5 if new == 1 else lens + new - 1
    block = row // 32
    as_bytes(c.vs)[:, block] = byte
    as_bytes(c.V)[:, 32 * block: 32 * block + 32] = 0
    # weights times such scales are out of range themselves where a logit is above the first ones: those of the block are the lowest
    as_bytes(c.K)[:, 32 * block: 32 * block + 32] = 0
    blind = ~c.seen(0)[:, row]
    assert int(blind.sum()) == max(new - 1, 1)
    for kw in ({}, dict(want_f32=False, want_bf16=True)):
        clean = c.run(**kw)
        as_bytes(c.V)[:, row, 5], as_bytes(c.V)[:, row, 6] = 0x7E, 0xFE
        r = c.run(**kw)
        as_bytes(c.V)[:, row] = 0
        a, b = (x.out if x.out is not None else x.out_bf16 for x in (r, clean))
        assert torch.equal(a[blind], b[blind]) and bool(torch.isfinite(a[blind]).all()) and torch.equal(r.lse, clean.lse)
        fine = [i for i in range(D) if i not in (5, 6)]
        assert torch.equal(a[..., fine], b[..., fine])


def _equal_weights(bits, rows, heads):
    """Keys that all weigh the same but for the first one, and values that are all the same: the result is that value, whatever the
    weights, which are no powers of two beside the first one's."""
    g = torch.Generator(device="cuda")
    g.manual_seed(24)
    K = torch.zeros(1, rows, D, device="cuda")
    K[0, 0] = 2.0 ** -5                                          # with queries of ones: a logit of 2^-5 * sqrt(128)
    V = (torch.randint(8, 16, (D,), generator=g, device="cuda") / 16.0).expand(1, rows, D)
    if bits == 16:
        return K.bfloat16().expand(heads, rows, D), V.bfloat16().contiguous().expand(heads, rows, D), {}
    K, V = (x.to(torch.float8_e4m3fn).view(torch.uint8).contiguous().expand(heads, rows, D).view(torch.float8_e4m3fn) for x in (K, V))
    scale = torch.full((heads, -(-rows // 32)), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
    return K, V, dict(k_scale=scale, v_scale=scale, scale_block=32)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("B, heads, new, tokens", [(512, 1, 1, 131071), (1, 512, 1, 131071), (1, 256, 1, 131071), (512, 1, 20, 100000),
                                                   (512, 1, 64, 65472), (512, 1, 128, 32640), (4, 64, 128, 32640), (1, 1, 65536, 0)])
def test_long_runs_of_equal_weights_keep_32_bits(B, heads, new, tokens, bits):
    """A wavefront that adds equal terms one after the other rounds them alike.  Runs that one workgroup takes whole, with one wavefront
    of rows, two and four, and runs in a few long parts.  z0 is the first key's logit, and the sum of its terms' sizes."""
    K, V, kw = _equal_weights(bits, tokens + new, heads)
    q = torch.ones(B * new, heads, D, dtype=torch.bfloat16, device="cuda")
    r = _dsk().window_attn(q, K, V, seq_row0=i32([0] * B), seq_len=i32([tokens] * B), cu_new=i32([new * s for s in range(B + 1)]),
                           max_new=new, max_seqlen=tokens, **kw)
    torch.cuda.synchronize()
    z0 = torch.tensor(2.0 ** -5 * math.sqrt(D), dtype=torch.float64, device="cuda")
    bar, want = float(f32_bar(z0)), V[0, 0].double()
    off = float(((r.out.double() - want).abs() / want).max())
    assert off <= bar, off
    seen = torch.arange(tokens, tokens + new, dtype=torch.float64, device="cuda").repeat(B)[:, None]
    lse = torch.log(torch.exp(z0) + seen)
    assert bool(((r.lse.double() - lse).abs() <= bar + 1e-5 * lse).all())


def test_bf16_results_are_bit_identical_from_call_to_call_on_another_stream_and_in_a_graph():
    kw = dict(want_f32=False, want_bf16=True)
    for bits in (8, 16):
        for new in ([1, 1], [7, 3], [16, 9], [30, 9], [300, 2]):
            c = Case([5000, 700], new, 8, 2, bits=bits, seed=25)
            a, b = c.run(**kw), c.run(**kw)
            st = torch.cuda.Stream()
            r = _dsk().make_window_attn_args(c.q, c.K, c.V, **c.kwargs(**kw))
            torch.cuda.synchronize()
            r.step(st)
            st.synchronize()
            for x in (b, r):
                assert torch.equal(a.out_bf16, x.out_bf16) and torch.equal(a.lse, x.lse)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                r.step(st)
            for _ in range(3):
                r.out_bf16.zero_()
                c.run(**kw)
                graph.replay()
                torch.cuda.synchronize()
                assert torch.equal(a.out_bf16, r.out_bf16) and torch.equal(a.lse, r.lse)


@pytest.mark.parametrize("bits", [8, 16])
def test_a_nan_in_a_query_is_its_rows_alone_in_bf16_results(bits):
    kw = dict(want_f32=False, want_bf16=True)
    for new in (1, 9, 30, 150):
        c = Case([5000, 20], [new, new], 8, 2, bits=bits, seed=26)
        a = c.run(**kw)
        c.q[new // 2, 3, 17] = float("nan")
        b = c.run(**kw)
        assert bool(torch.isnan(b.out_bf16[new // 2, 3]).all()) and bool(torch.isnan(b.lse[new // 2, 3]))
        keep = torch.ones(2 * new, 8, dtype=torch.bool, device="cuda")
        keep[new // 2, 3] = False
        assert torch.equal(a.out_bf16[keep], b.out_bf16[keep]) and torch.equal(a.lse[keep], b.lse[keep])


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("heads, Hkv, new, tokens, kw", [(4, 1, 1, 20000, {}), (8, 2, 8, 36000, dict(window=20011, sinks=40)),
                                                         (4, 1, 16, 9000, dict(sinks=3000, window=5000)), (1, 1, 100, 7000, {})])
def test_long_runs_that_one_workgroup_takes_in_segments(heads, Hkv, new, tokens, kw, bits):
    """So many sequences that none is split, over the same rows.  Results in 32 bits, an infinity of an early segment and a NaN among them."""
    B = 512 // Hkv
    c = Case([tokens] + [0] * (B - 1), [new] * B, heads, Hkv, bits=bits, seed=28, spare=0, sharp=0.2, **kw)
    c.row0 = [0] * B + [c.row0[B]]
    c.lens = [tokens - 7 * s for s in range(B)]
    clean = c.check()
    c.q[3 * new, 0, 17] = float("nan")
    if bits == 16:
        c.V[:, 10, 5] = float("inf")                             # of the first tokens, or of the longest windows
    r = c.run()
    sees = torch.cat([c.seen(s)[:, 10] for s in range(B)])
    keep = torch.ones(B * new, heads, dtype=torch.bool, device="cuda")
    keep[3 * new, 0] = False
    assert bool(torch.isnan(r.out[3 * new, 0]).all()) and bool(torch.isnan(r.lse[3 * new, 0]))
    fine = [i for i in range(D) if i != 5]
    assert torch.equal(r.out[..., fine][keep], clean.out[..., fine][keep]) and torch.equal(r.lse[keep], clean.lse[keep])
    if bits == 16:
        assert torch.equal(r.out[..., 5][keep] == float("inf"), sees[:, None].expand(-1, heads)[keep])
