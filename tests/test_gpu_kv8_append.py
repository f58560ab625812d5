"""dsk_kv8_append against the definition in 64 bits.
Bars: a rotated sum of two fp32 products of terms of size `size`, norm included, is off by a few units of 2^-24 of it: 2^-19 covers
them.  A code then lies within half an e4m3 step of the value.  Values are coded without arithmetic: bit for bit."""
import numpy as np
import pytest
import torch

from step_testutil import i32, rope_reference, starts
from window_testutil import D, E_MIN, as_bytes, e4m3, exponent, half_step, quantise, values

pytestmark = pytest.mark.gpu

OFF = 2.0 ** -19


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


class Case:
    """A batch with a region per sequence, some rows in it already."""

    def __init__(self, lens, new, Hq=4, Hkv=2, *, block=32, rot=128, inter=False, norm=True, far=None, nhd=False, seed=0, spare=5,
                 loud=1.0, queries=True):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.lens, self.new, self.Hq, self.Hkv, self.block, self.inter = lens, new, Hq, Hkv, block, inter
        self.row0 = starts([-(-(a + b + spare) // block) * block for a, b in zip(lens, new)])
        self.rows, self.cu = self.row0[-1] - 3, starts(new)      # the last block is cut off
        self.N = self.cu[-1] + 2                                 # rows behind the last sequence

        def cache():
            X = torch.randn(Hkv, self.rows, D, generator=g, device="cuda")
            X[..., 5::37] *= 8.0
            codes, scale = quantise(X.bfloat16(), block)
            if nhd:
                wide = torch.zeros(self.rows, Hkv, D + 16, dtype=torch.uint8, device="cuda")
                view = wide[..., :D].transpose(0, 1)
                view.copy_(as_bytes(codes))
                codes = view.view(torch.float8_e4m3fn)
            return codes, scale
        self.K, self.ks = cache()
        self.V, self.vs = cache()
        x = torch.randn(self.N, Hq + 2 * Hkv, D, generator=g, device="cuda")
        x = (x * torch.exp(loud * torch.randn(self.N, Hq + 2 * Hkv, 1, generator=g, device="cuda"))).bfloat16()
        self.q, self.k, self.v = x[:, :Hq], x[:, Hq: Hq + Hkv], x[:, Hq + Hkv:]
        self.queries = queries
        self.inv_freq = (1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda() if rot else None
        self.wq = self.wk = None
        if norm:
            self.wq, self.wk = (1.0 + 0.3 * torch.randn(D, generator=g, device="cuda") for _ in range(2))
        self.pos = None
        if far is not None:
            self.pos = torch.randint(0, far, (self.N,), generator=g, device="cuda", dtype=torch.int32)

    def handle(self, **over):
        kw = dict(scale_block=self.block, seq_row0=i32(self.row0[:-1]), seq_len=i32(self.lens), cu_new=i32(self.cu),
                  max_new=max(max(self.new), 1), pos=self.pos, q_weight=self.wq, k_weight=self.wk, eps=1e-5, inv_freq=self.inv_freq,
                  interleaved=self.inter)
        if self.queries:
            kw.update(q=self.q, q_out=torch.full((self.N, self.Hq, D), 9.0, dtype=torch.bfloat16, device="cuda"))
        kw.update(over)
        return _dsk().make_kv8_appender(self.k, self.v, self.K, self.V, self.ks, self.vs, **kw)

    def snapshot(self):
        return [as_bytes(t).clone() for t in (self.K, self.ks, self.V, self.vs)]

    def check(self, status=0):
        before = self.snapshot()
        h = self.handle()
        h.step()
        torch.cuda.synchronize()
        assert int(h.dev_status) == status
        after = [x.cpu() for x in self.snapshot()]
        before = [x.cpu() for x in before]
        pos = torch.cat([torch.arange(L, L + n) for L, n in zip(self.lens, self.new)] + [torch.zeros(2, dtype=torch.long)])
        pos = pos if self.pos is None else self.pos
        k, k_size = rope_reference(self.k, self.wk, 1e-5, pos, self.inv_freq, self.inter)
        for X, size, (b, bs, a, as_) in ((k, k_size, (*before[:2], *after[:2])),
                                         (self.v.double().cpu(), None, (*before[2:], *after[2:]))):
            self.check_rows(X, size, b, bs, a, as_)
        if self.queries:
            q, size = rope_reference(self.q, self.wq, 1e-5, pos, self.inv_freq, self.inter)
            n = self.cu[-1]
            out = h.q_out.double().cpu()
            assert bool(((out - q)[:n].abs() <= 2.0 ** -8 * q[:n].abs() + OFF * size[:n]).all())
            assert bool((out[n:] == 9.0).all())
        return h

    def check_rows(self, x, size, codes0, scale0, codes, scale):
        """x [tokens, Hkv, D] 64 bits; size: of the sums' terms, None: nothing was computed."""
        S = self.block
        want_c, want_s = codes0.clone(), scale0.clone()
        for s, (L, n) in enumerate(zip(self.lens, self.new)):
            begin, end = self.row0[s] + L, self.row0[s] + L + n
            for blk in range(begin // S, -(-end // S) if n else begin // S):
                lo, hi = max(begin, blk * S), min(end, blk * S + S)
                t = slice(self.cu[s] + lo - begin, self.cu[s] + hi - begin)
                for h in range(self.Hkv):
                    y, e = x[t, h], int(scale[h, blk]) - 127
                    old = int(scale0[h, blk]) - 127
                    begun = lo > blk * S
                    need = exponent(y)
                    if size is None:
                        assert e == (max(need, old) if begun else need)
                    else:                                        # the largest value may lie on either side of a border
                        near = {exponent(y * f) for f in (1 - 2 * OFF, 1.0, 1 + 2 * OFF)}
                        assert e in ({max(v, old) for v in near} if begun else near)
                    got = codes[h, lo:hi].view(torch.float8_e4m3fn).double()
                    if size is None:
                        want_c[h, lo:hi] = e4m3(y * 2.0 ** -e).to(torch.float8_e4m3fn).view(torch.uint8)
                        assert torch.equal(got, want_c[h, lo:hi].view(torch.float8_e4m3fn).double())
                    else:
                        z = y * 2.0 ** -e
                        assert bool(((got - z).abs() <= half_step(z) * (1 + 1e-9) + OFF * size[t, h] * 2.0 ** -e).all())
                    want_c[h, lo:hi] = codes[h, lo:hi]
                    want_s[h, blk] = scale[h, blk]
                    if begun and e > old:                        # rows of the block that were there
                        o = codes0[h, blk * S: lo].view(torch.float8_e4m3fn).double() * 2.0 ** (old - e)
                        want_c[h, blk * S: lo] = e4m3(o).to(torch.float8_e4m3fn).view(torch.uint8)
        same = (want_c == codes) | ((want_c | codes) == 0x80)    # 0 and -0
        assert bool(same.all()) and torch.equal(want_s, scale)


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("new", [1, 2, 31, 64, 129])
def test_blocks_and_numbers_of_tokens(block, new):
    lens = [0, 1, 31, 32, 63, 100, 127, 128, 200]
    Case(lens, [max(0, new - s % 3) for s in range(len(lens))], block=block, seed=new).check()


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (5, 1), (8, 8), (9, 3), (33, 11), (40, 8)])
def test_heads(Hq, Hkv):
    Case([7, 40], [35, 3], Hq, Hkv, seed=Hq).check()
    Case([70], [1], Hq, Hkv, seed=Hq, queries=False, block=128, nhd=True).check()


@pytest.mark.parametrize("rot", [0, 16, 32, 96, 128])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rotations_and_norms(rot, inter, norm):
    Case([3, 0], [40, 33], rot=rot, inter=inter, norm=norm, far=131072, seed=rot, nhd=inter).check()


def test_scales_that_grow_keep_or_start_again():
    """Rows after rows into the same blocks, some a thousand times as large as those before."""
    for block in (32, 128):
        c = Case([0, 10], [1, 3], block=block, seed=3, loud=3.0, spare=200)
        grown = 0
        for _ in range(40):
            before = c.snapshot()
            c.check()
            grown += int((as_bytes(c.vs) > before[3]).sum())
            c.lens = [L + n for L, n in zip(c.lens, c.new)]
            c.k, c.v, c.q = (t.roll(1, 0) * 1.5 for t in (c.k, c.v, c.q))
        assert grown > 10
        c.lens = [0, 10]                                         # a sequence that begins again: its first block forgets its scale
        c.check()


def test_appending_again_changes_nothing():
    c = Case([5, 50], [70, 9], seed=4)
    c.check()
    before = c.snapshot()
    c.handle().step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, c.snapshot()))


def test_values_that_are_not_finite_become_nan_and_do_not_count():
    c = Case([4], [20], Hq=2, Hkv=2, rot=0, norm=False, seed=5)
    x = torch.cat([c.q, c.k, c.v], 1)
    x[3, 2:, 7], x[5, 2:, 9], x[6, 2:, 100] = float("inf"), -float("inf"), float("nan")
    x[9, 2:] = 0.0
    c.q, c.k, c.v = x[:, :2], x[:, 2:4], x[:, 4:]
    c.handle().step()
    for X, scale, src in ((c.K, c.ks, c.k), (c.V, c.vs, c.v)):
        got = values(X, scale, c.block)[:, 4:24].transpose(0, 1)
        fine = torch.isfinite(src[:20].double())
        assert torch.equal(torch.isnan(got), ~fine)
        bound = 2.0 ** -4 * src[:20].double().abs() + 2.0 ** -10 * values(torch.ones_like(X), scale, c.block)[:, 4:24].transpose(0, 1).abs()
        assert bool(((got - src[:20].double()).abs() <= bound)[fine].all())


def test_nothing_but_zeros_and_the_ends_of_the_range():
    c = Case([0], [64], Hq=2, Hkv=2, rot=0, norm=False, seed=6)
    x = torch.cat([c.q, c.k, c.v], 1)
    x[:32, 2:] = 0.0
    x[32:64, 2:] *= 2.0 ** -115
    c.q, c.k, c.v = x[:, :2], x[:, 2:4], x[:, 4:]
    c.check()
    assert bool((as_bytes(c.vs)[:, 0] == E_MIN + 127).all())
    x[:64, 2:] = torch.where(x[:64, 2:] > 0, 448.0 * 2.0 ** 100, 448.0 * 2.0 ** 100 * (1 + 2.0 ** -7)).bfloat16()
    x[:32, 2:] = 448.0 * 2.0 ** 100                              # exactly the largest code; the next bf16 number takes the next scale
    c.k, c.v = x[:, 2:4], x[:, 4:]
    c.check()
    assert bool((as_bytes(c.vs)[:, 0] == 227).all()) and bool((as_bytes(c.vs)[:, 1] == 228).all())


def test_queries_in_place_and_positions_far_away():
    c = Case([9, 33], [6, 40], far=2 ** 31 - 1, seed=7)
    want = c.check().q_out
    q = c.q.contiguous()
    h = c.handle(q=q, q_out=q)
    h.step()
    torch.cuda.synchronize()
    n = c.cu[-1]
    assert torch.equal(q[:n], want[:n]) and torch.equal(q[n:], c.q[n:])


def test_malformed_tables():
    dsk = _dsk()

    def run(status, touched, **over):
        c = Case([40, 40], [10, 10], seed=8)
        before = c.snapshot()
        h = c.handle(**over)
        h.step()
        torch.cuda.synchronize()
        assert int(h.dev_status) == status
        for b, a in zip(before, c.snapshot()):
            if b.shape[1] < 20:
                continue
            rows = (b != a).flatten(2).any(2).any(0).nonzero()[:, 0].tolist()
            assert set(rows) <= set(touched), (over, rows)
        written = (h.q_out != 9.0).flatten(1).any(1)
        return written.tolist(), c
    c = Case([40, 40], [10, 10], seed=8)
    first, second = (list(range(c.row0[s] + 32, c.row0[s] + 50)) for s in range(2))
    w, _ = run(dsk.DSK_ERR_ALIGN, second, seq_row0=i32([16, c.row0[1]]))
    assert w == [False] * 10 + [True] * 10 + [False] * 2
    w, _ = run(dsk.DSK_ERR_SHAPE, second, seq_row0=i32([-32, c.row0[1]]))
    assert w == [False] * 10 + [True] * 10 + [False] * 2
    w, _ = run(dsk.DSK_ERR_SHAPE, first, seq_len=i32([40, -1]))
    assert w == [True] * 10 + [False] * 12
    w, _ = run(dsk.DSK_ERR_SHAPE, first + second, max_new=5)
    assert w == ([True] * 5 + [False] * 5) * 2 + [False] * 2
    w, _ = run(dsk.DSK_ERR_SHAPE, first, cu_new=i32([0, 10, 3]))
    assert w == [True] * 10 + [False] * 12
    w, _ = run(dsk.DSK_ERR_SHAPE, first + second + list(range(c.row0[1] + 50, c.row0[1] + 52)), cu_new=i32([0, 10, 400]), max_new=500)
    assert w == [True] * 22
    w, _ = run(dsk.DSK_ERR_CAPACITY, first + list(range(c.rows - 5, c.rows)), seq_len=i32([40, c.rows - 5 - c.row0[1]]))
    assert w == [True] * 15 + [False] * 7
    w, _ = run(dsk.DSK_ERR_CAPACITY, first, seq_len=i32([40, 2 ** 31 - 1]))
    assert w == [True] * 10 + [False] * 12


def test_long_prompts_and_many_sequences():
    Case([0], [5000], 8, 2, seed=9).check()
    rng = np.random.default_rng(10)
    lens, new = [int(x) for x in rng.integers(0, 90, 60)], [int(x) for x in rng.integers(0, 70, 60)]
    for block in (32, 64, 128):
        Case(lens, new, 4, 2, seed=11, block=block).check()


def test_large_cache_offsets():
    """Rows whose bytes lie beyond 2^32 of a head's first."""
    dsk, rows = _dsk(), (1 << 32) // (2 * D) + 64
    X = torch.zeros(rows, 2, D, dtype=torch.uint8, device="cuda")
    K, V = (X[:, h:h + 1].transpose(0, 1).view(torch.float8_e4m3fn) for h in range(2))
    assert K.stride(1) * rows > 1 << 32
    ks, vs = (torch.full((1, -(-rows // 32)), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2))
    k = torch.randn(40, 1, D, device="cuda").bfloat16()
    row0 = (rows - 64) // 32 * 32
    h = dsk.make_kv8_appender(k, k, K, V, ks, vs, scale_block=32, seq_row0=i32([row0]), seq_len=i32([0]), cu_new=i32([0, 40]),
                              max_new=40)
    h.step()
    torch.cuda.synchronize()
    assert int(h.dev_status) == 0
    codes, scale = quantise(k.transpose(0, 1), 32)
    for X8, s8 in ((K, ks), (V, vs)):
        assert torch.equal(as_bytes(X8)[:, row0: row0 + 40].contiguous(), as_bytes(codes))
        assert torch.equal(as_bytes(s8)[:, row0 // 32: row0 // 32 + 2], as_bytes(scale))
    assert int(as_bytes(K)[:, :row0].max()) == 0


def test_captured_and_on_another_stream():
    c = Case([5, 50], [4, 1], seed=12)
    h = c.handle()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    start = c.snapshot()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        h.step(stream)
    assert all(torch.equal(a, b) for a, b in zip(start, c.snapshot()))
    seq_len = h.keep[7]
    for step in range(4):
        eager = Case([5, 50], [4, 1], seed=12)
        for t, b in zip((eager.K, eager.ks, eager.V, eager.vs), start):
            as_bytes(t).copy_(b)
        eager.lens = [5 + 4 * step, 50 + step]
        eager.handle().step()
        seq_len.copy_(i32(eager.lens))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        start = c.snapshot()
        assert all(torch.equal(a, b) for a, b in zip(start, eager.snapshot()))


def test_a_bound_beyond_all_tokens_changes_nothing():
    a, b = Case([5, 50, 0], [4, 1, 70], seed=21), Case([5, 50, 0], [4, 1, 70], seed=21)
    ha, hb = a.handle(), b.handle(max_new=0x7FFFFFFF)
    for h in (ha, hb):
        h.step()
    torch.cuda.synchronize()
    assert int(hb.dev_status) == 0 and torch.equal(ha.q_out, hb.q_out)
    assert all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot()))


def test_the_largest_numbers_stay_finite():
    """What lies above the largest code that is finite with the scale 2^120, 240 * 2^120, becomes that: within 2^-4 of it."""
    for block in (32, 128):
        c = Case([0, 3], [20, 20], Hq=2, Hkv=2, rot=0, norm=False, seed=27, block=block)
        x = torch.cat([c.q, c.k, c.v], 1)
        big = torch.finfo(torch.bfloat16).max
        numbers = torch.tensor([big, -big, 1.9375 * 2.0 ** 127, 1.921875 * 2.0 ** 127, 1.875 * 2.0 ** 127, -1.75 * 2.0 ** 127, 2.0 ** 127,
                                float("inf"), float("nan")])
        x[:, 2:, :9] = numbers.bfloat16().cuda()
        x[:, 2:, 9:] = 0.0
        c.q, c.k, c.v = x[:, :2], x[:, 2:4], x[:, 4:]
        as_bytes(c.ks)[:, c.row0[1] // block], as_bytes(c.vs)[:, c.row0[1] // block] = 100, 253   # begun: smaller, or from elsewhere
        c.handle().step()
        torch.cuda.synchronize()
        assert int(as_bytes(c.vs)[0, 0]) == 247 and int(as_bytes(c.vs)[0, c.row0[1] // block]) == 253
        for X, scale, src in ((c.K, c.ks, c.k), (c.V, c.vs, c.v)):
            got = values(X, scale, block)
            for s in range(2):
                rows = slice(c.row0[s] + c.lens[s], c.row0[s] + c.lens[s] + 20)
                y, want = got[:, rows, :7], src[20 * s: 20 * s + 20, :, :7].transpose(0, 1).double()
                assert bool((y.abs() <= 240.0 * 2.0 ** 120).all()) and bool(torch.isfinite(y.float().bfloat16()).all())
                assert bool(((y - want).abs() <= 2.0 ** -4 * want.abs()).all())
                assert bool(torch.isnan(got[:, rows, 7:9]).all()) and bool((got[:, rows, 9:] == 0.0).all())
