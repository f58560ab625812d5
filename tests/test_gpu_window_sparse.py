"""dsk_window_sparse_decode_attn against the definition in 64 bits, on the numbers that the cache stands for; bars as for
dsk_window_attn."""
import math

import numpy as np
import pytest
import torch

from step_testutil import i32
from test_gpu_window_attn import BF16, Case as WindowCase
from window_testutil import D, TINY, as_bytes, attend, f32_bar

pytestmark = pytest.mark.gpu


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


class Case(WindowCase):
    """One query per sequence; `lens` count its own token.  A selection per list: any slots of 1..b tokens, in order."""

    def __init__(self, lens, Hq, Hkv, k, b, *, shared=False, window=0, empty=(), **kw):
        super().__init__(lens, [0] * len(lens), Hq, Hkv, pad=len(lens), window=window, **kw)
        rng = np.random.default_rng(kw.get("seed", 0))
        self.k, self.b, self.shared = k, b, shared
        H = Hkv if shared else Hq
        start = np.zeros((len(lens), H, k), dtype=np.int32)
        length, count = np.zeros_like(start), np.zeros(start.shape[:2], dtype=np.int32)
        for s, L in enumerate(lens):
            for h in range(H):
                slots = -(-L // b)
                n = min(k, slots) if (s, h) not in empty else 0
                pick = np.sort(rng.permutation(slots)[:n])
                start[s, h, :n] = self.row0[s] + pick * b
                length[s, h, :n] = np.minimum(rng.integers(1, b + 1, n), L - pick * b)
                count[s, h] = n
        self.sel = [start, length, count]

    def kwargs(self, **over):
        kw = super().kwargs()
        for name in ("cu_new", "max_new"):
            kw.pop(name)
        kw.update(zip(("sel_start", "sel_len", "sel_count"), (torch.from_numpy(x).cuda() for x in self.sel)), b=self.b)
        kw.update(over)
        return kw

    def run(self, **over):
        r = _dsk().make_window_sparse_args(self.q, self.K, self.V, **self.kwargs(**over))
        for t in (r.out, r.out_bf16, r.lse):
            if t is not None:
                t.fill_(9.0)
        r.step()
        torch.cuda.synchronize()
        return r

    def seen_rows(self, s, h):
        """Cache rows that query head h of sequence s sees, as often as it sees them."""
        G, L, r0 = self.Hq // self.Hkv, self.lens[s], self.row0[s]
        lo = max(0, L - self.window)
        few = min(self.sinks, lo)
        near = list(range(r0, r0 + few)) + list(range(r0 + lo, r0 + L))
        start, length, count = (x[s, h // G if self.shared else h].tolist() for x in self.sel)
        far = [r for a, n in zip(start[:count], length[:count]) for r in range(a, a + n) if r0 + few <= r < r0 + lo]
        return torch.tensor(near + far, dtype=torch.long, device="cuda")

    def reference(self, scale=None):
        G, B = self.Hq // self.Hkv, len(self.lens)
        K, V = self.numbers()
        out, size = (torch.zeros(B, self.Hq, D, dtype=torch.float64, device="cuda") for _ in range(2))
        lse, bar = (torch.zeros(B, self.Hq, dtype=torch.float64, device="cuda") for _ in range(2))
        for s in range(B):
            for h in range(self.Hq):
                rows = self.seen_rows(s, h)
                seen = torch.ones(1, len(rows), dtype=torch.bool, device="cuda")
                o, z, l, terms = attend(self.q[s, h: h + 1], K[h // G, rows], V[h // G, rows], seen, scale)
                out[s, h], size[s, h], lse[s, h], bar[s, h] = o[0], z[0], l[0], f32_bar(terms)[0]
        return out, size, lse, bar

    def check(self, scale=None, want=None):
        out, size, lse, bar = self.reference(scale) if want is None else want
        sc = 0.0 if scale is None else scale
        a = self.run(scale=sc)
        b = self.run(scale=sc, want_f32=False, want_bf16=True)
        c = self.run(scale=sc, want_bf16=True)
        assert bool(((a.out.double() - out).abs() <= bar[..., None] * size + TINY).all())
        assert bool(((b.out_bf16.double() - out).abs() <= BF16 * (1 + BF16) * out.abs() + (2.0 ** -15 + bar[..., None]) * size + TINY).all())
        assert torch.equal(c.out, a.out) and torch.equal(c.out_bf16, a.out.bfloat16())
        fine = torch.isfinite(lse)
        for r in (a, b, c):
            got = r.lse.double()
            assert torch.equal(got[~fine], lse[~fine])
            assert bool(((got - lse)[fine].abs() <= bar[fine] + 1e-5 * lse[fine].abs()).all())
        return a


LENS = [0, 1, 33, 500, 1500]


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("window, sinks", [(0, 0), (0, 5), (1, 0), (40, 4), (600, 33), (2000, 4)])
@pytest.mark.parametrize("b, k", [(1, 40), (8, 5), (16, 40), (32, 17), (64, 3), (1000, 2)])
def test_slots_windows_and_first_tokens(b, k, window, sinks, shared, bits):
    Case(LENS, 8, 2, k, b, shared=shared, window=window, sinks=sinks, bits=bits, seed=b + k, empty=((3, 0), (4, 1)),
         block=(32, 64, 128)[k % 3], nhd=b == 16).check()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (4, 4), (5, 1), (12, 4), (40, 1), (72, 2)])
def test_group_widths(Hq, Hkv, bits):
    for shared in (False, True):
        Case([300, 41], Hq, Hkv, 9, 16, shared=shared, window=50, sinks=3, bits=bits, seed=Hq).check()


@pytest.mark.parametrize("bits", [8, 16])
def test_long_lists_and_windows(bits):
    Case([30000, 7], 8, 2, 700, 16, shared=True, window=3000, sinks=100, bits=bits, seed=1).check()
    Case([20000, 19999, 1], 4, 2, 3000, 4, window=70, sinks=0, bits=bits, seed=2).check()
    Case([9000], 2, 1, 4, 1000, window=9000, sinks=0, bits=bits, seed=3).check()
    Case([40000] * 40, 1, 1, 20, 32, window=5000, sinks=64, bits=bits, seed=4).check()


def test_everything_selected_or_near_is_the_attention_over_all():
    dsk = _dsk()
    for bits in (8, 16):
        c = Case([777, 64], 8, 2, 100, 16, window=100, sinks=10, bits=bits, seed=5, empty=())
        c.sel[1][:] = 0
        for s, L in enumerate(c.lens):
            n = -(-L // 16)
            c.sel[0][s, :, :n] = c.row0[s] + 16 * np.arange(n)
            c.sel[1][s, :, :n] = np.minimum(16, L - 16 * np.arange(n))
            c.sel[2][s] = n
        _, size, lse, bar = want = c.reference()
        r = c.check(want=want)
        w = dsk.window_attn(c.q, c.K, c.V, seq_row0=i32(c.row0[:-1]), seq_len=i32([L - 1 for L in c.lens]), cu_new=i32([0, 1, 2]),
                            max_new=1, max_seqlen=776, k_scale=c.ks, v_scale=c.vs, scale_block=c.block)
        torch.cuda.synchronize()                                 # either is off by as much from the definition
        assert bool(((r.out - w.out).double().abs() <= 2 * bar[..., None] * size + TINY).all())
        assert bool(((r.lse - w.lse).double().abs() <= 2 * (bar + 1e-5 * lse.abs())).all())


def test_without_what_is_near_it_is_the_sparse_attention():
    dsk = _dsk()
    for shared in (False, True):
        c = Case([4000, 300], 8, 2, 30, 32, bits=16, seed=6, shared=shared)
        r = c.run()
        sel = [torch.from_numpy(x).cuda() for x in c.sel]
        s = dsk.make_attn_args(c.q, c.K, c.V, *sel, 32, flags=dsk.DSK_ATTN_SHARED_SELECTION if shared else 0)
        dsk.dsk_sparse_decode_attn(s.args)
        torch.cuda.synchronize()
        _, size, lse, bar = c.reference()                        # either is off by as much from the definition
        assert bool(((r.out - s.out).double().abs() <= 2 * bar[..., None] * size + TINY).all())
        assert bool(((r.lse - s.lse).double().abs() <= 2 * (bar + 1e-5 * lse.abs())).all())


def test_spans_outside_the_sequence_hold_nothing_and_repeated_ones_count_again():
    c = Case([200, 100], 4, 2, 6, 16, seed=4, window=20, sinks=2)
    start, length, count = c.sel
    room = [np.concatenate([x, x], axis=2) for x in (start, length)]
    n = start.shape[2]
    for s in range(2):
        for h in range(4):
            c0 = count[s, h]
            room[0][s, h, c0:c0 + 6] = [-3, c.rows - 2, 5, 2 ** 31 - 1, c.row0[s] + 50, c.row0[s] + 50]
            room[1][s, h, c0:c0 + 6] = [4, 7, -1, 9, 300, 300]   # the last two are cut to b = 16 tokens
            count[s, h] = c0 + 6
    room[1] = np.minimum(room[1], 16)
    c.sel = [room[0], room[1], count]
    assert count.max() <= 2 * n
    want = c.reference()
    c.sel[1] = np.where(room[1] == 16, 300, room[1])             # longer than b: cut
    c.check(want=want)
    c.sel[2] = np.where(count > 0, count, 0)
    r = c.run(sel_count=torch.full((2, 4), -7, dtype=torch.int32, device="cuda"))
    c.sel[2][:] = 0
    c.check()
    assert torch.equal(c.run().out, r.out)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_rows_that_are_not_seen_may_hold_anything(what, bits):
    c = Case([900, 130], 8, 2, 9, 16, window=50, sinks=3, bits=bits, seed=8)
    clean, bf16 = c.run(), c.run(want_f32=False, want_bf16=True)
    for h in range(2):
        seen = torch.zeros(c.rows, dtype=torch.bool, device="cuda")
        for s in range(2):
            for g in range(4):
                seen[c.seen_rows(s, 4 * h + g)] = True
        for X in (c.K, c.V):
            if bits == 16:
                X[h, ~seen] = what
            else:
                as_bytes(X)[h, ~seen] = 0x7F
    r, rb = c.run(), c.run(want_f32=False, want_bf16=True)
    assert torch.equal(r.out, clean.out) and torch.equal(r.lse, clean.lse) and torch.equal(rb.out_bf16, bf16.out_bf16)
    if bits == 16:                                               # and an infinity that is seen gives that infinity
        c.V[0, c.row0[0] + 899, 5] = float("inf")
        r = c.run()
        assert bool((r.out[0, :4, 5] == float("inf")).all()) and bool(torch.isfinite(r.out[1]).all())
        assert bool(torch.isfinite(r.out[0, :, :5]).all()) and bool(torch.isfinite(r.out[0, 4:]).all())


def test_malformed_tables_are_cut():
    c = Case([64, 640], 4, 2, 6, 16, window=20, sinks=3, seed=9)
    base = c.run()
    for kw in (dict(seq_row0=i32([-5, c.row0[1]])), dict(seq_len=i32([-5, 640])), dict(seq_row0=i32([2 ** 31 - 1, c.row0[1]])),
               dict(seq_row0=i32([c.rows, c.row0[1]]))):
        r = c.run(**kw)
        assert torch.equal(r.out[1], base.out[1]) and bool((r.out[0] == 0.0).all()) and bool((r.lse[0] == -math.inf).all())
    r = c.run(seq_len=i32([64, 2 ** 31 - 1]))                    # cut to max_seqlen
    assert torch.equal(r.out, base.out)
    r = c.run(max_seqlen=64)
    assert torch.equal(r.out[0], base.out[0]) and bool(torch.isfinite(r.out).all())


def test_bit_identical_from_call_to_call_on_another_stream_and_in_a_graph():
    for bits in (8, 16):
        c = Case([5000, 700], 8, 2, 60, 32, window=500, sinks=9, bits=bits, seed=10)
        a = c.run()
        st = torch.cuda.Stream()
        r = _dsk().make_window_sparse_args(c.q, c.K, c.V, **c.kwargs())
        torch.cuda.synchronize()
        r.step(st)
        st.synchronize()
        assert torch.equal(a.out, r.out) and torch.equal(a.lse, r.lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            r.step(st)
        for _ in range(3):
            r.out.zero_()
            c.run()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(a.out, r.out) and torch.equal(a.lse, r.lse)


def test_a_workspace_for_the_longest_cache_serves_shorter_ones():
    c = Case([900, 100], 8, 2, 9, 16, window=400, sinks=4, seed=11)
    r = _dsk().make_window_sparse_args(c.q, c.K, c.V, **c.kwargs(max_seqlen=120_000))
    out, size, _, bar = c.reference()
    for most in (120_000, 4000, 900):
        r.args.max_seqlen = most
        r.out.fill_(9.0)
        r.step()
        torch.cuda.synchronize()
        assert bool(((r.out.double() - out).abs() <= bar[..., None] * size + TINY).all())


def test_a_count_far_below_zero_selects_nothing():
    for bits in (8, 16):
        c = Case([5000, 700], 8, 2, 60, 32, window=50, sinks=3, bits=bits, seed=12)
        for count in (-1, -60, -2 ** 31):
            r = c.run(sel_count=torch.full((2, 8), count, dtype=torch.int32, device="cuda"))
            none = c.run(sel_count=torch.zeros(2, 8, dtype=torch.int32, device="cuda"))
            assert torch.equal(r.out, none.out) and torch.equal(r.lse, none.lse)
