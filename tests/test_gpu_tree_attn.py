"""dsk_tree_decode_attn against the definition in 64 bits.
Bars, with size = sum p |V| / sum p: fp32 logits (128 exact products summed), exponentials and sums are off by some units of 2^-24
of terms whose largest is about 2^5: 1e-5 of the size covers them.  bf16 outputs: the weights are rounded to bf16 for the products
with V, half a step 2^-8 of each and so of the size, the result once more, 2^-8 of it."""
import math

import numpy as np
import pytest
import torch

from step_testutil import D, ancestors, i32, pack_mask, random_parents, starts, tree_reference

pytestmark = pytest.mark.gpu

F32, BF16 = 1e-5, 2.0 ** -8


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


class Case:
    """A batch with a region per sequence, K and V with outlier channels, and its reference."""

    def __init__(self, lens, n_new, Hq, Hkv, *, packed=False, nhd=False, seed=0, masks="tree", spare=3, pad_tokens=0, sharp=1.0):
        self.rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.lens, self.n_new, self.Hq, self.Hkv, self.packed = lens, n_new, Hq, Hkv, packed
        self.row0 = starts([a + b + spare for a, b in zip(lens, n_new)])
        self.cu, self.rows = starts(n_new), self.row0[-1]
        self.N = self.cu[-1] + pad_tokens

        def rows(n):
            if nhd:
                X = torch.randn(max(n, 1), Hkv, D + 24, generator=g, device="cuda").bfloat16()[..., :D].transpose(0, 1)
            else:
                X = torch.randn(Hkv, max(n, 1), D, generator=g, device="cuda").bfloat16()
            X[..., 7::31] *= 4.0
            return X
        self.K, self.V = rows(self.rows), rows(self.rows)
        self.Kd, self.Vd = (rows(self.N), rows(self.N)) if packed else (None, None)
        self.q = (torch.randn(max(self.N, 1), Hq, D, generator=g, device="cuda") * sharp).bfloat16()[: self.N]
        self.words = (max(max(n_new), 1) + 31) // 32
        self.seen = []
        for n in n_new:
            if masks == "tree":
                self.seen.append(ancestors(random_parents(self.rng, n))[0])
            elif masks == "chain":
                self.seen.append(np.tril(np.ones((n, n), dtype=bool)))
            else:                                                # any bits at all, some rows empty, also of later nodes
                m = self.rng.random((n, n)) < self.rng.choice([0.0, 0.1, 0.9], (n, 1))
                self.seen.append(m)
        self.masks = masks
        self.sel = None

    def select(self, k, b, empty=()):
        """A selection per KV head: any slots of 1..b tokens, in order, the counts of `empty` (sequence, head) 0."""
        start = np.zeros((len(self.lens), self.Hkv, k), dtype=np.int32)
        length, count = np.zeros_like(start), np.zeros(start.shape[:2], dtype=np.int32)
        for s, L in enumerate(self.lens):
            for h in range(self.Hkv):
                slots = -(-L // b)
                n = min(k, slots) if (s, h) not in empty else 0
                pick = np.sort(self.rng.permutation(slots)[:n])
                start[s, h, :n] = self.row0[s] + pick * b
                length[s, h, :n] = np.minimum(self.rng.integers(1, b + 1, n), L - pick * b)
                count[s, h] = n
        self.sel, self.b = (start, length, count), b
        return self

    def kwargs(self, **over):
        kw = dict(seq_row0=i32(self.row0[:-1]), seq_len=i32(self.lens), cu_new=i32(self.cu), max_nodes=max(max(self.n_new), 1),
                  max_seqlen=max(self.lens), Kd=self.Kd, Vd=self.Vd, mask=None)
        if self.masks != "chain":
            m = pack_mask(self.seen, self.words)
            kw["mask"] = torch.cat([m, torch.zeros(self.N - len(m), self.words, dtype=torch.int32)]).cuda()
        if self.sel is not None:
            kw.update(zip(("sel_start", "sel_len", "sel_count"), (torch.from_numpy(x).cuda() for x in self.sel)), b=self.b)
        kw.update(over)
        return kw

    def run(self, **over):
        r = _dsk().make_tree_attn_args(self.q, self.K, self.V, **self.kwargs(**over))
        for t in (r.out, r.out_bf16, r.lse):
            if t is not None:
                t.fill_(9.0)
        _dsk().dsk_tree_decode_attn(r.args)
        torch.cuda.synchronize()
        return r

    def prefix(self, s, h):
        if self.sel is None:
            return torch.arange(self.row0[s], self.row0[s] + self.lens[s], device="cuda")
        start, length, count = (x[s, h] for x in self.sel)
        spans = [torch.arange(a, a + n, device="cuda") for a, n in zip(start[:count], length[:count])]
        return torch.cat(spans) if spans else torch.arange(0, device="cuda")

    def reference(self, scale=None):
        G = self.Hq // self.Hkv
        scale = 1.0 / math.sqrt(D) if scale is None else scale
        out, size = (torch.zeros(self.cu[-1], self.Hq, D, dtype=torch.float64, device="cuda") for _ in range(2))
        lse = torch.zeros(self.cu[-1], self.Hq, dtype=torch.float64, device="cuda")
        for s, n in enumerate(self.n_new):
            t = slice(self.cu[s], self.cu[s + 1])
            for h in range(self.Hkv):
                p, hs = self.prefix(s, h), slice(h * G, (h + 1) * G)
                nodes = slice(self.row0[s] + self.lens[s], self.row0[s] + self.lens[s] + n)
                Kn, Vn = (self.Kd[h, t], self.Vd[h, t]) if self.packed else (self.K[h, nodes], self.V[h, nodes])
                out[t, hs], size[t, hs], lse[t, hs] = tree_reference(self.q[t, hs], self.K[h][p], self.V[h][p], Kn, Vn,
                                                                     self.seen[s], scale)
        return out, size, lse

    def check(self, scale=None, want=None):
        out, size, lse = self.reference(scale) if want is None else want
        n = self.cu[-1]
        sc = 0.0 if scale is None else scale
        a = self.run(scale=sc)
        b = self.run(scale=sc, want_f32=False, want_bf16=True)
        c = self.run(scale=sc, want_bf16=True)
        assert bool(((a.out[:n].double() - out).abs() <= F32 * size).all())
        assert bool(((b.out_bf16[:n].double() - out).abs() <= BF16 * (out.abs() * (1 + BF16) + size) + F32 * size).all())
        assert torch.equal(c.out[:n], a.out[:n]) and torch.equal(c.out_bf16[:n], a.out[:n].bfloat16())
        fine = torch.isfinite(lse)
        for r in (a, b, c):
            got = r.lse[:n].double()
            assert torch.equal(got[~fine], lse[~fine])
            assert bool(((got - lse)[fine].abs() <= 1e-5 * (1 + lse[fine].abs())).all())
            for t in (r.out, r.out_bf16, r.lse):                 # rows behind the last sequence stay as they were
                assert t is None or bool((t[n:] == 9.0).all())


LENS = [0, 1, 31, 32, 33, 64, 127, 129, 700, 1025]


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (8, 8), (8, 2), (6, 2), (5, 1), (16, 2), (14, 2)])
@pytest.mark.parametrize("nodes", [1, 2, 7, 16, 33])
def test_group_widths_tree_sizes_and_ragged_lengths(Hq, Hkv, nodes):
    n_new = [max(0, nodes - (s % 3)) for s in range(len(LENS))]
    Case(LENS, n_new, Hq, Hkv, seed=nodes, packed=nodes % 2 == 0, nhd=nodes == 7).check()


@pytest.mark.parametrize("nodes", [64, 65, 100, 256])
@pytest.mark.parametrize("Hq, Hkv", [(4, 4), (8, 2), (8, 1)])
def test_large_trees(Hq, Hkv, nodes):
    Case([600, 45, 0], [nodes, nodes // 3, nodes], Hq, Hkv, seed=nodes, packed=nodes == 100).check()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("lens", [[0, 40, 300], [0, 0, 0]])
def test_any_mask_and_rows_that_see_nothing(packed, lens):
    c = Case(lens, [40, 33, 12], 8, 2, masks="any", packed=packed, seed=5)
    assert any((~m.any(1)).any() for m in c.seen)
    c.check()


@pytest.mark.parametrize("nodes", [1, 5, 40])
def test_no_mask_means_a_chain(nodes):
    Case([100, 0, 77], [nodes, nodes, 1], 8, 2, masks="chain", seed=nodes).check()


def test_bits_of_nodes_that_do_not_exist_are_ignored():
    c = Case([50, 20], [10, 3], 4, 2, seed=2)
    kw = c.kwargs()
    extra = kw["mask"].clone()
    extra[:10] |= ~((1 << 10) - 1)
    extra[10:] |= ~((1 << 3) - 1)
    a, b = c.run(), c.run(mask=extra)
    assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)


@pytest.mark.parametrize("b, k", [(1, 40), (8, 5), (16, 40), (32, 17), (64, 3), (1024, 2)])
@pytest.mark.parametrize("Hq, Hkv, nodes", [(8, 2, 9), (4, 4, 30), (16, 2, 1)])
def test_selected_slots(Hq, Hkv, nodes, b, k):
    c = Case([0, 1, 33, 500, 1500], [nodes, nodes, 0, nodes, 1], Hq, Hkv, seed=b + k, packed=nodes == 9)
    c.select(k, b, empty=((3, 0), (4, Hkv - 1))).check()


def test_spans_outside_the_cache_are_skipped():
    c = Case([200, 100], [5, 5], 4, 2, seed=4).select(6, 16)
    want = c.reference()
    start, length, count = c.sel
    bad = [(x.copy()) for x in c.sel]
    room = [np.concatenate([x, x], axis=2) for x in bad[:2]]
    n = start.shape[2]
    for s in range(2):
        for h in range(2):
            c0 = count[s, h]
            room[0][s, h, c0:c0 + 4] = [-3, c.rows - 2, 5, 2 ** 31 - 1]
            room[1][s, h, c0:c0 + 4] = [4, 7, -1, 9]
            bad[2][s, h] = c0 + 4
    assert bad[2].max() <= 2 * n
    c.sel = (room[0], room[1], bad[2])
    c.check(want=want)


def test_long_contexts_split_over_many_workgroups():
    Case([20011, 40000, 3], [12, 3, 12], 8, 2, seed=8).check()
    Case([33333], [16], 4, 4, seed=9, packed=True, nhd=True).check()
    Case([9000], [128], 8, 1, seed=10).check()
    Case([30000], [20], 8, 2, seed=11).select(400, 32).check()


def test_scale_and_sharp_logits():
    c = Case([300, 40], [9, 9], 8, 2, seed=6)
    c.check(scale=0.3)
    # queries as large as bf16 activations get: one key takes nearly all the weight.  A logit of some 2^8 is off by 2^-24 of the
    # sum of its terms' sizes, 2^11 at most here: 2^-13 of the weights
    c = Case([300, 40], [9, 9], 8, 2, seed=7, sharp=30.0)
    out, size, lse = c.reference()
    r = c.run()
    assert bool(((r.out.double() - out).abs() <= 2.0 ** -12 * size).all())
    assert bool(((r.lse.double() - lse).abs() <= 1e-5 * lse.abs()).all())


def test_logits_near_the_end_of_the_range():
    """Logits of 1e30: all the weight is on the largest, and nothing overflows.  That weight is no power of two (it is relative
    to a rounded maximum), so a bf16 result has its rounding, 2^-8 of the size, beside its own."""
    c = Case([400], [6], 4, 2, seed=12)
    c.q = (c.q.float() * 1e30).bfloat16()
    out, size, lse = c.reference()
    for kw in ({}, dict(want_f32=False, want_bf16=True)):
        r = c.run(**kw)
        if kw:
            assert bool(((r.out_bf16.double() - out).abs() <= BF16 * (out.abs() * (1 + BF16) + size) + F32 * size).all())
        else:
            assert bool(((r.out.double() - out).abs() <= F32 * size).all())
        assert bool(((r.lse.double() - lse).abs() <= 1e-5 * lse.abs()).all())


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_masked_may_hold_anything(what, packed):
    """K and V rows that no bit lets a node see: of other branches, of the room behind the nodes, of other sequences."""
    c = Case([70, 0, 33], [21, 40, 3], 8, 2, seed=13, packed=packed)
    want = c.reference()
    clean = [c.run(), c.run(want_f32=False, want_bf16=True)]
    for s, n in enumerate(c.n_new):
        for j in range(n):                                       # one node's rows at a time: the others must not notice
            if j % 5 != 3:
                continue
            blind = ~c.seen[s][:, j]
            X, at = ((c.Kd, c.Vd), c.cu[s] + j) if packed else ((c.K, c.V), c.row0[s] + c.lens[s] + j)
            old = [x[:, at].clone() for x in X]
            for x in X:
                x[:, at] = what
            for r0, kw in zip(clean, ({}, dict(want_f32=False, want_bf16=True))):
                r = c.run(**kw)
                t = torch.arange(c.cu[s], c.cu[s + 1], device="cuda")[torch.from_numpy(blind).cuda()]
                a, b = (x.out if x.out is not None else x.out_bf16 for x in (r, r0))
                assert torch.equal(a[t], b[t]) and torch.equal(r.lse[t], r0.lse[t])
            for x, o in zip(X, old):
                x[:, at] = o
    for s in range(3):                                           # the room behind every sequence
        for x in (c.K, c.V):
            x[:, c.row0[s] + c.lens[s] + (0 if packed else c.n_new[s]): c.row0[s + 1]] = what
    c.check(want=want)


def test_malformed_tables_are_cut():
    c = Case([64, 64], [8, 8], 4, 2, seed=14)
    base = c.run()
    r = c.run(cu_new=i32([0, 8, 400]))                           # more nodes than there are rows and max_nodes
    assert torch.equal(r.out, base.out)
    r = c.run(cu_new=i32([0, 8, 3]))
    assert torch.equal(r.out[:8], base.out[:8]) and bool((r.out[8:] == 9.0).all())
    r = c.run(cu_new=i32([-1, 8, 16]))
    assert bool((r.out[:8] == 9.0).all()) and torch.equal(r.out[8:], base.out[8:])
    r = c.run(seq_len=i32([10 ** 9, 64]))                        # cut to max_seqlen = 64
    assert torch.equal(r.out, base.out)
    for kw in (dict(seq_row0=i32([-5, c.row0[1]])), dict(seq_len=i32([-5, 64])), dict(seq_row0=i32([2 ** 31 - 1, c.row0[1]]))):
        r = c.run(**kw)
        assert torch.equal(r.out[8:], base.out[8:]) and bool(torch.isfinite(r.out).all())


def test_bit_identical_from_call_to_call_and_on_another_stream():
    c = Case([5000, 700], [20, 9], 8, 2, seed=15)
    a, b = c.run(), c.run()
    st = torch.cuda.Stream()
    r = _dsk().make_tree_attn_args(c.q, c.K, c.V, **c.kwargs())
    torch.cuda.synchronize()
    _dsk().dsk_tree_decode_attn(r.args, st)
    st.synchronize()
    for x in (b, r):
        assert torch.equal(a.out, x.out) and torch.equal(a.lse, x.lse)


def test_one_node_equals_the_decode_attention():
    """A tree of its root alone is a decode step: dense attention over the prefix and the new row."""
    dsk = _dsk()
    c = Case([3000], [1], 32, 8, seed=16, spare=0)
    den = dsk.dense_decode_attn(c.q, c.K, c.V, i32([0, c.rows]), c.rows)
    r = c.run()
    torch.cuda.synchronize()
    assert float((r.out - den.out).abs().max()) <= 1e-5 and float((r.lse - den.lse).abs().max()) <= 1e-5


# ---- more than 128 rows and their kernel (bf16 results, from 512 keys a workgroup on, 2048 for one sequence alone) ---
@pytest.mark.parametrize("lens, n_new, Hq, Hkv", [
    ([20000], [64], 32, 8),                                      # every wavefront has rows
    ([20033], [33], 40, 8),                                      # 165 rows: two wavefronts have none, one has five
    ([30000, 0, 21, 29999], [64, 64, 3, 40], 32, 8),             # an empty prefix, a short one, fewer nodes than announced
    ([70001, 4096], [256, 1], 8, 4),                             # 512 rows: two passes
    ([34100], [100], 32, 16),
    ([66000], [64], 32, 8),
    ([65999], [40], 40, 8),
    ([131100], [200], 8, 4),
])
@pytest.mark.parametrize("packed", [False, True])
def test_many_rows_over_long_contexts(lens, n_new, Hq, Hkv, packed):
    Case(lens, n_new, Hq, Hkv, seed=len(lens) + n_new[0], packed=packed, nhd=packed, pad_tokens=2).check()


@pytest.mark.parametrize("end", list(range(20480 - 3, 20480 + 3)) + [20480 + 31, 20480 + 33, 20480 + 64, 20480 + 127])
def test_many_rows_where_the_prefix_ends_in_any_place_of_a_step(end):
    Case([end], [40], 32, 8, seed=end).check()


def test_many_rows_any_mask():
    c = Case([20000, 100], [64, 64], 32, 8, masks="any", seed=21)
    assert any((~m.any(1)).any() for m in c.seen)
    c.check()


@pytest.mark.parametrize("packed", [False, True])
def test_many_rows_masked_rows_may_hold_anything(packed):
    c = Case([20017], [64], 32, 8, seed=22, packed=packed)
    bf16 = dict(want_f32=False, want_bf16=True)
    clean = c.run(**bf16)
    for j in (1, 14, 15, 30, 47, 63):                            # by 32 keys: the first, middle and last of a tile and its neighbour
        blind = torch.from_numpy(~c.seen[0][:, j]).cuda()
        X, at = ((c.Kd, c.Vd), j) if packed else ((c.K, c.V), c.lens[0] + j)
        old = [x[:, at].clone() for x in X]
        for x in X:
            x[:, at, ::3] = float("nan")
            x[:, at, 1::3] = float("inf")
        r = c.run(**bf16)
        assert torch.equal(r.out_bf16[blind], clean.out_bf16[blind]) and torch.equal(r.lse[blind], clean.lse[blind])
        assert bool(r.out_bf16[~blind].isnan().any(-1).all())
        for x, o in zip(X, old):
            x[:, at] = o
    for x in (c.K, c.V):                                         # the room behind
        x[:, c.lens[0] + (0 if packed else 64):] = float("nan")
    r = c.run(**bf16)
    assert torch.equal(r.out_bf16, clean.out_bf16) and torch.equal(r.lse, clean.lse)


@pytest.mark.parametrize("Hq, Hkv, nodes", [(8, 8, 5), (32, 8, 13), (32, 8, 30), (32, 8, 40)])
def test_caches_larger_than_the_memory_side_cache(Hq, Hkv, nodes):
    """288 MB of K and V and more are read past that cache, by kernels of their own for every number of rows."""
    c = Case([75001], [nodes], Hq, Hkv, seed=nodes)
    assert c.rows * Hkv * 512 >= 288 << 20
    c.check()


def test_a_nan_that_is_seen_reaches_those_who_see_it():
    c = Case([70, 20017], [21, 64], 32, 8, seed=23)
    for s, j in ((0, 4), (1, 9)):
        c.V[:, c.row0[s] + c.lens[s] + j, 5] = float("nan")
    for kw in ({}, dict(want_f32=False, want_bf16=True)):
        r = c.run(**kw)
        got = (r.out if r.out is not None else r.out_bf16).isnan()
        for s, j in ((0, 4), (1, 9)):
            sees = torch.from_numpy(c.seen[s][:, j]).cuda()
            own = got[c.cu[s]: c.cu[s + 1]]
            assert bool(own[sees][..., 5].all()) and not bool(own[~sees].any()) and not bool(own[..., :5].any())


# ---- offsets that pass 32 bits ----------------------------------------------------------------------------------
@pytest.fixture(scope="module")
def far():
    """K and V of three heads as views of rows of 10240 channels: 225,000 rows are 2^31 channels and more."""
    rows, g = 225_000, torch.Generator(device="cuda")
    g.manual_seed(31)
    X = torch.empty(rows, 80, D, dtype=torch.bfloat16, device="cuda")
    assert (rows - 5_000) * 80 * D > 2 ** 31
    X[:, :6] = torch.randn(rows, 6, D, generator=g, device="cuda").bfloat16()
    yield X[:, :3].transpose(0, 1), X[:, 3:6].transpose(0, 1)
    del X
    torch.cuda.empty_cache()


@pytest.mark.parametrize("Hq, nodes, packed", [(3, 9, False), (6, 40, False), (6, 40, True), (24, 30, False), (24, 30, True)])
def test_rows_beyond_32_bits(far, Hq, nodes, packed):
    for lens in ([224_900], [2_000, 222_800]):                   # the second sequence begins far away
        c = Case(lens, [nodes] * len(lens), Hq, 3, packed=packed, seed=nodes, spare=0)
        assert c.rows <= 225_000
        c.K, c.V = far
        c.check()


def test_selected_rows_beyond_32_bits(far):
    c = Case([224_950], [25], 12, 3, seed=33, spare=0)
    c.K, c.V = far
    c.select(40, 32)
    for h in range(3):
        c.sel[0][0, h, -30:] = np.sort(c.rng.choice(np.arange(219_000, 224_900, 32), 30, replace=False))
        c.sel[1][0, h, -30:] = 32
    c.check()


def test_no_token_at_all():
    c = Case([40, 3], [0, 0], 8, 2, seed=34)
    c.q = torch.empty(0, 8, D, dtype=torch.bfloat16, device="cuda")
    r = _dsk().tree_decode_attn(c.q, c.K, c.V, **{**c.kwargs(), "mask": None}, want_bf16=True)
    torch.cuda.synchronize()
    assert r.out.shape == r.out_bf16.shape == (0, 8, D)


def test_a_token_of_several_slots_counts_as_often():
    c = Case([300], [7], 8, 2, seed=35).select(6, 16)
    for x in c.sel[:2]:
        x[0, :, 1], x[0, :, 4] = x[0, :, 0], x[0, :, 3]
    c.check()


# ---- one sequence that gives every CU a workgroup of eight wavefronts, and many parts of a row -------------------
@pytest.mark.parametrize("end", [9000, 9216 - 30, 9216 - 1, 9216, 9216 + 1, 9216 + 63, 9216 + 65, 9216 + 127, 20001])
@pytest.mark.parametrize("nodes, packed", [(13, False), (30, True)])
def test_one_long_sequence(end, nodes, packed):
    Case([end], [nodes], 32, 8, seed=end, packed=packed, nhd=not packed, pad_tokens=1).check()


@pytest.mark.parametrize("nodes", [14, 31])
def test_one_long_sequence_any_mask_and_rows_that_hold_anything(nodes):
    c = Case([10007], [nodes], 32, 8, masks="any", seed=nodes)
    c.check()
    clean = c.run(want_bf16=True)
    j = nodes - 2
    blind = torch.from_numpy(~c.seen[0][:, j]).cuda()
    for x in (c.K, c.V):
        x[:, c.lens[0] + j, ::3] = float("nan")
        x[:, c.lens[0] + j, 1::3] = float("inf")
        x[:, c.lens[0] + nodes:] = float("nan")
    r = c.run(want_bf16=True)
    for a, b in ((r.out, clean.out), (r.out_bf16, clean.out_bf16), (r.lse, clean.lse)):
        assert torch.equal(a[blind], b[blind])
    assert bool(r.out[~blind].isnan().any(-1).all())


@pytest.mark.parametrize("Hq, Hkv, nodes", [(4, 1, 1), (4, 1, 16), (8, 1, 16), (8, 1, 33), (5, 1, 9)])
@pytest.mark.parametrize("lens", [[65537], [33000, 20, 32999]])
def test_one_head_in_many_parts(Hq, Hkv, nodes, lens):
    Case(lens, [nodes] * len(lens), Hq, Hkv, seed=nodes).check()


@pytest.mark.parametrize("end", list(range(20480 - 3, 20480 + 3)) + [20480 + 31, 20480 + 33, 20480 + 64, 20480 + 127])
def test_many_rows_of_two_sequences_where_the_prefix_ends_in_any_place_of_a_step(end):
    Case([end, 3], [40, 2], 32, 8, seed=end).check()


@pytest.mark.parametrize("packed", [False, True])
def test_many_rows_of_two_sequences_masked_rows_may_hold_anything(packed):
    c = Case([20017, 3], [64, 1], 32, 8, seed=41, packed=packed)
    bf16 = dict(want_f32=False, want_bf16=True)
    clean = c.run(**bf16)
    for j in (1, 14, 15, 30, 47, 63):
        blind = torch.from_numpy(np.append(~c.seen[0][:, j], True)).cuda()
        X, at = ((c.Kd, c.Vd), j) if packed else ((c.K, c.V), c.lens[0] + j)
        old = [x[:, at].clone() for x in X]
        for x in X:
            x[:, at, ::3] = float("nan")
            x[:, at, 1::3] = float("inf")
        r = c.run(**bf16)
        assert torch.equal(r.out_bf16[blind], clean.out_bf16[blind]) and torch.equal(r.lse[blind], clean.lse[blind])
        assert bool(r.out_bf16[~blind].isnan().any(-1).all())
        for x, o in zip(X, old):
            x[:, at] = o


def test_more_sequences_than_workgroups_and_the_largest_bounds():
    """Bounds as large as they may be (nothing lies there): 100 sequences of a part each, 2^31 keys and more in all."""
    c = Case([5 + s % 3 for s in range(100)], [2] * 100, 8, 8, seed=51)
    r = _dsk().make_tree_attn_args(c.q, c.K, c.V, **c.kwargs(max_seqlen=0x7FFF0000))
    r.args.total_rows = 0x7FFFFFFF
    assert _dsk().dsk_tree_attn_workspace_bytes(r.args) <= r.args.workspace_bytes
    _dsk().dsk_tree_decode_attn(r.args)
    torch.cuda.synchronize()
    out, size, _ = c.reference()
    assert bool(((r.out.double() - out).abs() <= F32 * size).all())


@pytest.mark.parametrize("lens, Hq, Hkv, nodes", [([40], 8, 2, 5), ([3000], 8, 2, 5), ([20000, 3], 32, 8, 40), ([9000], 32, 8, 30)])
def test_a_query_that_is_not_a_number_gets_none(lens, Hq, Hkv, nodes):
    c = Case(lens, [nodes] + [1] * (len(lens) - 1), Hq, Hkv, seed=61)
    for kw in ({}, dict(want_f32=False, want_bf16=True)):
        clean = c.run(**kw)
        c.q[2, 1] = float("nan")
        r = c.run(**kw)
        out, want = (x.out if x.out is not None else x.out_bf16 for x in (r, clean))
        hit = torch.zeros(c.N, Hq, dtype=torch.bool, device="cuda")
        hit[2, 1] = True
        assert bool(out[hit].isnan().all()) and bool(r.lse[hit].isnan().all())
        assert torch.equal(out[~hit], want[~hit]) and torch.equal(r.lse[~hit], clean.lse[~hit])
        c.q[2, 1] = 1.0


# ---- batches: workgroups are numbered through the parts that there are --------------------------------------------
@pytest.mark.parametrize("Hq, Hkv, nodes", [(8, 2, 3), (8, 2, 16), (32, 8, 40)])
def test_many_sequences_with_and_without_nodes(Hq, Hkv, nodes):
    """More sequences than lanes, some without nodes, some without a prefix, the last ones with none of both."""
    rng = np.random.default_rng(nodes)
    lens = [int(rng.integers(0, 900)) if s % 3 else 0 for s in range(150)]
    n_new = [0 if s % 4 == 1 or s > 146 else int(rng.integers(1, nodes + 1)) for s in range(150)]
    n_new[10] = nodes
    Case(lens, n_new, Hq, Hkv, seed=nodes, pad_tokens=1).check()


def test_sequences_that_share_their_prefix():
    """Several drafts over one prompt: the prefixes' keys are more than the cache has rows."""
    c = Case([30000, 5], [13, 13], 32, 8, seed=71, packed=True)
    c.row0, c.lens, c.n_new, c.seen = [0] * 5, [30000, 29000, 30000, 7, 30005], [13] * 5, c.seen[:1] * 5
    c.cu, c.N = starts(c.n_new), 65
    g = torch.Generator(device="cuda")
    g.manual_seed(72)
    c.Kd, c.Vd = (torch.randn(8, 65, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    c.q = torch.randn(65, 32, D, generator=g, device="cuda").bfloat16()
    c.row0.append(0)
    c.check()


def test_batches_whose_bounds_are_not_reached():
    """max_seqlen far above every length: parts that no sequence has."""
    c = Case([3000, 1, 0, 2999], [14, 14, 1, 9], 32, 8, seed=73)
    out, size, lse = c.reference()
    for kw in (dict(max_seqlen=200_000), dict(max_seqlen=3000)):
        r = c.run(**kw)
        assert bool(((r.out.double() - out).abs() <= F32 * size).all())
        assert bool(((r.lse.double() - lse).abs() <= 1e-5 * (1 + lse.abs())).all())


# ---- infinities in rows that are seen --------------------------------------------------------------------------------
@pytest.mark.parametrize("lens, n_new, Hq, Hkv, k", [
    ([300], [5], 4, 2, 0),                                       # up to 32 rows, stages of 128 keys, the last one with the nodes
    ([300], [21], 8, 4, 0),                                      # up to 64, stages of 64
    ([300], [40], 4, 2, 0),                                      # more, the same as four wavefronts' rows
    ([700, 300, 90], [30, 40, 9], 24, 8, 0),
    ([9003], [12], 32, 8, 0),                                    # eight wavefronts, many parts
    ([9003], [30], 32, 8, 0),
    ([20003], [64], 32, 8, 0),
    ([1500], [9], 8, 2, 40),                                     # a selection
    ([1500], [40], 8, 2, 40),
])
@pytest.mark.parametrize("f32", [True, False])
def test_an_infinite_value_gives_an_infinity_wherever_its_row_lies(lens, n_new, Hq, Hkv, k, f32):
    """No weight here is below 2^-90 of the largest (logits of K's scale, up to some 30 apart), so the weighted sum over a row of
    V with an infinity in a channel is that infinity for every node and head, whatever else it holds, and with both signs NaN."""
    c = Case(lens, n_new, Hq, Hkv, seed=81)
    if k:
        c.select(k, 16)
    kw = {} if f32 else dict(want_f32=False, want_bf16=True)
    clean, G, inf, n = c.run(**kw), Hq // Hkv, float("inf"), n_new[0]
    p = c.prefix(0, 1)
    L = len(p)
    for i in sorted({0, 1, 17, 32, 63, 64, 100, L // 3, L // 2, L - 130, L - 65, L - 33, L - 2, L - 1} & set(range(L))):
        old = c.V[1, p[i]].clone()
        c.V[1, p[i], 3], c.V[1, p[i], 77] = inf, -inf
        other = p[(i + L // 2) % L]
        was = c.V[1, other, 77].clone()
        r = c.run(**kw)
        a, b = (x.out if f32 else x.out_bf16 for x in (r, clean))
        hit = torch.zeros_like(a, dtype=torch.bool)
        hit[:n, G:2 * G, 3] = hit[:n, G:2 * G, 77] = True
        assert bool((a[:n, G:2 * G, 3] == inf).all()) and bool((a[:n, G:2 * G, 77] == -inf).all()), i
        assert torch.equal(a[~hit], b[~hit]) and torch.equal(r.lse, clean.lse), i
        c.V[1, other, 77] = inf
        r = c.run(**kw)
        a = r.out if f32 else r.out_bf16
        assert bool(a[:n, G:2 * G, 77].isnan().all()) and bool((a[:n, G:2 * G, 3] == inf).all()), i
        c.V[1, other, 77], c.V[1, p[i]] = was, old


# ---- long sums of equal weights ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("a", [2.15625, 4.1875])
@pytest.mark.parametrize("Hq, nodes, f32, waves", [(8, 4, True, 4), (8, 4, False, 4), (32, 10, True, 2), (32, 32, True, 1), (32, 64, False, 1)])
def test_long_sums_of_equal_weights(a, Hq, nodes, f32, waves):
    """64 sequences of 8 KV heads over one prefix, a part each: 128 keys of logit 0, then 65536 alike of logit a, which is not
    far enough above to become the reference of the exponents, so every weight is e^a.  `waves` wavefronts share the keys.
    lse: an exponent below 8 is off by 3 * 2^-24 of it (scale, product, rounding), a weight by 2^-22 and less of it; 16 of
    them and the parts of eight wavefronts are added up with 9 roundings: 2^-20 of the sum in all.  log2 of it (16 to 32) and what
    is added to it are rounded to 2^-20 each, the result once more: 2^-20 (1 + 2 ln 2 + 0.5) < 4e-6.
    out (the same in all rows of a channel): a tile is two sums of 16 products, of three terms each in fp32 results; each is added
    with 2^-24 of the sum so far, half of the final one in the mean."""
    dsk = _dsk()
    B, Hkv, L = 64, 8, 65536 + 128
    K = torch.zeros(Hkv, L, D, dtype=torch.bfloat16, device="cuda")
    K[:, 128:, 0] = a
    v = torch.linspace(1.0, 2.0, D, device="cuda").bfloat16()
    V = v.expand(Hkv, L, D).contiguous()
    q = torch.zeros(B * nodes, Hq, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    Kd = torch.zeros(Hkv, B * nodes, D, dtype=torch.bfloat16, device="cuda")
    Vd = v.expand(Hkv, B * nodes, D).contiguous()
    r = dsk.tree_decode_attn(q, K, V, seq_row0=i32([0] * B), seq_len=i32([L] * B), cu_new=i32(range(0, B * nodes + 1, nodes)),
                             mask=None, max_nodes=nodes, max_seqlen=L, Kd=Kd, Vd=Vd, scale=1.0, want_f32=f32, want_bf16=not f32)
    torch.cuda.synchronize()
    want = torch.tensor([math.log(128 + 1 + i + 65536 * math.exp(a)) for i in range(nodes)], dtype=torch.float64, device="cuda")
    assert float((r.lse.double().view(B, nodes, Hq) - want[None, :, None]).abs().max()) <= 4e-6
    adds = (L // 32 // waves) * 2 * (3 if f32 else 1)
    bar = adds / 2 * 2.0 ** -24 + 2.0 ** -20 + (0 if f32 else 2 * BF16)
    got = (r.out if f32 else r.out_bf16).double()
    assert bool(((got - v.double()).abs() <= bar * v.double()).all())


def test_a_kept_call_is_made_again():
    c = Case([300, 40], [9, 9], 8, 2, seed=91)
    want = c.run(want_bf16=True)
    r = _dsk().make_tree_attn_args(c.q, c.K, c.V, **c.kwargs(want_bf16=True))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, st):
        for t in (r.out, r.out_bf16, r.lse):
            t.fill_(9.0)
        torch.cuda.synchronize()
        assert r.step(stream) == _dsk().DSK_OK
        torch.cuda.synchronize()
        assert torch.equal(r.out, want.out) and torch.equal(r.out_bf16, want.out_bf16) and torch.equal(r.lse, want.lse)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("row0, length", [(-5, 64), (-5, 0), (0, -1), (70, -2 ** 31), (2 ** 31 - 1, 64)])
@pytest.mark.parametrize("k", [0, 4])
def test_a_sequence_that_has_no_place_reads_no_other_one(packed, row0, length, k):
    """Its nodes lie nowhere in the cache, so in place they see what a selection names at most, and nothing of the rows that begin
    the cache; in buffers of their own they see each other."""
    c = Case([64, 64], [8, 8], 4, 2, seed=92, packed=packed)
    if k:
        c.select(k, 16)
    base = c.run()
    kw = dict(seq_row0=i32([row0, c.row0[1]]), seq_len=i32([length, 64]))
    r = c.run(**kw)
    c.K[:, : c.row0[1]], c.V[:, : c.row0[1]] = float("nan"), float("nan")
    blind = c.run(**kw)
    assert torch.equal(r.out[8:], base.out[8:]) and torch.equal(r.lse[8:], base.lse[8:])
    if not k:                                                    # (a selection's slots are taken as they are, of any region)
        assert torch.equal(blind.out[:8], r.out[:8]) and torch.equal(blind.lse[:8], r.lse[:8])
    if not k and not packed:
        assert bool((r.out[:8] == 0).all()) and bool((r.lse[:8] == -math.inf).all())
    want = Case([0, 64], [8, 8], 4, 2, seed=92, packed=True)
    if packed and not k:
        want.Kd, want.Vd, want.q, want.seen = c.Kd, c.Vd, c.q, c.seen
        alone = want.run(seq_len=i32([0, 0]))
        assert torch.equal(alone.out[:8], r.out[:8]) and torch.equal(alone.lse[:8], r.lse[:8])


# ---- batches whose cache has room for all sequences at max_seqlen: parts of equal lengths, whatever the lengths are -------
ROOMY = dict(spare=4200)


def _even(c):
    """The split takes such a batch for one of sequences of one length."""
    assert len(c.lens) > 1 and c.rows >= len(c.lens) * max(c.lens)
    return c


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("lens, n_new, Hq, Hkv, more", [
    # 33 to 64 rows a KV head, from 256 x 256 keys times heads on: eight wavefronts a CU
    ([4096] * 4, [13] * 4, 32, 8, {}),
    ([4096, 1000, 0, 3333], [13, 0, 16, 9], 32, 8, ROOMY),       # different lengths, one without nodes, an empty prefix
    ([4095, 33, 4000, 1], [0, 9, 1, 13], 32, 8, ROOMY),
    ([2048] * 32, [9] * 32, 32, 8, {}),
    ([2048] * 70, [9] * 69 + [0], 16, 4, dict(pad_tokens=3)),    # more sequences than lanes
    # 65 to 128 rows
    ([4096] * 4, [30] * 4, 32, 8, {}),
    ([4096, 1000, 0, 3333], [30, 0, 32, 17], 32, 8, ROOMY),
    ([4111] * 3, [120, 1, 77], 16, 16, {}),
    # more: eight wavefronts' rows at once from 512 keys a part on
    ([20480] * 2, [40, 40], 32, 8, {}),
    ([8192] * 8, [64] * 8, 32, 8, {}),
    ([9001] * 4, [100, 3, 100, 99], 32, 8, {}),                  # two passes
    ([4096, 1000, 0, 4001], [64, 0, 33, 64], 16, 2, ROOMY),
])
def test_batches_of_one_length_and_roomy_ones(lens, n_new, Hq, Hkv, more, packed):
    _even(Case(lens, n_new, Hq, Hkv, seed=sum(n_new), packed=packed, nhd=packed, **more)).check()


@pytest.mark.parametrize("nodes", [13, 30, 64])
def test_batches_of_one_length_any_mask(nodes):
    c = _even(Case([4200] * 4, [nodes, nodes, 1, nodes - 1], 32, 8, masks="any", seed=nodes))
    assert any((~m.any(1)).any() for m in c.seen)
    c.check()


@pytest.mark.parametrize("nodes", [13, 30, 40])
def test_batches_of_one_length_larger_than_the_memory_side_cache(nodes):
    c = _even(Case([18501] * 4, [nodes] * 4, 32, 8, seed=nodes))
    assert c.rows * 8 * 512 >= 288 << 20
    c.check()


@pytest.mark.parametrize("nodes", [13, 30, 64])
def test_batches_of_one_length_rows_that_are_masked_or_free_may_hold_anything(nodes):
    c = _even(Case([4097, 4090, 20, 0], [nodes] * 4, 32, 8, seed=nodes, **ROOMY))
    kws = ({}, dict(want_f32=False, want_bf16=True))
    clean = [c.run(**kw) for kw in kws]
    for x in (c.K, c.V):
        for s in range(4):                                       # the room behind every sequence's nodes
            x[:, c.row0[s] + c.lens[s] + nodes: c.row0[s + 1]] = float("nan")
    for kw, want in zip(kws, clean):
        r = c.run(**kw)
        assert torch.equal(r.lse, want.lse)
        assert torch.equal(r.out, want.out) if r.out is not None else torch.equal(r.out_bf16, want.out_bf16)
    j = nodes - 2
    for x in (c.K, c.V):
        for s in range(4):
            x[:, c.row0[s] + c.lens[s] + j, ::3] = float("nan")
            x[:, c.row0[s] + c.lens[s] + j, 1::3] = float("inf")
    blind = torch.from_numpy(np.concatenate([~m[:, j] for m in c.seen])).cuda()
    for kw, want in zip(kws, clean):
        r = c.run(**kw)
        a, b = (x.out if x.out is not None else x.out_bf16 for x in (r, want))
        assert torch.equal(a[blind], b[blind]) and torch.equal(r.lse[blind], want.lse[blind])
        assert bool(a[~blind].isnan().any(-1).all())


@pytest.mark.parametrize("end", [4096 - 33, 4096 - 1, 4096, 4096 + 1, 4096 + 31, 4096 + 65, 4096 + 127])
@pytest.mark.parametrize("nodes", [13, 30, 64])
def test_batches_of_one_length_where_the_prefix_ends_in_any_place_of_a_stage(end, nodes):
    _even(Case([end] * 5, [nodes] * 5, 32, 8, seed=end)).check()


@pytest.mark.parametrize("B", [257, 4096, 65535])
@pytest.mark.parametrize("f32", [True, False])
def test_as_many_sequences_as_there_may_be(B, f32):
    """A part each, most of them over one of four prefixes with the nodes' rows in buffers of their own."""
    dsk, g = _dsk(), torch.Generator(device="cuda")
    g.manual_seed(B)
    K, V = (torch.randn(2, 400, D, generator=g, device="cuda").bfloat16() for _ in range(2))
    lens, row0 = [130, 0, 33, 64], [0, 7, 300, 140]
    kinds = torch.arange(B, device="cuda") % 4
    two = (torch.arange(B, device="cuda") // 4) % 2              # sequences of two nodes and of one
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), (1 + two).cumsum(0)]).int()
    n = int(cu[-1])
    first = cu[:-1].long()
    kind = torch.zeros(n, dtype=torch.int64, device="cuda")
    for t in (first, (first + two)):
        kind[t] = kinds
    second = torch.ones(n, dtype=torch.bool, device="cuda")
    second[first] = False
    q4, k4, v4 = (torch.randn(8, h, D, generator=g, device="cuda").bfloat16() for h in (6, 2, 2))
    pick = 2 * kind + second                                     # a node's rows: by its sequence's kind and its place
    q, Kd, Vd = q4[pick], k4[pick].transpose(0, 1).contiguous(), v4[pick].transpose(0, 1).contiguous()
    r = dsk.tree_decode_attn(q, K, V, seq_row0=i32(row0)[kinds], seq_len=i32(lens)[kinds], cu_new=cu, mask=None, max_nodes=2,
                             max_seqlen=130, Kd=Kd, Vd=Vd, want_f32=f32, want_bf16=not f32)
    torch.cuda.synchronize()
    got = (r.out if f32 else r.out_bf16).double()
    for k in range(4):
        for h in range(2):
            p, hs = slice(row0[k], row0[k] + lens[k]), slice(3 * h, 3 * h + 3)
            w = slice(2 * k, 2 * k + 2)
            out, size, lse = tree_reference(q4[w, hs], K[h, p], V[h, p], k4[w, h], v4[w, h], np.tril(np.ones((2, 2), dtype=bool)),
                                            1.0 / math.sqrt(D))
            for i in range(2):
                t = (kind == k) & (second == bool(i))
                bar = F32 * size[i] + (0 if f32 else BF16 * (out[i].abs() * (1 + BF16) + size[i]))
                assert bool(((got[t][:, hs] - out[i]).abs() <= bar).all())
                assert bool(((r.lse[t][:, hs].double() - lse[i]).abs() <= 1e-5 * (1 + lse[i].abs())).all())


@pytest.mark.parametrize("lens, n_new, Hq, Hkv, k", [
    ([0, 1, 31, 32, 33, 64, 127, 700], [8] * 8, 8, 2, 0),        # 32 rows
    ([300, 9], [16, 16], 32, 8, 0),                              # 64
    ([9000], [16], 32, 8, 0),
    ([20000, 30], [1, 1], 4, 4, 0),
    ([4096] * 4, [13] * 4, 32, 8, 0),
    ([75001], [5], 8, 8, 0),                                     # 288 MB and more
    ([75001], [12], 32, 8, 0),
    ([1500, 40], [8, 8], 8, 2, 40),                              # a selection
    ([1500, 40], [16, 3], 16, 4, 40),
])
def test_bf16_results_of_up_to_64_rows_are_rounded_once(lens, n_new, Hq, Hkv, k):
    """Their weights are off by 2^-16 of each, and so is the sum by 2^-16 of its size, beside the rounding of the result."""
    c = Case(lens, n_new, Hq, Hkv, seed=95)
    if k:
        c.select(k, 16)
    out, size, _ = c.reference()
    r = c.run(want_f32=False, want_bf16=True)
    near = (F32 + 2.0 ** -16) * size
    assert bool(((r.out_bf16.double() - out).abs() <= BF16 * (out.abs() + near) + near).all())
