"""The calls of a speculative decoding step as they are used together, on a batch with a region per sequence: plan, norm and
rotation into the cache, tree attention (over everything and over a selection), acceptance, the incremental update that takes
the accepted tokens, and the next selection; eagerly, in HIP graphs, on other streams."""
import math

import numpy as np
import pytest
import torch

from step_testutil import (D, accept_reference, ancestors, i32, random_parents, rope_reference, starts, tree_reference)

pytestmark = pytest.mark.gpu


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


class Loop:
    """A batch of sequences with tables, and everything a step needs made once."""
    HQ, HKV, B, NODES, STEPS, BSLOT = 8, 2, 3, 17, 4, 8

    def __init__(self, seed=0):
        dsk = _dsk()
        rng = np.random.default_rng(seed)
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.rng = rng
        self.lens0 = [700, 33, 260]
        room = [n + self.NODES * (self.STEPS + 2) for n in self.lens0]
        self.row0 = starts(room)
        rows = self.row0[-1]
        self.K = torch.randn(self.HKV, rows, D, generator=self.g, device="cuda").bfloat16()
        self.V = torch.randn(self.HKV, rows, D, generator=self.g, device="cuda").bfloat16()
        self.delim = i32(list(range(8)))
        self.ids = torch.randint(0, 60, (rows,), generator=self.g, device="cuda", dtype=torch.int32)
        self.wq = torch.randint(0, 11, (self.B, 8), generator=self.g, device="cuda", dtype=torch.uint8)
        self.C, self.delta = 16, 8
        self.rb = dsk.compress_regions(seq_row0=self.row0[:-1], seq_len=self.lens0, region_entries=[n // 8 + 3 for n in room],
                                       Hq=self.HQ, K=self.K, V=None, token_ids=self.ids, delim_ids=self.delim,
                                       class_weight_q=self.wq, C_per_seq=[self.C] * 3, delta_per_seq=[self.delta] * 3,
                                       alpha_num=5, alpha_den=10, b=self.BSLOT)
        N = self.N = self.B * self.NODES
        self.n_new = i32([0] * self.B)
        self.parent = torch.zeros(N, dtype=torch.int32, device="cuda")
        self.draft, self.target = torch.zeros_like(self.parent), torch.zeros_like(self.parent)
        self.x = torch.zeros(N, self.HQ + 2 * self.HKV, D, dtype=torch.bfloat16, device="cuda")
        q, k, v = self.x[:, : self.HQ], self.x[:, self.HQ: self.HQ + self.HKV], self.x[:, self.HQ + self.HKV:]
        self.qw, self.kw = (1.0 + 0.1 * torch.randn(D, generator=self.g, device="cuda") for _ in range(2))
        self.freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)).float()
        self.plan = dsk.make_step_plan(seq_row0=self.rb.seq_row0, seq_len=self.rb.seq_len, n_new=self.n_new, max_tokens=N,
                                       total_rows=rows, parent=self.parent, max_nodes=self.NODES)
        self.rope = dsk.make_norm_rope(q, k, v, self.K, self.V, pos=self.plan.tok_pos, row=self.plan.tok_row, q_weight=self.qw,
                                       k_weight=self.kw, inv_freq=self.freq)
        self.root = torch.zeros(self.B, self.HQ, D, dtype=torch.bfloat16, device="cuda")
        self.sel = dsk.make_select_args(self.rb, self.root, 64, shared=True)
        common = dict(seq_row0=self.rb.seq_row0, seq_len=self.rb.seq_len, cu_new=self.plan.cu_new, mask=self.plan.mask,
                      max_nodes=self.NODES, max_seqlen=max(room))
        self.dense = dsk.make_tree_attn_args(self.rope.q_out, self.K, self.V, **common)
        self.sparse = dsk.make_tree_attn_args(self.rope.q_out, self.K, self.V, sel_start=self.sel.sel_start,
                                              sel_len=self.sel.sel_len, sel_count=self.sel.sel_count, b=self.BSLOT,
                                              want_f32=False, want_bf16=True, **common)
        for t in (self.rope.q_out, self.dense.out, self.dense.lse, self.sparse.out_bf16, self.sparse.lse):
            t.zero_()                                            # rows behind the last sequence's nodes are never written
        self.app = dsk.make_batch_appender(self.rb, self.K, None, self.ids, self.delim, self.wq, C_=self.C, delta=self.delta,
                                           C_per_seq=None, delta_per_seq=None, alpha_num=5, alpha_den=10,
                                           max_new_tokens=self.NODES)
        self.acc = dsk.make_acceptor(self.K, self.V, seq_row0=self.rb.seq_row0, seq_len=self.rb.seq_len,
                                     cu_new=self.plan.cu_new, parent=self.parent, draft_ids=self.draft,
                                     target_ids=self.target, max_nodes=self.NODES, token_ids=self.ids,
                                     len_new=self.app.len_new)

    def draft_step(self):
        """New drafts and activations, in place."""
        n_new = [int(self.rng.integers(1, self.NODES + 1)) for _ in range(self.B)]
        n_new[int(self.rng.integers(0, self.B))] = self.NODES
        up = [random_parents(self.rng, n, 3) for n in n_new]
        tok = [self.rng.integers(0, 60, n).tolist() for n in n_new]
        tgt = []
        for p, t in zip(up, tok):
            y = self.rng.integers(0, 60, len(p)).tolist()
            for i in range(len(p)):
                kids = [j for j in range(len(p)) if p[j] == i]
                if kids and self.rng.random() < 0.9:
                    y[i] = t[kids[-1]]
            tgt.append(y)
        fill = [9] * (self.N - sum(n_new))                       # what lies behind the last sequence's nodes is never looked at
        self.n_new.copy_(i32(n_new))
        for to, vals in ((self.parent, up), (self.draft, tok), (self.target, tgt)):
            to.copy_(i32([v for y in vals for v in y] + fill))
        self.x.copy_(torch.randn(self.x.shape, generator=self.g, device="cuda"))
        self.root.copy_(torch.randn(self.root.shape, generator=self.g, device="cuda"))
        self.now = (n_new, up, tok, tgt)

    def calls(self, stream=None):
        dsk = _dsk()
        self.plan.step(stream)
        self.rope.step(stream)
        dsk.dsk_select_topk(self.sel.args, stream)
        dsk.dsk_tree_decode_attn(self.dense.args, stream)
        dsk.dsk_tree_decode_attn(self.sparse.args, stream)
        self.acc.step(stream)
        self.app.step(stream)

    def state(self):
        return [t.clone() for t in (self.K, self.V, self.ids, self.rb.seq_len, self.rb.block_start, self.rb.slot_base,
                                    self.rb.blocks_used, self.rb.ksum, self.rope.q_out, self.dense.out, self.dense.lse,
                                    self.sparse.out_bf16, self.sparse.lse, self.acc.path, self.acc.n_accepted,
                                    self.acc.next_id, self.plan.cu_new, self.plan.tok_row, self.plan.tok_pos)]


def test_steps_against_the_definitions():
    """Every call of four steps, on the state that the calls before it left."""
    dsk = _dsk()
    L = Loop()
    G = L.HQ // L.HKV
    for _ in range(L.STEPS):
        L.draft_step()
        n_new, up, tok, tgt = L.now
        lens = L.rb.seq_len.tolist()
        ids = L.ids.tolist()
        K0 = L.K.clone()
        L.plan.step()
        L.rope.step()
        dsk.dsk_select_topk(L.sel.args)
        torch.cuda.synchronize()
        cu = starts(n_new)
        q_want, q_size = rope_reference(L.x[:, : L.HQ], L.qw, 1e-6, L.plan.tok_pos, L.freq, False)
        k_want, k_size = rope_reference(L.x[:, L.HQ: L.HQ + L.HKV], L.kw, 1e-6, L.plan.tok_pos, L.freq, False)
        touched = torch.zeros(L.K.shape[1], dtype=torch.bool)
        for s in range(L.B):
            t = slice(cu[s], cu[s + 1])
            seen, depth = ancestors(up[s])
            assert L.plan.tok_pos[t].tolist() == [lens[s] + d for d in depth]
            r = slice(L.row0[s] + lens[s], L.row0[s] + lens[s] + n_new[s])
            touched[r] = True
            for got, want, size in ((L.rope.q_out[t].cpu(), q_want[t], q_size[t]),
                                    (L.K[:, r].transpose(0, 1).cpu(), k_want[t], k_size[t])):
                assert bool(((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * size).all())
            assert torch.equal(L.V[:, r].transpose(0, 1), L.x[t, L.HQ + L.HKV:])
        assert torch.equal(L.K[:, ~touched.cuda()], K0[:, ~touched.cuda()])
        dsk.dsk_tree_decode_attn(L.dense.args)
        dsk.dsk_tree_decode_attn(L.sparse.args)
        torch.cuda.synchronize()
        for s in range(L.B):
            t, seen = slice(cu[s], cu[s + 1]), ancestors(up[s])[0]
            nodes = slice(L.row0[s] + lens[s], L.row0[s] + lens[s] + n_new[s])
            for h in range(L.HKV):
                hs = slice(h * G, (h + 1) * G)
                n = int(L.sel.sel_count[s, h])
                spans = [torch.arange(a, a + b, device="cuda") for a, b in zip(L.sel.sel_start[s, h, :n].tolist(),
                                                                               L.sel.sel_len[s, h, :n].tolist())]
                every = torch.arange(L.row0[s], L.row0[s] + lens[s], device="cuda")
                for rows, r, half in ((every, L.dense, 0.0), (torch.cat(spans), L.sparse, 2.0 ** -8)):
                    out, size, lse = tree_reference(L.rope.q_out[t, hs], L.K[h][rows], L.V[h][rows], L.K[h][nodes],
                                                    L.V[h][nodes], seen, 1.0 / math.sqrt(D))
                    got = (r.out if r.out is not None else r.out_bf16)[t, hs].double()
                    assert bool(((got - out).abs() <= half * (out.abs() * (1 + half) + size) + 1e-5 * size).all())
                    assert bool(((r.lse[t, hs].double() - lse).abs() <= 1e-5 * (1 + lse.abs())).all())
        K1, V1 = L.K.clone(), L.V.clone()
        L.acc.step()
        L.app.step()
        torch.cuda.synchronize()
        for s in range(L.B):
            path, nxt = accept_reference(up[s], tok[s], tgt[s], L.NODES)
            assert L.acc.path[s, : len(path)].tolist() == path and int(L.acc.next_id[s]) == nxt
            assert int(L.rb.seq_len[s]) == lens[s] + len(path)
            first = L.row0[s] + lens[s]
            at = torch.tensor([first + p for p in path], device="cuda")
            assert torch.equal(L.K[:, first: first + len(path)], K1[:, at])
            assert torch.equal(L.V[:, first: first + len(path)], V1[:, at])
            ids[first: first + len(path)] = [tok[s][p] for p in path]
        assert L.ids.tolist() == ids
        assert not any(int(x.dev_status) for x in (L.plan, L.acc, L.rb))
    # the tables that four updates left are those of a compression of the sequences as they are now
    lens = L.rb.seq_len.tolist()
    assert all(n > m for n, m in zip(lens, L.lens0))
    want = dsk.compress_regions(seq_row0=L.row0[:-1], seq_len=lens, region_entries=np.diff(L.rb.cu_blocks.tolist()).tolist(),
                                Hq=L.HQ, K=L.K, V=None, token_ids=L.ids, delim_ids=L.delim, class_weight_q=L.wq,
                                C_per_seq=[L.C] * 3, delta_per_seq=[L.delta] * 3, alpha_num=5, alpha_den=10, b=L.BSLOT)
    torch.cuda.synchronize()
    assert torch.equal(L.rb.blocks_used, want.blocks_used)
    for s in range(L.B):
        a = int(want.cu_blocks[s])
        n = int(want.blocks_used[s])
        assert torch.equal(L.rb.block_start[a: a + n + 1], want.block_start[a: a + n + 1])
        assert torch.equal(L.rb.ksum[:, a: a + n], want.ksum[:, a: a + n])


def test_a_captured_step_replays_as_the_eager_one():
    """One graph for all steps: lengths, trees and activations change in place; every replay is checked against an eager
    run of the same step, with eager work and synchronizations between the replays."""
    eager, graphed = Loop(5), Loop(5)
    eager.draft_step()
    graphed.draft_step()
    eager.calls()
    graphed.calls()                                              # a warm-up, which is a step like the others
    torch.cuda.synchronize()
    for a, b in zip(eager.state(), graphed.state()):
        assert torch.equal(a, b)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            graphed.calls()
    for _ in range(3):
        eager.draft_step()
        graphed.draft_step()
        eager.calls()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager.state(), graphed.state()):
            assert torch.equal(a, b)


def test_two_steps_at_once_on_two_streams():
    """Two batches with workspaces of their own, their calls interleaved on two streams."""
    alone = [Loop(7), Loop(8)]
    both = [Loop(7), Loop(8)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for L in alone + both:
            L.draft_step()
        for L in alone:
            L.calls()
        torch.cuda.synchronize()
        for L, st in zip(both, streams):
            L.calls(st)
        torch.cuda.synchronize()
        for a, b in zip(alone, both):
            for x, y in zip(a.state(), b.state()):
                assert torch.equal(x, y)
