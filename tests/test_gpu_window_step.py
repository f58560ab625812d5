"""The calls on a cache in 8 bits one after the other, as a model's layer makes them: a prompt appended and attended to, block tables
of it, then steps of a token per sequence that append, attend to a window, select and attend to the selection and what is near.
Every result is held to the definition in 64 bits on the numbers that the cache stands for at that moment; bars as for the single
calls.  Captured steps and steps of two layers on two streams give the eager ones' bits."""
import pytest
import torch

from step_testutil import i32, starts
from test_gpu_window_attn import BF16, Case as WindowCase
from test_gpu_window_sparse import Case as SparseCase
from window_testutil import D, TINY, as_bytes, values

pytestmark = pytest.mark.gpu

ALL = 0x7FFFFFFF


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


class Layer:
    Hq, Hkv, BLOCK, BSLOT = 8, 2, 32, 16
    WINDOW, SINKS, NEAR = 128, 4, 64

    def __init__(self, prompts=(700, 45, 1100), seed=0):
        dsk = _dsk()
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.prompts, self.B = list(prompts), len(prompts)
        self.row0 = starts([-(-(n + 40) // self.BLOCK) * self.BLOCK for n in prompts])
        rows, N = self.row0[-1], sum(prompts)
        (self.K, self.ks), (self.V, self.vs) = (dsk.empty_kv8(self.Hkv, rows, scale_block=self.BLOCK) for _ in range(2))
        self.wq, self.wk = (1.0 + 0.1 * torch.randn(D, generator=self.g, device="cuda") for _ in range(2))
        self.freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)).float()
        self.first, self.len, self.len1 = i32(self.row0[:-1]), i32([0] * self.B), i32([0] * self.B)
        self.caches = dict(k_scale=self.ks, v_scale=self.vs, scale_block=self.BLOCK, seq_row0=self.first)
        # the prompts
        self.x = torch.zeros(N, self.Hq + 2 * self.Hkv, D, dtype=torch.bfloat16, device="cuda")
        self.prompt_append = self.appender(self.x, starts(self.prompts), max(prompts))
        self.prompt_attn = dsk.make_window_attn_args(self.prompt_append.q_out, self.K, self.V, seq_len=self.len,
                                                     cu_new=self.prompt_append.keep[8], max_new=max(prompts), max_seqlen=0,
                                                     want_f32=False, want_bf16=True, **self.caches)
        # a token of each sequence
        self.x1 = torch.zeros(self.B, self.Hq + 2 * self.Hkv, D, dtype=torch.bfloat16, device="cuda")
        self.append = self.appender(self.x1, list(range(self.B + 1)), 1)
        self.window = dsk.make_window_attn_args(self.append.q_out, self.K, self.V, seq_len=self.len, cu_new=self.append.keep[8],
                                                max_new=1, max_seqlen=max(prompts) + 40, window=self.WINDOW, n_sink=self.SINKS,
                                                want_f32=False, want_bf16=True, **self.caches)

    def appender(self, x, cu, max_new):
        q, k, v = x[:, : self.Hq], x[:, self.Hq: self.Hq + self.Hkv], x[:, self.Hq + self.Hkv:]
        return _dsk().make_kv8_appender(k, v, self.K, self.V, self.ks, self.vs, scale_block=self.BLOCK, seq_row0=self.first,
                                        seq_len=self.len, cu_new=i32(cu), max_new=max_new, q=q, q_weight=self.wq, k_weight=self.wk,
                                        inv_freq=self.freq)

    def fill(self, x):
        x.copy_(torch.randn(x.shape, generator=self.g, device="cuda") * torch.exp(torch.randn(*x.shape[:2], 1, generator=self.g, device="cuda")))

    def prompt(self):
        dsk = _dsk()
        self.fill(self.x)
        self.prompt_append.step()
        self.prompt_attn.step()
        torch.cuda.synchronize()
        self.check_window(self.prompt_attn, [0] * self.B, self.prompts, ALL, 0, self.prompt_append.q_out)
        # tables of the prompts' blocks, from the numbers that the codes stand for, which bf16 holds
        numbers = values(self.K, self.ks, self.BLOCK)
        K16 = numbers.bfloat16()
        assert torch.equal(K16.double(), numbers)
        ids = torch.randint(0, 60, (self.row0[-1],), generator=self.g, device="cuda", dtype=torch.int32)
        rb = dsk.compress_regions(seq_row0=self.row0[:-1], seq_len=self.prompts, region_entries=[n // 8 + 3 for n in self.prompts],
                                  Hq=self.Hq, K=K16, V=None, token_ids=ids,
                                  delim_ids=i32([3, 7, 11, 13, 17, 19, 23, 29]),
                                  class_weight_q=torch.randint(0, 11, (self.B, 8), generator=self.g, device="cuda", dtype=torch.uint8),
                                  C_per_seq=[16] * self.B, delta_per_seq=[8] * self.B, alpha_num=5, alpha_den=10, b=self.BSLOT)
        self.sel = dsk.make_select_args(rb, self.append.q_out, 256)
        self.sparse = dsk.make_window_sparse_args(self.append.q_out, self.K, self.V, seq_len=self.len1, sel_start=self.sel.sel_start,
                                                  sel_len=self.sel.sel_len, sel_count=self.sel.sel_count, b=self.BSLOT,
                                                  window=self.NEAR, n_sink=self.SINKS, max_seqlen=max(self.prompts) + 40, **self.caches)
        self.len.copy_(i32(self.prompts))
        torch.cuda.synchronize()

    def step(self, stream=None):
        """A token: every handle on the same stream (the current one, too, for the two small sums)."""
        self.append.step(stream)
        torch.add(self.len, 1, out=self.len1)
        self.window.step(stream)
        _dsk().dsk_select_topk(self.sel.args, stream)
        self.sparse.step(stream)
        self.len.copy_(self.len1)

    def results(self):
        return [as_bytes(t).clone() for t in (self.K, self.ks, self.V, self.vs)] + [
            t.clone() for t in (self.append.q_out, self.window.out_bf16, self.window.lse, self.sparse.out, self.sparse.lse, self.len)]

    def case(self, kind, lens, new, window, sinks, q):
        c = kind.__new__(kind)
        c.lens, c.new, c.Hq, c.Hkv, c.bits, c.block, c.window, c.sinks = lens, new, self.Hq, self.Hkv, 8, self.BLOCK, window, sinks
        c.row0, c.cu, c.rows, c.q = self.row0, starts(new), self.row0[-1], q
        c.K, c.ks, c.V, c.vs = self.K, self.ks, self.V, self.vs
        return c

    def check_window(self, r, lens, new, window, sinks, q):
        out, size, lse, bar = self.case(WindowCase, lens, new, window, sinks, q).reference()
        weights = 2.0 ** -16 if max(new) * self.Hq // self.Hkv <= 64 else BF16
        off = BF16 * (1 + BF16) * out.abs() + (weights * (1 + BF16) + bar[..., None]) * size + TINY
        assert bool(((r.out_bf16.double() - out).abs() <= off).all())
        assert bool(((r.lse.double() - lse).abs() <= bar + 1e-5 * lse.abs()).all())

    def check_step(self):
        """What the last step left, self.len counting its tokens."""
        assert int(self.append.dev_status) == 0 and int(self.prompt_append.dev_status) == 0
        lens = self.len.tolist()
        self.check_window(self.window, [n - 1 for n in lens], [1] * self.B, self.WINDOW, self.SINKS, self.append.q_out)
        c = self.case(SparseCase, lens, [0] * self.B, self.NEAR, self.SINKS, self.append.q_out)
        c.shared, c.sel = False, [t.cpu().numpy() for t in (self.sel.sel_start, self.sel.sel_len, self.sel.sel_count)]
        assert int(c.sel[2].min()) > 0
        out, size, lse, bar = c.reference()
        assert bool(((self.sparse.out.double() - out).abs() <= bar[..., None] * size + TINY).all())
        assert bool(((self.sparse.lse.double() - lse).abs() <= bar + 1e-5 * lse.abs()).all())


def test_a_prompt_and_steps_after_it():
    layer = Layer()
    layer.prompt()
    for step in range(5):
        layer.fill(layer.x1)
        layer.step()
        torch.cuda.synchronize()
        assert layer.len.tolist() == [n + step + 1 for n in layer.prompts]
        layer.check_step()


def test_captured_steps_replay_as_the_eager_ones():
    eager, layer = Layer(seed=3), Layer(seed=3)
    eager.prompt()
    layer.prompt()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        layer.step(stream)
    torch.cuda.synchronize()
    for step in range(36):                                       # over the end of a block of scales
        eager.fill(eager.x1)
        layer.x1.copy_(eager.x1)
        eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.results(), layer.results())), step
    layer.check_step()


def test_layers_on_two_streams_at_once():
    want, layers = [], [Layer(seed=5), Layer((300, 1200), seed=6)]
    for prompts, seed in (((700, 45, 1100), 5), ((300, 1200), 6)):
        layer = Layer(prompts, seed=seed)
        layer.prompt()
        layer.fill(layer.x1)
        for _ in range(6):
            layer.step()
        torch.cuda.synchronize()
        want.append(layer.results())
    streams = [torch.cuda.Stream() for _ in layers]
    for layer in layers:
        layer.prompt()
        layer.fill(layer.x1)
    torch.cuda.synchronize()
    for _ in range(6):
        for layer, stream in zip(layers, streams):
            with torch.cuda.stream(stream):
                layer.step()
    torch.cuda.synchronize()
    for layer, w in zip(layers, want):
        assert all(torch.equal(a, b) for a, b in zip(layer.results(), w))
        layer.check_step()
