"""Host-side checks of the calls on caches in 8 bits and with a sliding window (dsk_kv8_append, dsk_window_attn,
dsk_window_sparse_decode_attn): structs as in the header, bad arguments refused before anything is launched, workspaces."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000                    # never dereferenced: every call below is refused


@pytest.fixture(scope="module")
def dsk():
    import paper_2602_03184_amd as d
    return d


@pytest.mark.parametrize("name", ["dsk_kv8_append_args", "dsk_window_attn_args", "dsk_window_sparse_args"])
def test_struct_mirrors_the_header_field_by_field(dsk, tmp_path, name):
    st = getattr(dsk.binding, name)
    fields = [f[0] for f in st._fields_]
    prog = tmp_path / "st.c"
    prog.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"dsk.h\"\nint main(void) {\n"
                    "  printf(\"%%zu \", sizeof(%s));\n" % name
                    + "".join('  printf("%%zu ", offsetof(%s, %s));\n' % (name, f) for f in fields)
                    + "  printf(\"%d\\n\", (int)DSK_WINDOW_ALL);\n  return 0;\n}\n")
    exe = tmp_path / "st"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(prog), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert got == [C.sizeof(st)] + [getattr(st, f).offset for f in fields] + [dsk.DSK_WINDOW_ALL]


def _refused(call, make, cases):
    for field, value, want in cases:
        a = make()
        setattr(a, field, value)
        assert call(a, 0, check=False) == want, (field, value)


def _append(dsk):
    a = dsk.dsk_kv8_append_args()
    a.struct_size = C.sizeof(a)
    a.B, a.Hq, a.Hkv, a.D, a.n_tokens, a.max_new, a.total_rows, a.scale_block = 2, 4, 2, 128, 9, 5, 1000, 32
    for f in ("seq_row0", "seq_len", "cu_new", "tok_pos", "q", "k", "v", "q_weight", "k_weight", "inv_freq", "q_out", "K", "V",
              "k_scale", "v_scale"):
        setattr(a, f, FAKE)
    a.q_stride_tok = a.k_stride_tok = a.v_stride_tok = 8 * 128
    a.q_stride_head = a.k_stride_head = a.v_stride_head = 128
    a.kc_stride_tok = a.vc_stride_tok = 128
    a.kc_stride_head = a.vc_stride_head = 128 * 1000
    a.scale_stride_head, a.eps, a.rot_dim = 32, 1e-6, 128
    return a


def test_append_refuses(dsk):
    S, P, A, N = dsk.DSK_ERR_SHAPE, dsk.DSK_ERR_PARAM, dsk.DSK_ERR_ALIGN, dsk.DSK_ERR_NULL
    cases = [("struct_size", 8, dsk.DSK_ERR_VERSION), ("B", 0, S), ("B", 65536, S), ("Hkv", 0, S), ("Hq", 0, S), ("Hq", 4097, S), ("D", 64, S),
             ("n_tokens", -1, S), ("total_rows", -1, S), ("max_new", 0, P), ("scale_block", 16, P), ("scale_block", 0, P),
             ("scale_block", 256, P), ("scale_stride_head", 31, S), ("rot_dim", 24, P), ("rot_dim", 144, P), ("rot_dim", -16, P),
             ("flags", 2, P), ("eps", 0.0, P), ("eps", float("nan"), P), ("kc_stride_tok", 64, S), ("kc_stride_head", 0, S),
             ("vc_stride_tok", 136, A), ("kc_stride_head", 128 * 1000 + 8, A), ("q_stride_tok", 12, A), ("k_stride_head", -128, S),
             ("q", FAKE + 2, A), ("k", FAKE + 8, A), ("v", FAKE + 8, A), ("q_out", FAKE + 8, A), ("K", FAKE + 8, A),
             ("q_weight", FAKE + 4, A), ("k_weight", FAKE + 4, A), ("inv_freq", FAKE + 2, A)]
    cases += [(f, None, N) for f in ("seq_row0", "seq_len", "cu_new", "k", "v", "q_out", "K", "V", "k_scale", "v_scale", "inv_freq")]
    _refused(dsk.dsk_kv8_append, lambda: _append(dsk), cases)
    a = _append(dsk)
    a.n_tokens = 0                                               # nothing to do, nothing launched
    a.q = a.k = a.v = a.q_out = None
    assert dsk.dsk_kv8_append(a, 0, check=False) == dsk.DSK_OK


def _window(dsk, bits=8):
    a = dsk.dsk_window_attn_args()
    a.struct_size = C.sizeof(a)
    a.B, a.Hq, a.Hkv, a.D, a.n_tokens, a.max_new, a.max_seqlen, a.total_rows = 2, 4, 2, 128, 30, 20, 500, 1200
    a.window, a.n_sink = 100, 4
    for f in ("q", "K", "V", "seq_row0", "seq_len", "cu_new", "out", "out_bf16", "lse", "workspace"):
        setattr(a, f, FAKE)
    a.k_stride_tok = a.v_stride_tok = 128
    a.k_stride_head = a.v_stride_head = 128 * 1200
    if bits == 8:
        a.k_scale = a.v_scale = FAKE
        a.scale_stride_head, a.scale_block = 38, 32
    return a


def _sparse(dsk, bits=8):
    w, a = _window(dsk, bits), dsk.dsk_window_sparse_args()
    for f, _ in a._fields_:
        if hasattr(w, f):
            setattr(a, f, getattr(w, f))
    a.struct_size = C.sizeof(a)
    a.k, a.b = 8, 16
    a.sel_start = a.sel_len = a.sel_count = FAKE
    return a


def _common(dsk):
    S, P, A, N = dsk.DSK_ERR_SHAPE, dsk.DSK_ERR_PARAM, dsk.DSK_ERR_ALIGN, dsk.DSK_ERR_NULL
    cases = [("struct_size", 8, dsk.DSK_ERR_VERSION), ("B", 0, S), ("B", 65536, S), ("Hkv", 3, S), ("D", 64, S), ("total_rows", -1, S),
             ("max_seqlen", -1, S), ("max_seqlen", 0x7FFF0001, S), ("n_sink", -1, P), ("scale", -1.0, P), ("scale", float("nan"), P),
             ("k_stride_tok", 64, S), ("v_stride_head", -16, S), ("k_stride_tok", (1 << 24) + 16, S), ("scale_block", 48, P),
             ("scale_stride_head", 37, S), ("q", FAKE + 8, A), ("K", FAKE + 8, A), ("V", FAKE + 4, A), ("out", FAKE + 8, A),
             ("out_bf16", FAKE + 8, A), ("k_stride_tok", 136, A), ("v_stride_head", 128 * 1200 + 8, A),
             ("workspace_bytes", 0, dsk.DSK_ERR_WORKSPACE), ("workspace", None, dsk.DSK_ERR_WORKSPACE)]
    return cases + [(f, None, N) for f in ("q", "K", "V", "k_scale", "v_scale", "seq_row0", "seq_len")]


def test_window_attention_refuses(dsk):
    S, P, N = dsk.DSK_ERR_SHAPE, dsk.DSK_ERR_PARAM, dsk.DSK_ERR_NULL
    call = dsk.dsk_window_attn
    _refused(call, lambda: _window(dsk), _common(dsk) + [
        ("n_tokens", -1, S), ("max_new", 0, S), ("max_new", 0x7FFF0000, S), ("max_new", 2 ** 29, S), ("n_tokens", 2 ** 29, S),
        ("window", 0, P), ("window", -1, P), ("flags", 1, P), ("cu_new", None, N)])
    for bits in (8, 16):
        for change, want in (({}, dsk.DSK_ERR_WORKSPACE), (dict(out=None, out_bf16=None), N),
                             (dict(workspace=FAKE + 16, workspace_bytes=1 << 40), dsk.DSK_ERR_ALIGN),
                             (dict(n_tokens=0, q=None, out=None, out_bf16=None, workspace_bytes=1 << 40), dsk.DSK_OK),
                             (dict(n_tokens=0, total_rows=0, K=None, V=None, workspace_bytes=1 << 40), dsk.DSK_OK)):
            a = _window(dsk, bits)
            for f, x in change.items():
                setattr(a, f, x)
            assert call(a, 0, check=False) == want, (bits, change)
    a = _window(dsk, 16)
    a.k_stride_tok = 136                                         # bf16: multiples of 8
    assert call(a, 0, check=False) == dsk.DSK_ERR_WORKSPACE


def test_window_sparse_attention_refuses(dsk):
    S, P, N = dsk.DSK_ERR_SHAPE, dsk.DSK_ERR_PARAM, dsk.DSK_ERR_NULL
    call = dsk.dsk_window_sparse_decode_attn
    _refused(call, lambda: _sparse(dsk), _common(dsk) + [
        ("window", -1, P), ("k", 0, P), ("k", 0x7FFF0001, P), ("b", 0, P), ("b", 1025, P), ("flags", 1, P),
        ("sel_start", None, N), ("sel_len", None, N), ("sel_count", None, N)])
    a = _sparse(dsk)
    a.window, a.flags = 0, dsk.DSK_ATTN_SHARED_SELECTION
    assert call(a, 0, check=False) == dsk.DSK_ERR_WORKSPACE      # nothing else is wrong with it


def test_workspaces_do_not_shrink_as_the_cache_grows(dsk):
    lengths = sorted(set(range(0, 6000, 29)) | set(range(6000, 300_000, 1777)) | {2 ** e + d for e in range(5, 30) for d in (-17, 0, 1)}
                     | {0x7FFE0000})
    for B, Hq, Hkv, new, window in ((1, 32, 8, 1, dsk.DSK_WINDOW_ALL), (8, 32, 8, 4, dsk.DSK_WINDOW_ALL), (1, 8, 1, 1, 4096), (3, 5, 1, 9, 100),
                                    (65535, 8, 8, 300, dsk.DSK_WINDOW_ALL), (1, 64, 1, 40, dsk.DSK_WINDOW_ALL), (2, 40, 40, 8000, 70_000)):
        need = 0
        for L in lengths:
            a = _window(dsk)
            a.B, a.Hq, a.Hkv, a.max_new, a.window, a.max_seqlen = B, Hq, Hkv, new, window, L
            got = dsk.dsk_window_attn_workspace_bytes(a)
            assert got >= max(need, 256), (B, Hq, Hkv, new, window, L)
            need = got
        assert need <= 256 + a.n_tokens * Hq * 128 * 520 + 512   # 128 parts of a row at most, (m, l) and 128 channels each
    for B, Hq, Hkv, flags, b in ((1, 32, 8, 0, 32), (8, 32, 8, 2, 16), (1, 1, 1, 0, 1), (200, 8, 8, 0, 1000), (3, 64, 1, 2, 700)):
        for field, sizes in (("max_seqlen", lengths), ("k", sorted(set(range(1, 3000, 7)) | {2 ** e for e in range(30)})),
                             ("window", range(0, 9000, 13))):
            need = 0
            for x in sizes:
                a = _sparse(dsk)
                a.B, a.Hq, a.Hkv, a.flags, a.b, a.window, a.max_seqlen = B, Hq, Hkv, flags, b, 5000, 100_000
                setattr(a, field, x)
                got = dsk.dsk_window_sparse_workspace_bytes(a)
                assert got >= max(need, 256), (B, Hq, Hkv, b, field, x)
                need = got


def test_helpers_check_their_tensors(dsk):
    import torch
    i, X = torch.zeros(5, dtype=torch.int32), torch.zeros(2, 70, 128, dtype=torch.bfloat16)
    K, ks = dsk.empty_kv8(2, 70, scale_block=64, device="cpu")
    assert K.shape == (2, 70, 128) and ks.shape == (2, 2) and bool((ks.float() == 1.0).all())
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    kw = dict(seq_row0=i[:1], seq_len=i[:1], cu_new=i[:2], max_new=3)
    a = dsk.make_kv8_appender(x, x, K, K.clone(), ks, ks.clone(), scale_block=64, **kw)
    assert a.q_out is None and a.args.scale_stride_head == 2 and a.args.kc_stride_head == 70 * 128
    w = dsk.make_window_attn_args(x, K, K, k_scale=ks, v_scale=ks, scale_block=64, max_seqlen=4, **kw)
    assert w.args.k_stride_tok == 128 and w.args.window == dsk.DSK_WINDOW_ALL
    sel = dict(sel_start=torch.zeros(1, 2, 4, dtype=torch.int32), sel_len=torch.zeros(1, 2, 4, dtype=torch.int32),
               sel_count=torch.zeros(1, 2, dtype=torch.int32), b=8, seq_row0=i[:1], seq_len=i[:1])
    s = dsk.make_window_sparse_args(x[:1], X, X, window=0, **sel)
    assert s.args.flags == 0 and s.args.max_seqlen == 70
    wide = dsk.make_window_sparse_args(torch.zeros(1, 4, 128, dtype=torch.bfloat16), X, X, window=0, **sel)
    assert wide.args.flags == dsk.DSK_ATTN_SHARED_SELECTION
    for made in (a, w, s):                                       # no call on tensors that are not on the GPU
        with pytest.raises(AssertionError):
            made.step()
    bad = [lambda: dsk.make_kv8_appender(x, x, K, K, ks, ks, scale_block=32, **kw),                  # too few scales
           lambda: dsk.make_kv8_appender(x, x, X, X, ks, ks, scale_block=64, **kw),                  # a cache in bf16
           lambda: dsk.make_kv8_appender(x, x, K, K, ks.view(torch.uint8), ks, scale_block=64, **kw),
           lambda: dsk.make_kv8_appender(x[:, :1], x, K, K, ks, ks, scale_block=64, **kw),
           lambda: dsk.make_window_attn_args(x, K, K, max_seqlen=4, **kw),                           # codes without scales
           lambda: dsk.make_window_attn_args(x, X, X, k_scale=ks, v_scale=ks, scale_block=64, max_seqlen=4, **kw),
           lambda: dsk.make_window_attn_args(x, K, K, k_scale=ks, scale_block=64, max_seqlen=4, **kw),
           lambda: dsk.make_window_attn_args(x, K, K[:, :64], k_scale=ks, v_scale=ks, scale_block=64, max_seqlen=4, **kw),
           lambda: dsk.make_window_attn_args(x, X, X, max_seqlen=4, **dict(kw, seq_len=i[:1].to("meta"))),
           lambda: dsk.make_window_sparse_args(torch.zeros(1, 6, 128, dtype=torch.bfloat16), X, X[:1], window=0, **sel)]
    for make in bad:
        with pytest.raises(AssertionError):
            make()


def test_kept_calls_are_made_on_the_device_of_their_tensors(dsk, monkeypatch):
    import contextlib

    import torch
    i, X = torch.zeros(3, dtype=torch.int32), torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    K, ks = dsk.empty_kv8(2, 32, device="cpu")
    sel = torch.zeros(1, 2, 4, dtype=torch.int32)
    x = X[:1].contiguous()

    class Elsewhere:
        device = torch.device("cuda", 1)

    order = []

    @contextlib.contextmanager
    def on(device):
        order.append(device.index)
        yield
        order.append(0)

    def noted(args, stream, check):
        order.append((args, stream, check))
        return 0
    for name in ("dsk_kv8_append", "dsk_window_attn", "dsk_window_sparse_decode_attn"):
        monkeypatch.setattr(dsk.binding, name, noted)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", on)
    new = dict(seq_row0=i[:1], seq_len=i[:1], cu_new=i[:2], max_new=1)
    app = dsk.make_kv8_appender(x[:, :2], x[:, :2], K, K.clone(), ks, ks.clone(), scale_block=32, **new)
    app.dev_status = Elsewhere()
    made = [dsk.make_window_attn_args(x, X, X, max_seqlen=4, **new),
            dsk.make_window_sparse_args(x, X, X, seq_row0=i[:1], seq_len=i[:1], sel_start=sel, sel_len=sel, sel_count=sel[..., 0].contiguous(),
                                        b=8, window=0)]
    for kept in made:
        kept.lse = Elsewhere()
    for kept in [app] + made:
        order.clear()
        assert kept.step(5, check=False) == 0
        assert order[0] == 1 and order[2] == 0 and order[1][0] is kept.args and order[1][1:] == (5, False)


def test_selections_beyond_what_a_launch_holds_are_refused(dsk):
    """Lists times 32 query heads each are one side of the grid, parts of a list another, and a row has a workgroup where its parts
    are put together."""
    for B, Hq, Hkv, flags, k, b, fits in (
            (2, 2048, 1, 0, 8, 16, False), (2, 1440, 1, 0, 8, 16, True), (2, 1472, 1, 0, 8, 16, False), (2, 2048, 1, 2, 8, 16, True),
            (2, 65535, 65535, 0, 8, 16, True), (2, 65534, 32767, 0, 8, 16, True), (2, 65535, 1, 2, 8, 16, True),
            (2, 65535, 1, 0, 8, 16, False), (2, 62016, 1938, 0, 8, 16, True), (2, 62130, 1365, 0, 8, 16, False),
            (1, 1, 1, 0, 2 ** 25, 1000, False), (1, 1, 1, 0, 2 ** 25 - 2048, 1000, True), (1, 1, 1, 0, 2 ** 30, 1, True),
            (1, 1, 1, 0, 2 ** 30, 64, False), (1, 1, 1, 0, 2 ** 28, 64, True),
            (65535, 512, 1, 0, 1000, 64, False), (65535, 512, 1, 0, 8, 64, True), (65535, 256, 1, 0, 1000, 64, True)):
        a = _sparse(dsk)
        a.B, a.Hq, a.Hkv, a.flags, a.k, a.b, a.workspace_bytes = B, Hq, Hkv, flags, k, b, 0
        want = dsk.DSK_ERR_WORKSPACE if fits else dsk.DSK_ERR_SHAPE          # (nothing else is wrong with it)
        assert dsk.dsk_window_sparse_decode_attn(a, 0, check=False) == want, (B, Hq, Hkv, flags, k, b)


def test_new_tokens_beyond_what_a_launch_holds_are_refused(dsk):
    """256 rows of a KV head, or 128 of a result in 32 bits, are a workgroup of 512 or 256 threads, of which a launch has fewer than 2^32;
    so are 256 threads for a block of rows to append, and one more block that tokens can meet."""
    for Hq, Hkv, max_new, f32, fits in ((40000, 40000, 53687, False, False), (40000, 40000, 53687, True, False), (40000, 40000, 53504, False, True),
                                        (1, 1, 0x7FFE0000, False, True), (1, 1, 0x7FFE0000, True, True), (65535, 65535, 32767, False, True),
                                        (65535, 65535, 1, True, True)):
        a = _window(dsk)
        a.Hq, a.Hkv, a.max_new, a.workspace_bytes = Hq, Hkv, max_new, 0
        if not f32:
            a.out = None
        want = dsk.DSK_ERR_WORKSPACE if fits else dsk.DSK_ERR_SHAPE
        assert dsk.dsk_window_attn(a, 0, check=False) == want, (Hq, Hkv, max_new, f32)
    for block, n in ((32, 2 ** 29), (32, 2 ** 29 - 30), (64, 2 ** 30), (128, 2 ** 31 - 1)):
        a = _append(dsk)
        a.scale_block, a.n_tokens, a.max_new = block, n, 0x7FFFFFFF
        assert dsk.dsk_kv8_append(a, 0, check=False) == dsk.DSK_ERR_SHAPE, (block, n)
