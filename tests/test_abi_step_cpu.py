"""Host-side checks of the calls of a step of several new tokens per sequence (dsk_step_plan, dsk_qk_norm_rope,
dsk_tree_decode_attn, dsk_accept_draft): structs as in the header, bad arguments refused before anything is launched."""
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


@pytest.mark.parametrize("name", ["dsk_step_plan_args", "dsk_norm_rope_args", "dsk_tree_attn_args", "dsk_accept_args"])
def test_struct_mirrors_the_header_field_by_field(dsk, tmp_path, name):
    st = getattr(dsk.binding, name)
    fields = [f[0] for f in st._fields_]
    prog = tmp_path / "st.c"
    prog.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"dsk.h\"\nint main(void) {\n"
                    "  printf(\"%%zu \", sizeof(%s));\n" % name
                    + "".join('  printf("%%zu ", offsetof(%s, %s));\n' % (name, f) for f in fields)
                    + "  printf(\"%d %d\\n\", (int)DSK_TREE_MAX_NODES, (int)DSK_ROPE_INTERLEAVED);\n  return 0;\n}\n")
    exe = tmp_path / "st"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(prog), "-o",
                           str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)]).split()]
    assert got == [C.sizeof(st)] + [getattr(st, f).offset for f in fields] + [dsk.DSK_TREE_MAX_NODES,
                                                                              dsk.DSK_ROPE_INTERLEAVED]


def _refused(call, make, cases):
    for field, value, want in cases:
        a = make()
        setattr(a, field, value)
        assert call(a, 0, check=False) == want, (field, value)


def _plan(dsk):
    a = dsk.dsk_step_plan_args()
    a.struct_size = C.sizeof(a)
    a.B, a.max_tokens, a.total_rows, a.max_nodes, a.mask_words = 3, 40, 1000, 33, 2
    for f in ("seq_row0", "seq_len", "n_new", "parent", "cu_new", "tok_seq", "tok_pos", "tok_row", "mask"):
        setattr(a, f, FAKE)
    return a


def test_plan_refuses(dsk):
    cases = [("struct_size", 8, dsk.DSK_ERR_VERSION), ("B", 0, dsk.DSK_ERR_SHAPE), ("B", 65536, dsk.DSK_ERR_SHAPE),
             ("max_tokens", 0, dsk.DSK_ERR_SHAPE), ("total_rows", -1, dsk.DSK_ERR_SHAPE),
             ("max_nodes", 0, dsk.DSK_ERR_PARAM), ("max_nodes", 257, dsk.DSK_ERR_PARAM),
             ("mask_words", 1, dsk.DSK_ERR_PARAM), ("mask_words", 9, dsk.DSK_ERR_PARAM)]
    cases += [(f, None, dsk.DSK_ERR_NULL) for f in ("seq_row0", "seq_len", "n_new", "cu_new", "tok_seq", "tok_pos", "tok_row")]
    _refused(dsk.dsk_step_plan, lambda: _plan(dsk), cases)


def _rope(dsk):
    a = dsk.dsk_norm_rope_args()
    a.struct_size = C.sizeof(a)
    a.n_tokens, a.Hq, a.Hkv, a.D, a.total_rows = 5, 4, 2, 128, 1000
    for f in ("q", "k", "v", "q_weight", "k_weight", "tok_pos", "tok_row", "inv_freq", "q_out", "K", "V"):
        setattr(a, f, FAKE)
    a.q_stride_tok = a.k_stride_tok = a.v_stride_tok = 8 * 128
    a.q_stride_head = a.k_stride_head = a.v_stride_head = 128
    a.kc_stride_tok = a.vc_stride_tok = 128
    a.kc_stride_head = a.vc_stride_head = 128 * 1000
    a.eps, a.rot_dim = 1e-6, 128
    return a


def test_norm_rope_refuses(dsk):
    cases = [("struct_size", 8, dsk.DSK_ERR_VERSION), ("D", 64, dsk.DSK_ERR_SHAPE), ("n_tokens", -1, dsk.DSK_ERR_SHAPE),
             ("Hq", 0, dsk.DSK_ERR_SHAPE), ("Hkv", 0, dsk.DSK_ERR_SHAPE), ("total_rows", -1, dsk.DSK_ERR_SHAPE),
             ("flags", 2, dsk.DSK_ERR_PARAM), ("rot_dim", 24, dsk.DSK_ERR_PARAM), ("rot_dim", 144, dsk.DSK_ERR_PARAM),
             ("rot_dim", -16, dsk.DSK_ERR_PARAM), ("eps", 0.0, dsk.DSK_ERR_PARAM), ("eps", float("nan"), dsk.DSK_ERR_PARAM),
             ("tok_pos", None, dsk.DSK_ERR_NULL), ("inv_freq", None, dsk.DSK_ERR_NULL), ("q_out", None, dsk.DSK_ERR_NULL),
             ("K", None, dsk.DSK_ERR_NULL), ("V", None, dsk.DSK_ERR_NULL), ("kc_stride_tok", 64, dsk.DSK_ERR_SHAPE),
             ("kc_stride_head", 0, dsk.DSK_ERR_SHAPE), ("vc_stride_head", 4, dsk.DSK_ERR_ALIGN),
             ("q_stride_tok", 12, dsk.DSK_ERR_ALIGN), ("q_stride_head", -128, dsk.DSK_ERR_SHAPE),
             ("q", FAKE + 2, dsk.DSK_ERR_ALIGN), ("k", FAKE + 8, dsk.DSK_ERR_ALIGN), ("v", FAKE + 8, dsk.DSK_ERR_ALIGN),
             ("q_out", FAKE + 8, dsk.DSK_ERR_ALIGN), ("K", FAKE + 8, dsk.DSK_ERR_ALIGN),
             ("q_weight", FAKE + 4, dsk.DSK_ERR_ALIGN), ("inv_freq", FAKE + 4, dsk.DSK_ERR_ALIGN)]
    _refused(dsk.dsk_qk_norm_rope, lambda: _rope(dsk), cases)
    a = _rope(dsk)
    a.q = a.k = None
    assert dsk.dsk_qk_norm_rope(a, 0, check=False) == dsk.DSK_ERR_NULL
    a = _rope(dsk)
    a.n_tokens = 0                                               # nothing to do, nothing launched
    assert dsk.dsk_qk_norm_rope(a, 0, check=False) == dsk.DSK_OK
    a.q_out = None
    assert dsk.dsk_qk_norm_rope(a, 0, check=False) == dsk.DSK_OK
    a.q = a.k = a.v = a.tok_pos = a.tok_row = None
    assert dsk.dsk_qk_norm_rope(a, 0, check=False) == dsk.DSK_OK


def _tree(dsk):
    a = dsk.dsk_tree_attn_args()
    a.struct_size = C.sizeof(a)
    a.B, a.Hq, a.Hkv, a.D = 2, 4, 2, 128
    a.n_tokens, a.max_nodes, a.max_seqlen, a.total_rows = 30, 20, 500, 1200
    for f in ("q", "K", "V", "Kd", "Vd", "seq_row0", "seq_len", "cu_new", "mask", "sel_start", "sel_len", "sel_count", "out",
              "out_bf16", "lse", "workspace"):
        setattr(a, f, FAKE)
    a.k_stride_tok = a.v_stride_tok = a.kd_stride_tok = a.vd_stride_tok = 128
    a.k_stride_head = a.v_stride_head = a.kd_stride_head = a.vd_stride_head = 128 * 1200
    a.mask_words, a.k, a.b = 1, 8, 16
    a.workspace_bytes = 0
    return a


def test_tree_attention_refuses(dsk):
    assert dsk.dsk_tree_attn_workspace_bytes(_tree(dsk)) >= 256
    a = _tree(dsk)
    a.sel_start = a.sel_len = a.sel_count = None
    a.B, a.total_rows, a.max_seqlen = 65535, 0x7FFFFFFF, 0x7FFF0000      # more sequences than workgroups: a part each
    assert dsk.dsk_tree_attn_workspace_bytes(a) == 256
    cases = [("struct_size", 8, dsk.DSK_ERR_VERSION), ("D", 64, dsk.DSK_ERR_SHAPE), ("B", 0, dsk.DSK_ERR_SHAPE),
             ("Hkv", 3, dsk.DSK_ERR_SHAPE), ("n_tokens", -1, dsk.DSK_ERR_SHAPE), ("max_seqlen", -1, dsk.DSK_ERR_SHAPE),
             ("total_rows", -1, dsk.DSK_ERR_SHAPE), ("max_nodes", 0, dsk.DSK_ERR_PARAM), ("max_nodes", 257, dsk.DSK_ERR_PARAM),
             ("max_nodes", 33, dsk.DSK_ERR_PARAM), ("scale", -1.0, dsk.DSK_ERR_PARAM), ("scale", float("nan"), dsk.DSK_ERR_PARAM),
             ("flags", 1, dsk.DSK_ERR_PARAM), ("k", 0, dsk.DSK_ERR_PARAM), ("b", 0, dsk.DSK_ERR_PARAM),
             ("b", 1025, dsk.DSK_ERR_PARAM), ("k_stride_tok", 64, dsk.DSK_ERR_SHAPE), ("vd_stride_tok", 64, dsk.DSK_ERR_SHAPE),
             ("v_stride_head", -8, dsk.DSK_ERR_SHAPE), ("kd_stride_head", 12, dsk.DSK_ERR_ALIGN),
             ("k_stride_tok", 132, dsk.DSK_ERR_ALIGN), ("K", FAKE + 8, dsk.DSK_ERR_ALIGN), ("Vd", FAKE + 8, dsk.DSK_ERR_ALIGN),
             ("q", FAKE + 8, dsk.DSK_ERR_ALIGN), ("out", FAKE + 8, dsk.DSK_ERR_ALIGN), ("out_bf16", FAKE + 8, dsk.DSK_ERR_ALIGN),
             ("k_stride_tok", (1 << 24) + 8, dsk.DSK_ERR_SHAPE), ("v_stride_tok", (1 << 24) + 8, dsk.DSK_ERR_SHAPE),
             ("max_seqlen", 0x7FFF0001, dsk.DSK_ERR_SHAPE),
             ("workspace_bytes", 0, dsk.DSK_ERR_WORKSPACE), ("workspace", None, dsk.DSK_ERR_WORKSPACE)]
    cases += [(f, None, dsk.DSK_ERR_NULL) for f in ("q", "K", "V", "Kd", "Vd", "seq_row0", "seq_len", "cu_new", "sel_start",
                                                    "sel_len", "sel_count")]
    _refused(dsk.dsk_tree_decode_attn, lambda: _tree(dsk), cases)
    a = _tree(dsk)
    a.out = a.out_bf16 = None
    assert dsk.dsk_tree_decode_attn(a, 0, check=False) == dsk.DSK_ERR_NULL
    a = _tree(dsk)
    a.workspace, a.workspace_bytes = FAKE + 16, 1 << 40
    assert dsk.dsk_tree_decode_attn(a, 0, check=False) == dsk.DSK_ERR_ALIGN
    a = _tree(dsk)
    a.n_tokens, a.workspace_bytes = 0, 1 << 40                   # no node: nothing launched
    a.q = a.out = a.out_bf16 = None
    assert dsk.dsk_tree_decode_attn(a, 0, check=False) == dsk.DSK_OK


def _accept(dsk):
    a = dsk.dsk_accept_args()
    a.struct_size = C.sizeof(a)
    a.B, a.Hkv, a.D, a.n_layers = 2, 2, 128, 3
    a.total_rows, a.n_tokens, a.max_nodes, a.max_path = 1000, 30, 20, 8
    for f in ("seq_row0", "seq_len", "cu_new", "parent", "draft_ids", "target_ids", "K", "V", "Kd", "Vd", "path",
              "n_accepted", "next_id", "token_ids"):
        setattr(a, f, FAKE)
    a.len_new, a.token_ids = 2 * FAKE, 4 * FAKE
    for x in ("k", "v", "kd", "vd"):
        setattr(a, x + "_stride_tok", 128)
        setattr(a, x + "_stride_head", 128 * 1000)
        setattr(a, x + "_stride_layer", 128 * 2000)
    return a


def test_accept_refuses(dsk):
    cases = [("struct_size", 8, dsk.DSK_ERR_VERSION), ("D", 64, dsk.DSK_ERR_SHAPE), ("B", 0, dsk.DSK_ERR_SHAPE),
             ("Hkv", 0, dsk.DSK_ERR_SHAPE), ("n_layers", 0, dsk.DSK_ERR_SHAPE), ("n_tokens", -1, dsk.DSK_ERR_SHAPE),
             ("max_nodes", 257, dsk.DSK_ERR_PARAM), ("max_path", 0, dsk.DSK_ERR_PARAM), ("max_path", 21, dsk.DSK_ERR_PARAM),
             ("len_new", FAKE, dsk.DSK_ERR_PARAM), ("len_new", FAKE + 4, dsk.DSK_ERR_PARAM),
             ("token_ids", FAKE - 4 * 999, dsk.DSK_ERR_PARAM), ("target_ids", 4 * FAKE + 4 * 999, dsk.DSK_ERR_PARAM),
             ("k_stride_layer", 0, dsk.DSK_ERR_SHAPE),
             ("vd_stride_layer", 4, dsk.DSK_ERR_ALIGN), ("k_stride_tok", 64, dsk.DSK_ERR_SHAPE),
             ("v_stride_head", 0, dsk.DSK_ERR_SHAPE), ("Kd", FAKE + 8, dsk.DSK_ERR_ALIGN), ("V", FAKE + 8, dsk.DSK_ERR_ALIGN)]
    cases += [(f, None, dsk.DSK_ERR_NULL) for f in ("seq_row0", "seq_len", "cu_new", "parent", "draft_ids", "target_ids", "K",
                                                    "V", "Kd", "Vd", "path", "n_accepted", "len_new", "next_id")]
    _refused(dsk.dsk_accept_draft, lambda: _accept(dsk), cases)
    a = _accept(dsk)
    a.K = a.V = None                                             # the nodes' own buffers without a cache to move them to
    assert dsk.dsk_accept_draft(a, 0, check=False) == dsk.DSK_ERR_NULL


def test_helpers_refuse_tensors_that_are_not_on_the_gpu(dsk):
    import torch
    i = torch.zeros(4, dtype=torch.int32)
    X = torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    for made in (dsk.make_step_plan(seq_row0=i, seq_len=i, n_new=i, max_tokens=3, total_rows=8),
                 dsk.make_norm_rope(X, X, X, X.transpose(0, 1), X.transpose(0, 1)),
                 dsk.make_acceptor(X, X, seq_row0=i, seq_len=i, cu_new=torch.zeros(5, dtype=torch.int32), parent=i,
                                   draft_ids=i, target_ids=i, max_nodes=2)):
        with pytest.raises(AssertionError):
            made.step()
    with pytest.raises(AssertionError):
        dsk.tree_decode_attn(X, X, X, seq_row0=i[:1], seq_len=i[:1], cu_new=i, mask=None, max_nodes=2, max_seqlen=4)
    with pytest.raises(AssertionError):                          # one of them elsewhere
        dsk.make_step_plan(seq_row0=i, seq_len=i.to("meta"), n_new=i, max_tokens=3, total_rows=8)


def test_norm_rope_helper_skips_no_token_in_silence(dsk):
    """Rows of a cache that the call does not see lie above the number of tokens; rows by number need one for every token."""
    import torch
    X = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    row, pos, f = torch.tensor([900, 901, 902], dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.ones(64)
    with pytest.raises(AssertionError):
        dsk.make_norm_rope(X, None, None, None, None, row=row, pos=pos, inv_freq=f)
    assert dsk.make_norm_rope(X, None, None, None, None, row=row, pos=pos, inv_freq=f, total_rows=1000).args.total_rows == 1000
    assert dsk.make_norm_rope(X, None, None, None, None, pos=pos, inv_freq=f).args.total_rows == 3
    cache = torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        dsk.make_norm_rope(X, X, X, cache, cache)
    with pytest.raises(AssertionError):
        dsk.make_norm_rope(None, X, None, cache, None)
    with pytest.raises(AssertionError):
        dsk.make_norm_rope(X, None, None, None, None, total_rows=2)
    assert dsk.make_norm_rope(X, X, X, cache, cache, row=row).args.total_rows == 2


def test_norm_rope_helper_writes_no_row_behind_the_cache(dsk):
    """total_rows bounds the rows that are written, so it is no larger than the shorter of K and V."""
    import torch
    X, row = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    K, V = torch.zeros(2, 9, 128, dtype=torch.bfloat16), torch.zeros(2, 7, 128, dtype=torch.bfloat16)
    for k, v, most in ((X, X, 7), (X, None, 9)):
        assert dsk.make_norm_rope(X, k, v, K, None if v is None else V, row=row, total_rows=most).args.total_rows == most
        with pytest.raises(AssertionError):
            dsk.make_norm_rope(X, k, v, K, None if v is None else V, row=row, total_rows=most + 1)


def test_a_kept_tree_attention_is_called_on_the_device_of_its_tensors(dsk, monkeypatch):
    """As the other kept calls: refused where the tensors are not on the GPU, otherwise with that device as the current one."""
    import contextlib

    import torch
    i, X = torch.zeros(3, dtype=torch.int32), torch.zeros(2, 8, 128, dtype=torch.bfloat16)
    kept = dsk.make_tree_attn_args(X, X, X, seq_row0=i[:1], seq_len=i[:1], cu_new=i[:2], mask=None, max_nodes=2, max_seqlen=4)
    with pytest.raises(AssertionError):
        kept.step()

    class Elsewhere:
        device = torch.device("cuda", 1)

    b, order = dsk.binding, []

    @contextlib.contextmanager
    def on(device):
        order.append(device.index)
        yield
        order.append(0)
    monkeypatch.setattr(b, "dsk_tree_decode_attn", lambda args, stream, check: order.append((args is kept.args, stream, check)) or 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", on)
    kept.lse = Elsewhere()
    assert kept.step(5, check=False) == 0 and order == [1, (True, 5, False), 0]


def test_tree_attention_refuses_more_slots_than_it_counts(dsk):
    """Slots and a part's of them are added up in 32 bits."""
    for k, ok in ((0x7FFF0000, True), (0x7FFF0001, False), (2 ** 31 - 1, False)):
        a = _tree(dsk)
        a.k = k
        assert (dsk.dsk_tree_attn_workspace_bytes(a) > 0) == ok
        a.workspace_bytes = 0
        assert dsk.dsk_tree_decode_attn(a, 0, check=False) == (dsk.DSK_ERR_WORKSPACE if ok else dsk.DSK_ERR_PARAM)


def test_acceptor_helper_drops_no_argument(dsk):
    """K without V, the nodes' own buffers without a cache, and more rows than the cache's are refused; fewer bound the call."""
    import torch
    i, X = torch.zeros(3, dtype=torch.int32), torch.zeros(2, 9, 128, dtype=torch.bfloat16)
    own = torch.zeros(2, 3, 128, dtype=torch.bfloat16)
    kw = dict(seq_row0=i[:1], seq_len=i[:1], cu_new=i[:2], parent=i, draft_ids=i, target_ids=i, max_nodes=3)
    assert dsk.make_acceptor(X, X, Kd=own, Vd=own, **kw).args.total_rows == 9
    assert dsk.make_acceptor(X[None], X[None], total_rows=8, **kw).args.total_rows == 8
    assert dsk.make_acceptor(None, None, total_rows=7, **kw).args.total_rows == 7
    for K, V, more in ((None, None, dict(Kd=own, Vd=own, total_rows=9)), (X, None, {}), (None, X, dict(total_rows=9)),
                       (X, X, dict(Kd=own)), (X, X, dict(total_rows=10)), (None, None, {})):
        with pytest.raises(AssertionError):
            dsk.make_acceptor(K, V, **more, **kw)


def test_tree_attention_workspace_does_not_shrink_as_the_cache_grows(dsk):
    """A workspace for the longest cache serves every shorter one: heads, trees and batches of all kernels, bounds around the cache's
    rows a sequence, where its sequences count as of one length below and as ragged above."""
    lengths = sorted(set(range(0, 6000, 29)) | set(range(6000, 300_000, 1777)) | {2 ** e + d for e in range(5, 30) for d in (-17, 0, 1)}
                     | {0x7FFF0000})
    for B, Hq, Hkv, nodes, rows in ((1, 32, 8, 64, 2 ** 17), (1, 32, 8, 16, 2 ** 17), (8, 32, 8, 13, 400_000), (8, 32, 8, 13, 2 ** 19),
                                    (3, 5, 1, 9, 100_000), (1, 8, 1, 256, 2 ** 21), (64, 32, 8, 4, 2 ** 18), (4, 40, 40, 16, 2 ** 17),
                                    (2, 8, 2, 33, 0), (300, 32, 8, 40, 2 ** 20), (5, 32, 8, 75, 70_000), (65535, 8, 8, 256, 2 ** 31 - 1)):
        a = _tree(dsk)
        a.sel_start = a.sel_len = a.sel_count = None
        a.B, a.Hq, a.Hkv, a.max_nodes, a.mask_words, a.total_rows = B, Hq, Hkv, nodes, 8, rows
        need = 0
        for L in lengths:
            a.max_seqlen = L
            got = dsk.dsk_tree_attn_workspace_bytes(a)
            assert got >= max(need, 256), (B, Hq, Hkv, nodes, rows, L)
            need = got
        assert need <= 256 + a.n_tokens * Hq * 128 * 520 + 512   # 128 parts of a row at most, (m, l) and 128 channels each
