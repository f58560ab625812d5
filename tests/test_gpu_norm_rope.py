"""dsk_qk_norm_rope against the formula in 64 bits.  A value is rounded to bf16 once (half a step: 2^-8 of it) after some ten
operations in fp32 on terms that are as large as the two channels of its pair (2^-24 each, cos and sin to 2^-22):
|got - want| <= 2^-8 |want| + 2^-19 (|a| + |b|)."""
import pytest
import torch

from step_testutil import D, i32, rope_reference

pytestmark = pytest.mark.gpu


def _dsk():
    import paper_2602_03184_amd as dsk
    return dsk


def _close(got, want, size):
    got = got.double().cpu()
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * size).all())


def _inputs(n, Hq, Hkv, seed=0, wide=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(n, Hq + 2 * Hkv, D + wide, generator=g, device="cuda").mul_(3.0).bfloat16()[..., :D]
    w = [1.0 + 0.3 * torch.randn(D, generator=g, device="cuda") for _ in range(2)]
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], w[0], w[1], g


def _freq(rot, theta=10000.0):
    return (theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)).float()


@pytest.mark.parametrize("n, Hq, Hkv", [(1, 1, 1), (1, 32, 8), (3, 5, 1), (17, 28, 4), (130, 8, 8), (1025, 6, 2)])
@pytest.mark.parametrize("rot, inter", [(128, False), (128, True), (96, False), (64, True), (32, False), (16, False), (16, True)])
@pytest.mark.parametrize("norm", [True, False])
def test_against_the_formula(n, Hq, Hkv, rot, inter, norm):
    dsk = _dsk()
    q, k, v, wq, wk, g = _inputs(n, Hq, Hkv, wide=8)
    rows = n + 7
    row = torch.randperm(rows, generator=g, device="cuda")[:n].int()
    pos = torch.randint(0, 131072, (n,), generator=g, device="cuda", dtype=torch.int32)
    K = torch.full((Hkv, rows, D), 5.0, dtype=torch.bfloat16, device="cuda")
    V = torch.full((rows, Hkv, D + 16), 5.0, dtype=torch.bfloat16, device="cuda")[..., :D].transpose(0, 1)
    f = _freq(rot)
    r = dsk.make_norm_rope(q, k, v, K, V, pos=pos, row=row, q_weight=wq if norm else None, k_weight=wk if norm else None,
                           eps=1e-5, inv_freq=f, interleaved=inter)
    r.step()
    torch.cuda.synchronize()
    _close(r.q_out, *rope_reference(q, wq if norm else None, 1e-5, pos, f, inter))
    at = row.long()
    _close(K[:, at].transpose(0, 1), *rope_reference(k, wk if norm else None, 1e-5, pos, f, inter))
    assert torch.equal(V[:, at].transpose(0, 1), v)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert bool((K[:, rest] == 5.0).all()) and bool((V[:, rest] == 5.0).all())


def test_far_positions_and_the_first():
    """Angles of up to 2^31 radians: whole turns are taken off in 64 bits."""
    dsk = _dsk()
    pos = i32([0, 1, 65535, 131071, 2 ** 24 + 1, 2 ** 31 - 1])
    q, k, v, wq, wk, _ = _inputs(6, 4, 2)
    K, V = torch.zeros(2, 6, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 6, D, dtype=torch.bfloat16, device="cuda")
    f = _freq(128)
    r = dsk.make_norm_rope(q, k, v, K, V, pos=pos, inv_freq=f)
    r.step()
    torch.cuda.synchronize()
    _close(r.q_out, *rope_reference(q, None, 0, pos, f, False))
    _close(K.transpose(0, 1), *rope_reference(k, None, 0, pos, f, False))
    assert torch.equal(r.q_out[0], q[0]) and torch.equal(V.transpose(0, 1), v)


@pytest.mark.parametrize("weights", [(True, False), (False, True)])
def test_one_norm_only_and_no_rotation(weights):
    dsk = _dsk()
    q, k, v, wq, wk, _ = _inputs(9, 3, 3)
    wq, wk = (w if on else None for w, on in zip((wq, wk), weights))
    K, V = torch.zeros(3, 9, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 9, D, dtype=torch.bfloat16, device="cuda")
    r = dsk.make_norm_rope(q, k, v, K, V, q_weight=wq, k_weight=wk, eps=0.5)
    r.step()
    torch.cuda.synchronize()
    _close(r.q_out, *rope_reference(q, wq, 0.5, None, None, False))
    _close(K.transpose(0, 1), *rope_reference(k, wk, 0.5, None, None, False))
    assert torch.equal(V.transpose(0, 1), v)


@pytest.mark.parametrize("which", ["q", "k", "kv"])
def test_parts_of_the_inputs(which):
    dsk = _dsk()
    q, k, v, wq, wk, _ = _inputs(20, 7, 2)
    pos, f = torch.arange(20, dtype=torch.int32, device="cuda"), _freq(64)
    K, V = torch.zeros(2, 20, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 20, D, dtype=torch.bfloat16, device="cuda")
    r = dsk.make_norm_rope(q if which == "q" else None, k if "k" in which else None, v if "v" in which else None,
                           K if "k" in which else None, V if "v" in which else None, pos=pos, q_weight=wq, k_weight=wk, inv_freq=f)
    r.step()
    torch.cuda.synchronize()
    if which == "q":
        _close(r.q_out, *rope_reference(q, wq, 1e-6, pos, f, False))
    else:
        assert r.q_out is None
        _close(K.transpose(0, 1), *rope_reference(k, wk, 1e-6, pos, f, False))
        assert torch.equal(V.transpose(0, 1), v if "v" in which else torch.zeros_like(v))


def test_skipped_tokens_leave_everything_as_it_was():
    dsk = _dsk()
    q, k, v, wq, wk, _ = _inputs(6, 4, 2)
    row = i32([3, -1, 0, 8, 7, 2 ** 31 - 1])                     # of 8 rows
    K, V = (torch.full((2, 8, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.full((6, 4, D), 5.0, dtype=torch.bfloat16, device="cuda")
    pos, f = i32([4, 5, 6, 7, 8, 9]), _freq(128)
    dsk.make_norm_rope(q, k, v, K, V, pos=pos, row=row, q_weight=wq, k_weight=wk, inv_freq=f, q_out=out).step()
    torch.cuda.synchronize()
    kept = torch.tensor([0, 2, 4], device="cuda")
    w, size = rope_reference(q, wq, 1e-6, pos, f, False)
    _close(out[kept], w[kept.cpu()], size[kept.cpu()])
    assert bool((out[torch.tensor([1, 3, 5], device="cuda")] == 5.0).all())
    assert torch.equal(V[:, row[kept].long()].transpose(0, 1), v[kept])
    rest = torch.tensor([1, 2, 4, 5, 6], device="cuda")
    assert bool((K[:, rest] == 5.0).all()) and bool((V[:, rest] == 5.0).all())


def test_in_place_queries_and_another_stream():
    dsk = _dsk()
    q, _, _, wq, _, _ = _inputs(50, 9, 1)
    mine = q.contiguous()
    pos, f = torch.arange(50, dtype=torch.int32, device="cuda") * 1000, _freq(128)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    dsk.make_norm_rope(mine, None, None, None, None, pos=pos, q_weight=wq, inv_freq=f, q_out=mine).step(st)
    st.synchronize()
    _close(mine, *rope_reference(q, wq, 1e-6, pos, f, False))


def test_values_that_are_not_finite_stay_in_their_row():
    """A NaN or an infinity makes its own head's row what it makes it, and no other row."""
    dsk = _dsk()
    q, k, v, wq, wk, _ = _inputs(4, 4, 2)
    q = q.clone()
    want, size = rope_reference(q, wq, 1e-6, i32([1, 2, 3, 4]), _freq(128), False)
    q[1, 2, 5], q[2, 0, 127] = float("nan"), float("inf")
    r = dsk.make_norm_rope(q, None, None, None, None, pos=i32([1, 2, 3, 4]), q_weight=wq, inv_freq=_freq(128))
    r.step()
    torch.cuda.synchronize()
    hit = torch.zeros(4, 4, dtype=torch.bool)
    hit[1, 2] = hit[2, 0] = True
    assert bool(r.q_out.cpu()[hit].isnan().any(-1).all())
    _close(r.q_out.cpu()[~hit], want[~hit], size[~hit])


def test_rows_and_tokens_beyond_32_bits():
    """Tokens, results and cache rows of which the last lie more than 2^31 channels behind the first."""
    dsk = _dsk()
    n, step = 3, 1 << 30
    x = torch.empty(2 * step + 8 * D, dtype=torch.bfloat16, device="cuda").as_strided((n, 8, D), (step, D, 1))
    x.copy_(torch.randn(n, 8, D, device="cuda") * 3)
    cache = torch.empty(225_000, 80, D, dtype=torch.bfloat16, device="cuda")
    K, V = cache[:, 40:42].transpose(0, 1), cache[:, 78:80].transpose(0, 1)
    pos, row, f = i32([5, 6, 7]), i32([224_999, 17, 224_000]), _freq(128)
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:8]
    r = dsk.make_norm_rope(q, k, v, K, V, pos=pos, row=row, inv_freq=f)
    r.step()
    torch.cuda.synchronize()
    _close(r.q_out, *rope_reference(q, None, 0, pos, f, False))
    _close(K[:, row.long()].transpose(0, 1), *rope_reference(k, None, 0, pos, f, False))
    assert torch.equal(V[:, row.long()].transpose(0, 1), v)
    del x, cache, K, V, q, k, v
    one = torch.randn(1, 128, D, device="cuda").bfloat16()
    many = one.expand(132_000, 128, D)                           # 2^31 channels and more of results
    assert many.numel() > 2 ** 31
    pos = torch.full((132_000,), 9, dtype=torch.int32, device="cuda")
    r = dsk.make_norm_rope(many, None, None, None, None, pos=pos, inv_freq=f, total_rows=132_000)
    r.step()
    torch.cuda.synchronize()
    _close(r.q_out[:1], *rope_reference(one, None, 0, pos[:1], f, False))
    assert all(torch.equal(r.q_out[t], r.q_out[0]) for t in (1, 65_535, 131_072, 131_999))
    torch.cuda.empty_cache()


def test_no_token_at_all():
    dsk = _dsk()
    q, k, v, wq, wk, _ = _inputs(1, 4, 2)
    K, V = (torch.full((2, 5, D), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    r = dsk.make_norm_rope(q[:0], k[:0], v[:0], K, V, pos=i32([]), q_weight=wq, k_weight=wk, inv_freq=_freq(128))
    r.step()
    torch.cuda.synchronize()
    assert r.q_out.shape == (0, 4, D) and bool((K == 5.0).all()) and bool((V == 5.0).all())


@pytest.mark.parametrize("rot, inter", [(0, False), (32, False), (32, True), (96, False), (96, True), (112, False), (112, True)])
def test_channels_that_are_not_rotated_are_copied_bit_for_bit(rot, inter):
    """Without a norm, whatever they hold: infinities, NaNs of any payload and sign, zeros of both signs, subnormal numbers."""
    dsk = _dsk()
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randint(-2 ** 15, 2 ** 15, (9, 8, D), generator=g, device="cuda", dtype=torch.int16)
    x[:, :, rot:][torch.rand(9, 8, D - rot, generator=g, device="cuda") < 0.3] = 0x7F80
    x[:, :, rot:][torch.rand(9, 8, D - rot, generator=g, device="cuda") < 0.1] = -0x8000
    x[:, :, :rot] = torch.randn(9, 8, rot, generator=g, device="cuda").bfloat16().view(torch.int16)
    x = x.view(torch.bfloat16)
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    K, V = (torch.zeros(2, 9, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos, f = torch.arange(9, dtype=torch.int32, device="cuda") * 77, _freq(rot) if rot else None
    r = dsk.make_norm_rope(q, k, v, K, V, pos=pos, inv_freq=f, interleaved=inter)
    r.step()
    torch.cuda.synchronize()
    for got, was in ((r.q_out, q), (K.transpose(0, 1), k)):
        assert torch.equal(got[..., rot:].contiguous().view(torch.int16), was[..., rot:].contiguous().view(torch.int16))
        if rot:
            want, size = rope_reference(was[..., :rot].contiguous(), None, 0, pos, f, inter)
            _close(got[..., :rot], want, size)
    assert torch.equal(V.transpose(0, 1).contiguous().view(torch.int16), v.contiguous().view(torch.int16))


@pytest.mark.parametrize("inter", [False, True])
def test_an_infinity_that_is_not_rotated_stays_one_behind_a_norm(inter):
    """x / sqrt(mean of squares + eps) of a row with an infinity is 0 in its finite channels and NaN in that one; a weight of the
    other tensor alone leaves the row as it is."""
    dsk = _dsk()
    q, k, v, wq, wk, _ = _inputs(3, 4, 2)
    q, k = q.clone(), k.clone()
    q[1, 2, 100], k[1, 1, 100] = float("inf"), float("inf")
    K, V = (torch.zeros(2, 3, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    r = dsk.make_norm_rope(q, k, v, K, V, pos=i32([1, 2, 3]), q_weight=wq, inv_freq=_freq(32), interleaved=inter)
    r.step()
    torch.cuda.synchronize()
    rest = torch.arange(D, device="cuda") != 100
    assert bool(r.q_out[1, 2, 100].isnan()) and bool((r.q_out[1, 2, rest] == 0).all())
    assert torch.equal(K.transpose(0, 1)[..., 32:], k[..., 32:])
