"""What the int8 entry points refuse, and what they answer without a device (no GPU needed: a refused call launches nothing)."""
import ctypes as C

import pytest
import torch

NULL, BAD, WORKSPACE, TOO_LARGE = -1, -14, -9, -12
P = C.c_void_p(1 << 20)      # an aligned address that a refused call does not touch
ODD = C.c_void_p((1 << 20) + 8)


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


def _quantise(rs, inp=P, rows=4, n=64, codes=P, scales=P):
    return rs._lib.relserve_quantise_rows_i8(inp, rows, n, codes, scales, None)


def _norm(rs, x=P, f32=0, delta=None, w=P, rows=4, n=64, total=None, codes=P, scales=P):
    return rs._lib.relserve_add_rmsnorm_i8(x, f32, delta, w, 1e-5, rows, n, total, codes, scales, None)


def _linear(rs, a=P, a_scale=P, w=P, w_scale=P, t=4, n=64, k=128, epilogue=0, residual=None, out=P, packed=0, ws=None, ws_bytes=0):
    return rs._lib.relserve_linear_i8(a, a_scale, w, w_scale, t, n, k, epilogue, residual, out, packed, ws, ws_bytes, None)


def test_rows(rs):
    assert _quantise(rs, rows=-1) == BAD and _quantise(rs, n=0) == BAD and _quantise(rs, n=-8) == BAD and _quantise(rs, n=60) == BAD
    assert _quantise(rs, rows=0, inp=None) == 0
    for name in ("inp", "codes", "scales"):
        assert _quantise(rs, **{name: None}) == NULL
    assert _quantise(rs, inp=ODD) == BAD and _quantise(rs, codes=ODD) == BAD
    assert _norm(rs, rows=-1) == BAD and _norm(rs, n=0) == BAD and _norm(rs, n=4) == BAD
    assert _norm(rs, rows=0, x=None) == 0
    assert _quantise(rs, rows=(1 << 30) + 1) == TOO_LARGE and _norm(rs, rows=2147483647) == TOO_LARGE
    for name in ("x", "w", "codes", "scales"):
        assert _norm(rs, **{name: None}) == NULL
    for name in ("x", "w", "codes", "delta", "total"):
        assert _norm(rs, **{name: ODD}) == BAD


def test_linear(rs):
    for bad in ({"t": -1}, {"n": 0}, {"n": 62}, {"k": 0}, {"k": 64}, {"k": 192}, {"epilogue": -1}, {"epilogue": 4}, {"epilogue": 3, "n": 40}):
        assert _linear(rs, **bad) == BAD, bad
    assert _linear(rs, t=0, a=None) == 0
    for name in ("a", "a_scale", "w", "w_scale", "out"):
        assert _linear(rs, **{name: None}) == NULL
    assert _linear(rs, epilogue=2) == NULL
    for name in ("a", "w", "w_scale", "out", "residual"):
        assert _linear(rs, **{name: ODD}, epilogue=1) == BAD
    # sums of 32 bits, indices of 32 bits
    assert _linear(rs, k=131072) == TOO_LARGE
    assert _linear(rs, t=1 << 24, k=128) == TOO_LARGE and _linear(rs, n=1 << 24, k=128) == TOO_LARGE
    assert _linear(rs, n=(1 << 24) - 128, k=128, packed=1) == TOO_LARGE     # padded to whole blocks of 256 rows


def test_linear_workspace(rs):
    need = rs.relserve_linear_i8_workspace_bytes(24, 5120)
    assert need >= 24 * 5120 * 4 and rs.relserve_linear_i8_workspace_bytes(5000, 5120) > 0
    assert _linear(rs, t=24, n=5120, ws=P, ws_bytes=need - 1) == WORKSPACE
    assert _linear(rs, t=24, n=5120, ws=C.c_void_p((1 << 20) + 128), ws_bytes=need) == WORKSPACE
    out = C.c_size_t()
    assert rs._lib.relserve_linear_i8_workspace_bytes(24, 5120, None) == NULL
    assert rs._lib.relserve_linear_i8_workspace_bytes(-1, 5120, C.byref(out)) == BAD
    assert rs._lib.relserve_linear_i8_workspace_bytes(24, 0, C.byref(out)) == BAD


def test_binding_takes_whole_matrices_of_the_right_types(rs):
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    codes, scales = torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)
    with pytest.raises(ValueError, match="values"):
        rs.relserve_quantise_rows_i8(x[:, ::2], torch.zeros(4, 32, dtype=torch.int8), scales)
    with pytest.raises(ValueError, match="codes"):
        rs.relserve_quantise_rows_i8(x, codes[:3], scales)
    with pytest.raises(ValueError, match="scales"):
        rs.relserve_quantise_rows_i8(x, codes, scales.double())
    with pytest.raises(ValueError, match="current device"):      # host memory
        rs.relserve_quantise_rows_i8(x, codes, scales)
    w = torch.zeros(64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="delta"):
        rs.relserve_add_rmsnorm_i8(x, w, 1e-5, codes, scales, delta=x.float())
    with pytest.raises(ValueError, match="sum_out"):
        rs.relserve_add_rmsnorm_i8(x, w, 1e-5, codes, scales, sum_out=x.float())
    with pytest.raises(ValueError, match="x must"):
        rs.relserve_add_rmsnorm_i8(x.double(), w, 1e-5, codes, scales)
    a, wc, ws = torch.zeros(4, 128, dtype=torch.int8), torch.zeros(64, 128, dtype=torch.int8), torch.zeros(64)
    out = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="w must"):
        rs.relserve_linear_i8(a, scales, wc.t().contiguous(), ws, 0, None, out)
    with pytest.raises(ValueError, match="out must"):
        rs.relserve_linear_i8(a, scales, wc, ws, 1, None, out)
    with pytest.raises(ValueError, match="residual must"):
        rs.relserve_linear_i8(a, scales, wc, ws, 2, out, out)
    with pytest.raises(ValueError, match="w must"):               # packed weights hold whole blocks of 256 rows
        rs.relserve_linear_i8(a, scales, wc.view(-1), ws, 0, None, out, n=64)
