"""What the block-scaled projections' entry points and relserve_logprobs refuse, and what they answer without a device (no GPU needed: a refused
call launches nothing)."""
import ctypes as C

import pytest
import torch

NULL, BAD, WORKSPACE, TOO_LARGE = -1, -14, -9, -12
P = C.c_void_p(1 << 20)      # an aligned address that a refused call does not touch
ODD = C.c_void_p((1 << 20) + 8)
ODDER = C.c_void_p((1 << 20) + 2)


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


def _quantise(rs, inp=P, rows=4, n=128, block_rows=1, codes=P, scales=P):
    return rs._lib.relserve_quantise_f8b(inp, rows, n, block_rows, codes, scales, None)


def _norm(rs, x=P, f32=0, delta=None, w=P, rows=4, n=128, total=None, codes=P, scales=P):
    return rs._lib.relserve_add_rmsnorm_f8b(x, f32, delta, w, 1e-5, rows, n, total, codes, scales, None)


def _linear(rs, a=P, a_scale=P, w=P, w_scale=P, t=4, n=64, k=128, epilogue=0, residual=None, out=P, packed=0, ws=None, ws_bytes=0):
    return rs._lib.relserve_linear_f8b(a, a_scale, w, w_scale, t, n, k, epilogue, residual, out, packed, ws, ws_bytes, None)


def _logprobs(rs, logits=P, f32=1, rows=4, vocab=100, pitch=100, ids=P, n_ids=1, out=P, entropy=P, n_top=2, top_ids=P, top=P, ws=None, ws_bytes=0):
    return rs._lib.relserve_logprobs(logits, f32, rows, vocab, pitch, ids, n_ids, out, entropy, n_top, top_ids, top, ws, ws_bytes, None)


def test_rows(rs):
    for bad in ({"rows": -1}, {"n": 0}, {"n": -128}, {"n": 64}, {"n": 200}, {"block_rows": 0}, {"block_rows": 64}, {"block_rows": 129}):
        assert _quantise(rs, **bad) == BAD, bad
    assert _quantise(rs, rows=0, inp=None) == 0 and _norm(rs, rows=0, x=None) == 0
    assert _quantise(rs, rows=(1 << 30) + 1) == TOO_LARGE and _quantise(rs, n=(1 << 22) + 128) == TOO_LARGE
    assert _norm(rs, rows=2147483647) == TOO_LARGE and _norm(rs, n=(1 << 22) + 128) == TOO_LARGE
    for name in ("inp", "codes", "scales"):
        assert _quantise(rs, **{name: None}) == NULL
    for name in ("inp", "codes"):
        assert _quantise(rs, **{name: ODD}) == BAD
    assert _quantise(rs, scales=ODDER) == BAD and _norm(rs, scales=ODDER) == BAD
    for bad in ({"rows": -1}, {"n": 0}, {"n": 136}):
        assert _norm(rs, **bad) == BAD, bad
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
    for name in ("a", "w", "out", "residual"):
        assert _linear(rs, **{name: ODD}, epilogue=1) == BAD
    for name in ("a_scale", "w_scale"):
        assert _linear(rs, **{name: ODDER}) == BAD
    assert _linear(rs, t=1 << 24, k=128) == TOO_LARGE and _linear(rs, n=1 << 24, k=128) == TOO_LARGE
    assert _linear(rs, n=(1 << 24) - 128, k=128, packed=1) == TOO_LARGE     # padded to whole blocks of 256 rows


def test_linear_workspace(rs):
    need = rs.relserve_linear_f8b_workspace_bytes(24, 5120)
    assert need > 0 and rs.relserve_linear_f8b_workspace_bytes(5000, 5120) > 0
    assert _linear(rs, t=24, n=5120, ws=P, ws_bytes=need - 1) == WORKSPACE
    assert _linear(rs, t=24, n=5120, ws=C.c_void_p((1 << 20) + 128), ws_bytes=need) == WORKSPACE
    out = C.c_size_t()
    assert rs._lib.relserve_linear_f8b_workspace_bytes(24, 5120, None) == NULL
    assert rs._lib.relserve_linear_f8b_workspace_bytes(-1, 5120, C.byref(out)) == BAD
    assert rs._lib.relserve_linear_f8b_workspace_bytes(24, 0, C.byref(out)) == BAD


def test_logprobs(rs):
    for bad in ({"rows": -1}, {"vocab": 0}, {"pitch": 99}, {"n_ids": -1}, {"n_top": -1}, {"n_top": 33}):
        assert _logprobs(rs, **bad) == BAD, bad
    assert _logprobs(rs, rows=0, logits=None) == 0
    assert _logprobs(rs, rows=(1 << 22) + 1) == TOO_LARGE and _logprobs(rs, vocab=(1 << 24) + 1, pitch=1 << 25) == TOO_LARGE
    for name in ("logits", "ids", "out", "top_ids", "top"):
        assert _logprobs(rs, **{name: None}) == NULL
    for name in ("logits", "ids", "out", "entropy", "top_ids", "top"):
        assert _logprobs(rs, **{name: ODDER}) == BAD
    assert _logprobs(rs, logits=C.c_void_p((1 << 20) + 1), f32=0) == BAD
    need = rs.relserve_logprobs_workspace_bytes(1, 100000, 20)
    assert need > 0
    assert _logprobs(rs, rows=1, vocab=100000, pitch=100000, n_top=20, ws=P, ws_bytes=need - 1) == WORKSPACE
    assert _logprobs(rs, rows=1, vocab=100000, pitch=100000, n_top=20, ws=C.c_void_p((1 << 20) + 128), ws_bytes=need) == WORKSPACE
    out = C.c_size_t()
    assert rs._lib.relserve_logprobs_workspace_bytes(1, 100, 1, None) == NULL
    for rows, vocab, top in ((-1, 100, 1), (1, 0, 1), (1, 100, -1), (1, 100, 33)):
        assert rs._lib.relserve_logprobs_workspace_bytes(rows, vocab, top, C.byref(out)) == BAD


def test_binding_takes_matrices_of_the_right_types(rs):
    x, w = torch.zeros(4, 256, dtype=torch.bfloat16), torch.zeros(256, dtype=torch.bfloat16)
    codes, scales = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(2, 4)
    with pytest.raises(ValueError, match="values"):
        rs.relserve_quantise_f8b(x[:, ::2], torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(1, 4))
    with pytest.raises(ValueError, match="codes"):
        rs.relserve_quantise_f8b(x, codes.to(torch.int8), scales)
    with pytest.raises(ValueError, match="scales"):                 # of tokens they lie block by block
        rs.relserve_quantise_f8b(x, codes, scales.t().contiguous())
    with pytest.raises(ValueError, match="scales"):
        rs.relserve_quantise_f8b(x, codes, scales, block_rows=128)
    for fine in (codes, codes.view(torch.float8_e4m3fn)):           # all that is wrong with these is where they lie
        with pytest.raises(ValueError, match="current device"):
            rs.relserve_quantise_f8b(x, fine, scales)
    with pytest.raises(ValueError, match="delta"):
        rs.relserve_add_rmsnorm_f8b(x, w, 1e-5, codes, scales, delta=x.float())
    with pytest.raises(ValueError, match="sum_out"):
        rs.relserve_add_rmsnorm_f8b(x, w, 1e-5, codes, scales, sum_out=x.float())
    a, wc, ws = codes, torch.zeros(192, 256, dtype=torch.uint8), torch.zeros(2, 2)
    out = torch.zeros(4, 192, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="w must"):
        rs.relserve_linear_f8b(a, scales, wc.t().contiguous(), ws, 0, None, torch.zeros(4, 256, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="w_scale must"):           # a gate and an up matrix of 96 rows have a block each, a matrix of 192 has two
        rs.relserve_linear_f8b(a, scales, wc, ws[:1], 0, None, out)
    with pytest.raises(ValueError, match="out must"):
        rs.relserve_linear_f8b(a, scales, wc, ws, 1, None, out)
    with pytest.raises(ValueError, match="residual must"):
        rs.relserve_linear_f8b(a, scales, wc, ws, 2, out, out)
    with pytest.raises(ValueError, match="adds no residual"):
        rs.relserve_linear_f8b(a, scales, wc, ws, 0, out, out)
    with pytest.raises(ValueError, match="w must"):                 # packed weights hold whole blocks of 256 rows
        rs.relserve_linear_f8b(a, scales, wc.view(-1), ws, 0, None, out, n=192)
    with pytest.raises(ValueError, match="workspace must"):
        rs.relserve_linear_f8b(a, scales, wc, ws, 0, None, out, workspace=torch.zeros(64, dtype=torch.uint8)[::2])
    logits, ids, lp = torch.zeros(4, 100), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for bad in (logits.t(), logits.half(), logits[:, ::2], logits[:1].expand(4, 100)):
        with pytest.raises(ValueError, match="logits must"):
            rs.relserve_logprobs(bad, ids, lp)
    with pytest.raises(ValueError, match="together"):
        rs.relserve_logprobs(logits, ids)
    with pytest.raises(ValueError, match="together"):
        rs.relserve_logprobs(logits, top_logprobs=lp)
    with pytest.raises(ValueError, match="ids must"):
        rs.relserve_logprobs(logits, ids.long(), lp)
    with pytest.raises(ValueError, match="top_ids must"):
        rs.relserve_logprobs(logits, top_ids=ids[:3], top_logprobs=lp)
    for fine in (logits, logits[:, :50], logits.bfloat16()):
        with pytest.raises(ValueError, match="current device"):
            rs.relserve_logprobs(fine, ids, lp)
