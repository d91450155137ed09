"""What the binding refuses of an int8 step's buffers, before anything reaches the library (no GPU needed).

A pool, a workspace or a table of another type or size than the step takes it for would be read and written past its end."""
import types

import pytest
import torch

from paper_2601_11546_amd import workloads as W

SHAPE = W.LayerShape(256, 4, 2, 64, 384)
T, PAGES = 3, 5


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


def _weights():
    s, w = SHAPE, {n: torch.zeros(SHAPE.hidden, dtype=torch.bfloat16) for n in ("w_in_norm", "w_post_norm")}
    for n, (r, k) in {"qkv": (s.qkv_dim, s.hidden), "o": (s.hidden, s.q_dim), "gate_up": (2 * s.mlp_dim, s.hidden), "down": (s.hidden, s.mlp_dim)}.items():
        w["w_" + n], w["s_" + n] = torch.zeros(r, k, dtype=torch.int8), torch.zeros(r)
    return w


def _pool(pages=PAGES, dtype=torch.bfloat16, page_size=SHAPE.page_size, d=64):
    return torch.zeros(pages, page_size, SHAPE.n_kv_heads, d, dtype=dtype)


def _step(rs, k=None, v=None, ws=None):
    x = torch.zeros(T, SHAPE.hidden, dtype=torch.bfloat16)
    rs.relserve_layer_step_i8(types.SimpleNamespace(shape=SHAPE, handle=None), types.SimpleNamespace(T=T, handle=None), _weights(), x, x,
                              _pool() if k is None else k, _pool() if v is None else v, torch.zeros(64, dtype=torch.uint8) if ws is None else ws)


def _qkv(rs, k=None, v=None):
    s, layer = SHAPE, types.SimpleNamespace(shape=SHAPE, handle=None)
    rs.relserve_qkv_rope_append_i8(layer, types.SimpleNamespace(T=T, handle=None), torch.zeros(T, s.hidden, dtype=torch.int8), torch.zeros(T),
                                   torch.zeros(s.qkv_dim, s.hidden, dtype=torch.int8), torch.zeros(s.qkv_dim),
                                   torch.zeros(T, s.q_dim, dtype=torch.bfloat16), _pool() if k is None else k, _pool() if v is None else v)


def _model(rs, k=None, v=None, ws=None):
    model = {"embedding": torch.zeros(8, 256, dtype=torch.bfloat16), "layers": [_weights()], "w_final_norm": torch.zeros(256, dtype=torch.bfloat16),
             "w_lm_head": torch.zeros(8, 256, dtype=torch.bfloat16), "caches": [(_pool() if k is None else k, _pool() if v is None else v)]}
    rs.relserve_model_step(types.SimpleNamespace(shape=SHAPE, handle=None), types.SimpleNamespace(T=T, handle=None), model,
                           torch.zeros(T, dtype=torch.int32), torch.zeros(1, 8), torch.zeros(64, dtype=torch.uint8) if ws is None else ws)


@pytest.mark.parametrize("call", [_step, _qkv, _model])
def test_pools(rs, call):
    for bad in (_pool(dtype=torch.uint8), _pool(dtype=torch.float32), _pool(dtype=torch.float16), _pool(page_size=SHAPE.page_size // 2), _pool(d=32),
                _pool(d=128)[..., ::2]):
        with pytest.raises(ValueError, match="k_pages must"):
            call(rs, k=bad)
        with pytest.raises(ValueError, match="v_pages must"):
            call(rs, v=bad)
    with pytest.raises(ValueError, match="v_pages must"):       # fewer pages than the keys'
        call(rs, v=_pool(pages=PAGES - 1))
    quant = rs.QuantPool(_pool(dtype=torch.uint8), 0.1)
    with pytest.raises(ValueError, match="k_pages must"):
        call(rs, k=rs.QuantPool(_pool(), 0.1), v=quant)
    with pytest.raises(ValueError, match="v_pages must"):
        call(rs, k=quant, v=rs.QuantPool(_pool(d=32, dtype=torch.uint8), 0.1))
    for fine in (_pool(), quant, rs.QuantPool(_pool(dtype=torch.uint8).view(torch.float8_e4m3fn), 0.1)):       # all that is wrong with these is where they lie
        with pytest.raises(ValueError, match="current device"):
            call(rs, k=fine, v=fine)


@pytest.mark.parametrize("call", [_step, _model])
def test_workspaces(rs, call):
    with pytest.raises(ValueError, match="workspace must"):     # every other byte of a buffer is not a buffer of half its size
        call(rs, ws=torch.zeros(128, dtype=torch.uint8)[::2])
    with pytest.raises(ValueError, match="current device"):
        call(rs, ws=torch.zeros(16, dtype=torch.float32))


def test_a_residual_that_the_epilogue_does_not_add(rs):
    a, scale, w, w_scale = torch.zeros(4, 128, dtype=torch.int8), torch.zeros(4), torch.zeros(64, 128, dtype=torch.int8), torch.zeros(64)
    for epilogue, n in ((0, 64), (3, 32)):
        for dtype in (torch.float32, torch.bfloat16):
            with pytest.raises(ValueError, match="residual"):
                rs.relserve_linear_i8(a, scale, w, w_scale, epilogue, torch.zeros(4, 64, dtype=dtype), torch.zeros(4, n, dtype=torch.bfloat16))
