"""The feed-forward block on the int8 operators as a whole, against the block in 64 bits."""
import numpy as np
import pytest
import torch

from tests.test_gpu_i8 import B, _mlp, _mlp_buffers
from tests.test_gpu_i8_layer import _rows64

pytestmark = pytest.mark.gpu


def _block(b, s, quantised):
    """What the block adds to the stream s, in 64 bits on dequantised weights; quantised: both products' inputs through their row quantisers, the
    SwiGLU product through bf16 before its own."""
    x = s * b["w_norm"].double() / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5)
    gate, up = (((_rows64(x) if quantised else x) @ b["gu"].w.double().t()) * b["gu"].w_scale.double()).chunk(2, 1)
    act = gate * torch.sigmoid(gate) * up
    if quantised:
        act = _rows64(act.float().bfloat16().double())
    return (act @ b["down"].w.double().t()) * b["down"].w_scale.double()


@pytest.mark.parametrize("t,h,inner", [(1, 256, 384), (29, 1024, 2816), (150, 512, 1408), (640, 1024, 2816)])
def test_block_is_off_by_its_quantisers_alone(t, h, inner):
    """The kernels and the block with the same quantisers in 64 bits differ where a rounding of fp32 or bf16 takes a code to the next one, a whole step
    for each.  A code is off by step / sqrt(12) on average, so if one in twelve went that way the difference would be as large as what the
    quantisers themselves cost.  Of the norm's codes fewer than 1e-4 can (its quotients are off by some 2^-16 of a step); of the product's, whose
    inputs the norm's few move by a thousandth of a step, about one in a hundred.  So that distance is the bound, with the output's own rounding; it is a
    few per cent of the block's contribution, while a lost term, a wrong scale or an input of another row is of its size."""
    from paper_2601_11546_amd import binding as rs
    print(f"[case] feed-forward block i8 as a whole T={t} H={h} I={inner}", flush=True)
    b = _mlp_buffers(rs, t, h, inner, t + h)
    b["down"].w_scale *= 256.0        # the block's contribution outweighs the stream, whose rounding to bf16 would hide it
    _mlp(rs, b)
    torch.cuda.synchronize()
    s = b["sum"].double()
    assert torch.equal(b["sum"], b["x"] + b["delta"].float())
    with_q, without = _block(b, s, True), _block(b, s, False)
    noise, own, off = (float(v.norm()) for v in (with_q - without, without, b["out"].double() - s - with_q))
    rounding = float(b["out"].double().norm()) * B / np.sqrt(3)
    print(f"[parity] off {off / own:.2e} of the block's contribution, quantisers {noise / own:.2e}, the output's rounding {rounding / own:.2e}", flush=True)
    assert noise <= 0.1 * own and off <= noise + rounding
