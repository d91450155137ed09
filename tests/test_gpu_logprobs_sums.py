"""Sums of long rows of logits in relserve_logprobs, whose error has to go with the row's chunks and not with all values that a thread meets: rows of few
different values, whose largest one stands in every chunk of every wave, so that equal terms are added in the same place over and over.

Tolerances count roundings of fp32 (U = 2^-24), S of them in a sum relative to it: an exponential 2, its argument d log2 e and the difference 3 |d|, 31
additions in a thread's chunk of 32 values, one for each chunk, and at most 24 behind them (a wave's lanes 6, its workgroup's waves 4, 64 parts 6 and 4, moves).
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


def _check(rs, logits, n_top, scratch, what):
    t, v = logits.shape
    print(f"[case] sums {what} {t} x {v} {logits.dtype} scratch={scratch} top={n_top}", flush=True)
    ids = torch.tensor([0, 1, v - 1], dtype=torch.int32, device="cuda").repeat(t, 1)
    lp, h = torch.empty(t, 3, device="cuda"), torch.empty(t, device="cuda")
    top, tlp = torch.empty(t, n_top, dtype=torch.int32, device="cuda"), torch.empty(t, n_top, device="cuda")
    ws = torch.empty(max(256, rs.relserve_logprobs_workspace_bytes(t, v, n_top)), dtype=torch.uint8, device="cuda") if scratch else None
    rs.relserve_logprobs(logits, ids, lp, h, top if n_top else None, tlp if n_top else None, workspace=ws)
    d = logits.double() - logits.double().amax(1, keepdim=True)
    e = d.exp()
    z, s = e.sum(1), 2 + 3 * float(-d.min()) + 31 + -(-v // 8192) + 24
    lz, mean = z.log(), (-d * e).sum(1) / z
    want = d.gather(1, ids.long()) - lz[:, None]
    tol = U * (s + 4 * lz[:, None] + 2 * want.abs())               # log1p and the last difference beside the sum's
    off = (lp.double() - want).abs()
    assert bool((off <= tol).all()), f"{what}: a log probability is off by {float(off.max() / U):.0f} U of {float(tol.min() / U):.0f}"
    off, tol = (h.double() - (lz + mean)).abs(), U * (s + 4 * lz + (2 * s + 4) * mean + 2 * (lz + mean))
    assert bool((off <= tol).all()), f"{what}: the entropy is off by {float(off.max() / U):.0f} U of {float(tol.min() / U):.0f}"
    if n_top:
        assert bool((top.long() == torch.sort(logits.float(), dim=1, descending=True, stable=True).indices[:, :n_top]).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("v", [1 << 20, 1 << 22])
@pytest.mark.parametrize("n_top", [0, 3])
def test_two_values(rs, v, n_top, dtype):
    at = torch.arange(v, device="cuda")
    low = torch.tensor([-0.75, -1.25, -0.3125, -2.0], device="cuda")[:, None]
    x = torch.where(at % 256 == 0, torch.zeros_like(low), low).to(dtype)
    for scratch in (False, True):
        _check(rs, x, n_top, scratch, "two values")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_nearly_undecided_rows(rs, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = (torch.randint(-4, 1, (3, 1000003), generator=g, device="cuda") * 0.25).to(dtype)
    for scratch in (False, True):
        _check(rs, x, 5, scratch, "five values")


def test_large_logits(rs):
    """Largest values beyond what the pass over smaller chunks takes."""
    at = torch.arange(1 << 20, device="cuda")
    x = torch.where(at % 5000 == 0, 40000.0, 39999.25)[None]
    for scratch in (False, True):
        _check(rs, x, 0, scratch, "large logits")


def test_rising_rows(rs):
    """Every chunk has a larger value than all before it."""
    x = (torch.arange(1 << 20, device="cuda", dtype=torch.float32) * 2.0 ** -21)[None]
    for scratch in (False, True):
        _check(rs, x, 0, scratch, "rising")
