"""relserve_logprobs against plain 64-bit arithmetic on the same logits, through the C-ABI binding.

Tolerances count roundings of fp32 (U = 2^-24 of the value): of x - m one; Z is a sum of positive terms, a thread's share one behind the other and a
tree of the rest, each term an exponential whose argument is rounded twice.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
GUARD = 3


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


def _call(rs, logits, ids=None, n_top=0, scratch=True, stream=None):
    """(logprobs, entropy, top_ids, top_logprobs), with rows behind the last one left as they were."""
    t, v = logits.shape
    full = {"lp": torch.full((t + GUARD, 0 if ids is None else ids.shape[1]), 5.0, device="cuda"), "h": torch.full((t + GUARD,), 5.0, device="cuda"),
            "id": torch.full((t + GUARD, n_top), 77, dtype=torch.int32, device="cuda"), "tlp": torch.full((t + GUARD, n_top), 5.0, device="cuda")}
    need = rs.relserve_logprobs_workspace_bytes(t, v, n_top)
    ws = torch.full((max(256, need),), 255, dtype=torch.uint8, device="cuda") if scratch else None
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())   # the fills above too
    rs.relserve_logprobs(logits, ids, None if ids is None else full["lp"][:t], full["h"][:t], full["id"][:t] if n_top else None,
                         full["tlp"][:t] if n_top else None, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for name, f in full.items():
        assert bool((f[t:] == (77 if name == "id" else 5.0)).all()), name
    return full["lp"][:t].cpu().double(), full["h"][:t].cpu().double(), full["id"][:t].cpu(), full["tlp"][:t].cpu().double()


def _check(rs, logits, ids, n_top, what):
    print(f"[case] logprobs {what}", flush=True)
    x = logits.cpu().double()
    t, v = x.shape
    # rows without a distribution: a NaN, an infinity, nothing above -infinity
    sound = (torch.isfinite(x) | (x == -float("inf"))).all(1) & (x > -float("inf")).any(1)
    m = x.masked_fill(torch.isnan(x), -float("inf")).amax(1, keepdim=True)
    # the largest term apart, as 1 + 1e-20 is 1 in 64 bits too: a row with one entry at 0 and 59 at -50 has an entropy of 51 * 59 e^-50, of which
    # log(Z) itself would lose a fifty-first
    d, largest = x - m, x.masked_fill(torch.isnan(x), -float("inf")).argmax(1, keepdim=True)
    e = torch.exp(d)
    log_z = torch.log1p(e.scatter(1, largest, 0.0).sum(1, keepdim=True))
    p = d - log_z
    entropy = (log_z - (torch.where(e > 0, d, torch.zeros_like(d)) * e).sum(1, keepdim=True) / e.sum(1, keepdim=True)).squeeze(1)
    # Z: v / 256 terms one behind the other, 16 merges of at most 3 roundings and an exponential, each term's exponential 2 U and 2 |x - m| U of its
    # argument; a term e^d is off by (2 + 2 |d|) e^d <= 4 e^(d / 2) .. of which all together are no more than the chain's share: doubled
    z = 2 * (v / 256 + 64)
    for scratch in (True, False):
        lp, h, top, tlp = _call(rs, logits, ids, n_top, scratch)
        if ids is not None:
            at = ids.cpu().long()
            valid = (at >= 0) & (at < v)
            want = torch.where(valid, p.gather(1, at.clamp(0, v - 1)), torch.full_like(lp, float("nan")))
            want[~sound] = float("nan")
            assert torch.equal(torch.isnan(lp), torch.isnan(want)), what
            low = want == -float("inf")
            assert torch.equal(low, lp == -float("inf"))
            ok = ~torch.isnan(want) & ~low
            d = (x.gather(1, at.clamp(0, v - 1)) - m)[ok].abs()
            lz = -(p.amax(1, keepdim=True)).expand_as(want)[ok]
            assert bool(((lp - want)[ok].abs() <= U * (2 * d + (z + 8) * lz.clamp(max=1.0) + 4 * lz)).all()), f"{what}: a log probability is off by {(lp - want)[ok].abs().max()}"
        assert torch.equal(torch.isnan(h), ~sound), what
        # both terms of H are positive: sums' errors as Z's
        assert bool(((h - entropy).abs()[sound] <= U * (2 * z + 16) * entropy[sound].clamp(min=1e-30)).all()), f"{what}: entropy {(h - entropy).abs()[sound].max()}"
        if n_top:
            for r in range(t):
                num = (~torch.isnan(x[r])).nonzero().flatten()
                order = num[torch.sort(x[r][num], descending=True, stable=True).indices][:n_top]
                want_ids = torch.full((n_top,), -1, dtype=torch.int32)
                want_ids[:len(order)] = order.int()
                assert torch.equal(top[r], want_ids), f"{what}: row {r} {top[r].tolist()} for {want_ids.tolist()}"
                if not sound[r]:
                    assert bool(torch.isnan(tlp[r]).all())
                    continue
                assert bool((tlp[r, len(order):] == -float("inf")).all())
                w = p[r, order]
                fine = w > -float("inf")
                assert torch.equal(tlp[r, :len(order)] == -float("inf"), ~fine)
                lz = float(-p[r].max())
                tol = U * (2 * (x[r, order] - m[r]).abs() + (z + 8) * min(lz, 1.0) + 4 * lz)
                assert bool(((tlp[r, :len(order)] - w).abs()[fine] <= tol[fine]).all()), what


def _logits(seed, t, v, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(t, v, generator=g, device="cuda") * 2
    x += torch.randn(t, v, generator=g, device="cuda").clamp(min=2.5) * torch.rand(t, 1, generator=g, device="cuda") * 6
    return x.to(dtype), torch.randint(0, v, (t, 3), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("t,v,top", [(1, 1, 1), (2, 5, 32), (3, 100, 0), (7, 1000, 5), (1, 8192, 20), (2, 8193, 32), (24, 32000, 5), (5, 50257, 20),
                                     (1, 152065, 32), (300, 4097, 1), (600, 16387, 7), (1, 600001, 32), (70, 31999, 9)])
def test_sizes(rs, t, v, top, dtype):
    x, ids = _logits(t * 3 + v, t, v, dtype)
    ids[-1, -1] = v
    ids[0, 0] = -1
    _check(rs, x, ids, top, f"{t} x {v} top {top} {dtype}")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("v,times", [(60, 1), (9001, 1), (40000, 1), (20000, 5)])
def test_rows_that_are_hard(rs, v, times, dtype):
    inf, nan = float("inf"), float("nan")
    x, _ = _logits(v, 16, v, torch.float32)
    x[0] = 0.0                                                       # all alike
    x[1] = torch.arange(v, device="cuda") * 0.25                     # rising: every chunk has new ones
    x[2] = -torch.arange(v, device="cuda") * 0.25
    x[3] = -inf
    x[4, 1:] = -inf                                                  # one entry left
    x[5, ::2] = -inf
    x[6, v // 2] = nan
    x[7, v - 1] = inf
    x[8] = nan
    x[9, :] = -inf
    x[9, v - 3:] = torch.tensor([1.0, -inf, 1.0], device="cuda")
    x[10] = -50.0                                                    # nearly sure
    x[10, v // 3] = 0.0
    x[11, :] = torch.where(torch.arange(v, device="cuda") % 2 == 0, 0.0, -0.0)
    x[12] = 3e38
    x[12, 5] = -3e38
    x[13] = -3e38                                                    # masks of the type's lowest value
    x[13, 7] = 1.0
    x[14, :32] = 60.0                                                # all alternatives in one thread's reach, and ties behind them
    x[15, :] = torch.where(torch.arange(v, device="cuda") % 1024 < 4, 9.0, -1.0)
    ids = torch.arange(16 * 4, device="cuda", dtype=torch.int32).view(16, 4) % v
    x[8, v // 2:] = -inf                                             # no number above -infinity, NaN ahead of them
    _check(rs, x.to(dtype).repeat(times, 1), ids.repeat(times, 1), 20, f"hard rows of {v}")


def test_columns_behind_the_vocabulary_are_not_read(rs):
    for dtype in (torch.float32, torch.bfloat16):
        wide, ids = _logits(4, 9, 5008, dtype)
        wide[:, 5001:] = float("nan")
        _check(rs, wide[:, :5001], ids % 5001, 8, "the first columns of a wider matrix")


def test_a_nearly_sure_row_keeps_its_digits(rs):
    x = torch.full((1, 2000), -40.0, device="cuda")
    x[0, 9] = -20.0
    lp, h, _, _ = _call(rs, x, torch.tensor([[9]], dtype=torch.int32, device="cuda"))
    want = -np.log1p(1999 * np.exp(-20.0))
    assert abs(float(lp) - want) <= 100 * U * abs(want)
    p = np.exp(-20.0)
    assert abs(float(h) - (-want + 1999 * 20.0 * p / (1 + 1999 * p))) <= 100 * U * float(h)


def test_nothing_asked_but_the_entropy(rs):
    x, _ = _logits(8, 4, 300, torch.float32)
    _check(rs, x, None, 0, "entropy alone")


def test_another_stream_and_the_same_bits(rs):
    x, ids = _logits(9, 3, 70000, torch.float32)
    want = _call(rs, x, ids, 10)
    for got in (_call(rs, x, ids, 10), _call(rs, x, ids, 10, stream=torch.cuda.Stream())):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_the_first_alternative_is_the_greedy_token(rs):
    x, _ = _logits(11, 40, 32000, torch.float32)
    token = torch.empty(40, dtype=torch.int32, device="cuda")
    rs.relserve_greedy_sample(x, token)
    assert torch.equal(_call(rs, x, None, 1)[2][:, 0], token.cpu())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("v,times", [(8192 * 3 + 2049, 90), (8192 * 18 + 2047, 1), (8192 * 33 + 1, 1)])
def test_long_rows_that_are_hard(rs, v, times, dtype):
    """Several chunks of a row one behind the other: where the largest values lie, how large they are, and how many are alike."""
    at = torch.arange(v, device="cuda")
    x, ids = _logits(v, 12, v, torch.float32)
    x[0] = at * 1e-4                                                 # every chunk reaches the largest value so far
    x[1] = at * -1e-4                                                # none does
    x[2] += 1e4                                                      # the largest value's product with log2 e lacks digits
    x[3] -= 1.6e4
    x[4] += 3e4                                                      # beyond what the plain pass takes
    x[5, 8192:16384] = -float("inf")                                 # a chunk without a number
    x[6, :-1] = -float("inf")
    x[7, 100:8000] = float("inf")                                    # no distribution, alternatives all the same
    x[8] = torch.where(at % 97 == 3, 12.0, 0.0)                      # the bound's value in more stretches than are dealt out
    x[9] = torch.where(at % 8192 < 8, 7.5, -3.0)                     # in a thread or two, in every chunk
    x[10] = 1e4 - (at + 1) * 2.0 ** -10                              # one step of fp32 below the largest value
    x[10, 0] = 1e4
    x[11, v - 1] = 40.0
    x[11, 9000] = float("nan")
    _check(rs, x.to(dtype).repeat(times, 1), ids.repeat(times, 1), 13, f"long hard rows of {v}")
