"""The codes of the int8 operators are the nearest integers to value * 127 / m, ties to even, for every row that the entry points take.

Rows of bf16 values, and norms of bf16 streams, have exact codes: there value * 127 / m of the numbers that the kernel divides (values, or
products of two bf16 numbers, which fp32 holds exactly) is either an integer and a half or further from one than a rounding to fp32 reaches:
  |254 v - (2 j + 1) m| is at least 1 in units of the last place of v or m.  With v an integer of at most 255^2 of them, the quotient Q is
  Q / (254 v) > Q 2^-24 away, with m one, 1 / (2 m) > 2^-17; a rounding of Q to 24 bits moves it by at most Q 2^-24, and below 128 by 2^-18.
So the comparisons below are of equal integers."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


def _want(values):
    """The codes of rows given in 64 bits (exact products and, at ties, exact quotients; torch rounds ties to even)."""
    m = values.abs().amax(1, keepdim=True)
    return torch.round(values * 127.0 / torch.where(m > 0, m, torch.ones_like(m))).to(torch.int8)


def _every_value_up_to(top, below, n):
    """[rows, n]: every bf16 magnitude from `below` binades under the row's top (its bit pattern) up to the top, both signs, top first."""
    at = top[:, None] - torch.arange(128 * below, device="cuda")[None]
    at = torch.where(at > 0, at, torch.zeros_like(at))
    bits = torch.cat([at, at + 0x8000, at[:, :1].expand(-1, n - 2 * at.shape[1])], 1)
    return torch.where(bits >= 0x8000, bits - 0x10000, bits).to(torch.int16).view(torch.bfloat16)


@pytest.mark.parametrize("n", [2312, 4104, 33000])
def test_every_quotient_of_two_bf16_values(rs, n):
    """All 128 mantissas of the largest value, at both ends of the exponents and between, against every value within nine binades: among
    them all ties, |v| = m / 2 (63.5) in every row.  The row lengths take a chunk, two and more a thread, and the second read."""
    tops = torch.cat([torch.arange(128, device="cuda") + 128 * e for e in (0, 1, 2, 26, 27, 28, 126, 127, 190, 253, 254)])
    x = _every_value_up_to(tops, 9, n)
    want = _want(x.double())
    ties = (x.double().abs() * 254 / x.double().abs().amax(1, keepdim=True).clamp_min(1e-300)) % 2 == 1
    assert int(ties.sum()) > len(tops)
    codes, scales = torch.full((len(tops), n), 77, dtype=torch.int8, device="cuda"), torch.empty(len(tops), device="cuda")
    print(f"[case] every quotient {len(tops)} x {n}", flush=True)
    rs.relserve_quantise_rows_i8(x, codes, scales)
    torch.cuda.synchronize()
    bad = codes != want
    assert not bool(bad.any()), f"{int(bad.sum())} codes are not the nearest integer, first at {bad.nonzero()[0].tolist()}"


@pytest.mark.parametrize("t,n,delta", [(512, 28672, False), (1030, 512, True), (40, 5120, True), (9, 40000, True), (8300, 8192, True)])
def test_norms_of_bf16_streams(rs, t, n, delta):
    g = torch.Generator(device="cuda")
    g.manual_seed(t + n)
    x = torch.randn(t, n, generator=g, device="cuda")
    x[:, ::61] *= 8.0
    x = x.to(torch.bfloat16)
    w = (1.0 + 0.02 * torch.randn(n, generator=g, device="cuda")).to(torch.bfloat16)
    d = (0.5 * torch.randn(t, n, generator=g, device="cuda")).to(torch.bfloat16) if delta else None
    stream = x if d is None else (x.float() + d.float()).to(torch.bfloat16)
    codes, scales = torch.full((t, n), 77, dtype=torch.int8, device="cuda"), torch.empty(t, device="cuda")
    print(f"[case] codes of a norm {t} x {n} delta={delta}", flush=True)
    rs.relserve_add_rmsnorm_i8(x, w, 1e-5, codes, scales, delta=d)
    torch.cuda.synchronize()
    for rows in range(0, t, 1024):
        bad = codes[rows:rows + 1024] != _want(stream[rows:rows + 1024].double() * w.double())
        assert not bool(bad.any()), f"{int(bad.sum())} codes are not the nearest integer, first at {bad.nonzero()[0].tolist()} of {rows}"


@pytest.mark.parametrize("t,n", [(512, 28672), (2049, 512)])
def test_ties_are_as_frequent_as_ordinary_rows_have_them(rs, t, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    x = torch.randn(t, n, generator=g, device="cuda").to(torch.bfloat16)
    codes, scales = torch.full((t, n), 77, dtype=torch.int8, device="cuda"), torch.empty(t, device="cuda")
    print(f"[case] codes of ordinary rows {t} x {n}", flush=True)
    rs.relserve_quantise_rows_i8(x, codes, scales)
    torch.cuda.synchronize()
    assert torch.equal(codes, _want(x.double()))


ROWS = 2 ** 26 + 5      # of 64 threads each: 2^32 threads and a few more, which one launch cannot count


def _many(dtype, period, fill):
    """ROWS rows of 8 values that repeat after an odd number of them."""
    return fill(period).to(dtype).repeat(-(-ROWS // period), 1)[:ROWS].contiguous()


def _all_periods_alike(out, period):
    whole = ROWS // period * period
    return bool((out[:whole].view(-1, period, *out.shape[1:]) == out[:period]).all()) and torch.equal(out[whole:], out[:ROWS - whole])


def test_more_rows_than_a_launch_has_threads_for(rs):
    """Every row of a GB of short ones is written, by its own values: rows, and the norm with its sum in place."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    period = 2 ** 20 + 1
    x = _many(torch.bfloat16, period, lambda n: torch.randn(n, 8, generator=g, device="cuda"))
    codes, scales = torch.full((ROWS, 8), 77, dtype=torch.int8, device="cuda"), torch.full((ROWS,), -3.0, device="cuda")
    print(f"[case] rows {ROWS} x 8", flush=True)
    rs.relserve_quantise_rows_i8(x, codes, scales)
    torch.cuda.synchronize()
    assert torch.equal(codes[:period], _want(x[:period].double()))
    # m / 127 rounded once (in 32 bits torch divides by a number as it multiplies with its rounded reciprocal; the quotient of 53 bits is not
    # within a rounding of halfway between two of 24, from which m / 127 is 2^-32 of its value at least)
    assert torch.equal(scales[:period], (x[:period].double().abs().amax(1) / 127.0).float())
    assert _all_periods_alike(codes, period) and _all_periods_alike(scales, period)
    d = _many(torch.bfloat16, period, lambda n: torch.randn(n, 8, generator=g, device="cuda"))
    w = torch.tensor([1.0, 0.5, 1.5, 1.0, 2.0, 0.75, 1.25, 1.0], device="cuda").to(torch.bfloat16)
    want = (x[:period].float() + d[:period].float()).to(torch.bfloat16)
    codes.fill_(77)
    scales.fill_(-3.0)
    print(f"[case] norm {ROWS} x 8, the sum in place", flush=True)
    rs.relserve_add_rmsnorm_i8(x, w, 1e-5, codes, scales, delta=d, sum_out=x)
    torch.cuda.synchronize()
    s = want.double()
    m = (s * w.double()).abs().amax(1) / torch.sqrt(s.square().mean(1) + 1e-5)
    assert torch.equal(x[:period], want) and torch.equal(codes[:period], _want(s * w.double()))
    # squares of eight values in one chain, 63 additions of the lanes' zeros, root, reciprocal, m, its product, the division
    assert bool(((scales[:period].double() - m / 127.0).abs() <= 12 * U * m / 127.0).all())
    assert _all_periods_alike(x, period) and _all_periods_alike(codes, period) and _all_periods_alike(scales, period)
