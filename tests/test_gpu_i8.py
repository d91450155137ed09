"""The int8 operators (rows as 8-bit integers with a scale each, the norm that writes them, the projections that multiply them) against
plain 64-bit arithmetic on the same inputs, through the C-ABI binding.

Tolerances count roundings: one of fp32 is off by at most U = 2^-24 of its value, one to bf16 by B = 2^-8.  Sums of products of codes are
exact on both sides.
"""
import numpy as np
import pytest
import torch

from tests.gpu_harness import host_f32

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
GUARD = 3     # rows behind the last one, which no call may touch


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *size):
    return torch.randn(*size, generator=g, device="cuda", dtype=torch.float32)


def _stream(g, t, n):
    x = _randn(g, t, n)
    x[:, ::61] *= 8.0
    return x


def _with_guard(t, *rest, dtype, fill):
    full = torch.full((t + GUARD, *rest), fill, dtype=dtype, device="cuda")
    return full, full[:t]


def _untouched(full, t, fill):
    return bool((full[t:] == fill).all())


def _check_codes(codes, scales, values, scale_tol, code_tol, what):
    """codes, scales of rows whose exact values are `values` (64 bits): every code the nearest integer to value * 127 / m, but for what the
    roundings of that quotient move (code_tol, relative to 127); every scale m / 127."""
    m = values.abs().amax(1, keepdim=True)
    want = values * 127.0 / torch.where(m > 0, m, torch.ones_like(m))
    off = (codes.double() - want).abs().amax().item()
    assert off <= 0.5 + 127.0 * code_tol, f"{what}: a code is {off} from its quotient"
    assert int(codes.abs().amax()) <= 127
    rel = ((scales.double() - m[:, 0] / 127.0).abs() / torch.where(m[:, 0] > 0, m[:, 0] / 127.0, torch.ones_like(m[:, 0]))).amax().item()
    assert rel <= scale_tol, f"{what}: a scale is off by {rel} of its value"
    assert bool((scales[m[:, 0] == 0] == 0).all())


ROW_SIZES = [(1, 8), (5, 64), (300, 256), (37, 1000), (24, 2048), (9, 2056), (130, 5120), (1282, 5120), (7, 8192), (33, 13824), (3, 28672),
             (2, 65544), (2049, 512), (4100, 136), (1030, 1336), (1030, 2048), (60, 11000), (5, 20488)]


@pytest.mark.parametrize("t,n", ROW_SIZES)
def test_quantise_rows(rs, t, n):
    print(f"[case] quantise rows {t} x {n}", flush=True)
    g = _gen(t * 31 + n)
    x = _stream(g, t, n) * torch.exp(4 * _randn(g, t, 1))     # rows of very different magnitudes
    x = x.to(torch.bfloat16)
    if t > 2:
        x[t // 2] = 0
    full_c, codes = _with_guard(t, n, dtype=torch.int8, fill=77)
    full_s, scales = _with_guard(t, dtype=torch.float32, fill=-3.0)
    rs.relserve_quantise_rows_i8(x, codes, scales)
    torch.cuda.synchronize()
    assert _untouched(full_c, t, 77) and _untouched(full_s, t, -3.0)
    # m is exact; 127 / m and its product with the value are rounded, m / 127 once
    _check_codes(codes, scales, x.double(), 1.01 * U, 2.02 * U, f"{t} x {n}")


@pytest.mark.parametrize("t,n", ROW_SIZES)
@pytest.mark.parametrize("f32,delta,kept", [(False, True, "sum"), (True, False, None), (True, True, "in place"), (False, False, None),
                                            (False, True, None), (True, False, "sum")],
                         ids=["bf16+delta", "f32", "f32+delta in place", "bf16", "bf16+delta not kept", "f32 copied"])
def test_add_rmsnorm(rs, t, n, f32, delta, kept):
    print(f"[case] add rmsnorm {t} x {n} f32={f32} delta={delta} sum={kept}", flush=True)
    g = _gen(t * 37 + n)
    dtype = torch.float32 if f32 else torch.bfloat16
    full_x = torch.full((t + GUARD, n), 5.0, dtype=dtype, device="cuda")
    full_x[:t] = (_stream(g, t, n) * torch.exp(_randn(g, t, 1))).to(dtype)
    x = full_x[:t]
    d = (_randn(g, t, n) * 0.5).to(torch.bfloat16) if delta else None
    w = (1.0 + 0.1 * _randn(g, n)).to(torch.bfloat16)
    before = x.clone()
    want = before if d is None else (before.float() + d.float()).to(dtype)     # one fp32 addition: the same bits on both sides
    full_c, codes = _with_guard(t, n, dtype=torch.int8, fill=77)
    full_s, scales = _with_guard(t, dtype=torch.float32, fill=-3.0)
    full_o, out = _with_guard(t, n, dtype=dtype, fill=9.0)
    rs.relserve_add_rmsnorm_i8(x, w, 1e-5, codes, scales, delta=d, sum_out={"sum": out, "in place": x, None: None}[kept])
    torch.cuda.synchronize()
    assert _untouched(full_c, t, 77) and _untouched(full_s, t, -3.0) and _untouched(full_x, t, 5.0) and _untouched(full_o, t, 9.0)
    if kept:
        assert torch.equal(out if kept == "sum" else x, want)
    if kept != "in place":
        assert torch.equal(x, before)
    s = want.double()
    values = s * w.double() / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5)
    # codes: the products s w, 127 / m, their product, and m's own rounding.  The scale: at most n / 64 squares in one chain, a tree of the
    # rest, of which the root halves the error, the quotient, root and reciprocal, m, its product and the division by 127
    _check_codes(codes, scales, values, ((n / 64 + 16) / 2 + 7) * U, 4.04 * U, f"{t} x {n}")


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("n", [2056, 4104, 6152, 8200])
def test_sum_in_place_whose_last_values_are_the_largest(rs, n, f32):
    """Rows that end just behind a multiple of the threads, the sum written over x: threads past the end read the last chunk again, which
    its owner may already have stored."""
    t = 4100
    print(f"[case] sum in place {t} x {n} f32={f32}", flush=True)
    g = _gen(n)
    dtype = torch.float32 if f32 else torch.bfloat16
    x = _randn(g, t, n).to(dtype)
    d = torch.zeros(t, n, dtype=torch.bfloat16, device="cuda")
    d[:, -8:] = 100.0
    w = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    want = (x.float() + d.float()).to(dtype)
    codes, scales = torch.empty(t, n, dtype=torch.int8, device="cuda"), torch.empty(t, device="cuda")
    rs.relserve_add_rmsnorm_i8(x, w, 1e-5, codes, scales, delta=d, sum_out=x)
    torch.cuda.synchronize()
    assert torch.equal(x, want)
    s = want.double()
    _check_codes(codes, scales, s / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5), ((n / 64 + 16) / 2 + 7) * U, 4.04 * U, f"{n}")


@pytest.mark.parametrize("t,n", [(8300, 5136), (2500, 28680)])
def test_rows_of_more_than_the_caches_hold(rs, t, n):
    """As above where the passes stream; 64 of the rows, and the others' codes by their range and the scale they have."""
    print(f"[case] large rows {t} x {n}", flush=True)
    g = _gen(9)
    x, d = (_stream(g, t, n) * 0.7).to(torch.bfloat16), _randn(g, t, n).to(torch.bfloat16)
    w = (1.0 + 0.1 * _randn(g, n)).to(torch.bfloat16)
    some = torch.arange(0, t, t // 64, device="cuda")
    full_c, codes = _with_guard(t, n, dtype=torch.int8, fill=77)
    full_s, scales = _with_guard(t, dtype=torch.float32, fill=-3.0)
    full_o, out = _with_guard(t, n, dtype=torch.bfloat16, fill=9.0)
    rs.relserve_add_rmsnorm_i8(x, w, 1e-5, codes, scales, delta=d, sum_out=out)
    torch.cuda.synchronize()
    assert torch.equal(out, (x.float() + d.float()).to(torch.bfloat16))
    s = out[some].double()
    _check_codes(codes[some], scales[some], s * w.double() / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5), ((n / 64 + 16) / 2 + 7) * U,
                 4.04 * U, f"{t} x {n}")
    assert bool((codes.abs().amax(1) == 127).all())
    x = torch.cat([x, x])
    full_c, codes = _with_guard(2 * t, n, dtype=torch.int8, fill=77)
    full_s, scales = _with_guard(2 * t, dtype=torch.float32, fill=-3.0)
    rs.relserve_quantise_rows_i8(x, codes, scales)
    torch.cuda.synchronize()
    _check_codes(codes[some], scales[some], x[some].double(), 1.01 * U, 2.02 * U, f"{t} x {n}")
    assert torch.equal(codes[:t], codes[t:]) and torch.equal(scales[:t], scales[t:]) and bool((codes.abs().amax(1) == 127).all())
    assert _untouched(full_c, 2 * t, 77) and _untouched(full_s, 2 * t, -3.0) and _untouched(full_o, t, 9.0)


def test_rows_out_of_the_ordinary(rs):
    """Zeros, the smallest and largest magnitudes, infinities, NaN: each row by itself, the others as they would be without it."""
    n = 1000
    g = _gen(5)
    x = _randn(g, 12, n)
    plain = [0, 1, 11]
    x[2] = 0
    x[3] *= 1e-38          # bf16 (and fp32) numbers below the normal range
    x[4] = 0
    x[4, 17] = 9.2e-41     # the smallest bf16 number
    x[5] *= 2.5e37
    x[6, 999] = float("inf")
    x[7, 0] = float("-inf")
    x[8, 500] = float("nan")
    x[9, 3] = float("nan")
    x[9, 4] = float("inf")
    x[10] = -3.0
    x = x.to(torch.bfloat16)
    codes = torch.full((12, n), 77, dtype=torch.int8, device="cuda")
    scales = torch.full((12,), -3.0, device="cuda")
    rs.relserve_quantise_rows_i8(x, codes, scales)
    torch.cuda.synchronize()
    finite = [0, 1, 2, 5, 10, 11]
    _check_codes(codes[finite], scales[finite], x[finite].double(), 1.01 * U, 2.02 * U, "rows")
    # below 2^-126 the scale itself is rounded to a multiple of 2^-149; the codes are not affected
    _check_codes(codes[[3, 4]], x[[3, 4]].double().abs().amax(1) / 127.0, x[[3, 4]].double(), 1e-9, 2.02 * U, "tiny rows")
    assert bool(((scales[[3, 4]].double() - x[[3, 4]].double().abs().amax(1) / 127.0).abs() <= 2.0 ** -149).all())
    assert bool((codes[6:10] == 0).all()) and not bool(torch.isfinite(scales[6:10]).any()) and bool(torch.isnan(scales[8:10]).all())
    assert bool((codes[10] == -127).all())

    # the norm: such a row's scale is not finite either, zeros are zeros
    w = (1.0 + 0.1 * _randn(g, n)).to(torch.bfloat16)
    w[40] = 0
    rs.relserve_add_rmsnorm_i8(x, w, 1e-5, codes, scales)
    torch.cuda.synchronize()
    assert bool((codes[6:10] == 0).all()) and bool(torch.isnan(scales[6:10]).all())
    assert bool((codes[2] == 0).all()) and float(scales[2]) == 0.0
    s = x[plain].double()
    _check_codes(codes[plain], scales[plain], s * w.double() / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5), 24 * U, 4.04 * U, "rows")
    # a row of denormals: 1 / sqrt(mean + eps) is about 316, so the scale is a normal number's neighbour and absolutely exact to 2^-149 * 316
    values = x[3].double() * w.double() / np.sqrt(1e-5)
    assert abs(float(scales[3]) - float(values.abs().max()) / 127.0) <= 320 * 2.0 ** -149


def _codes(g, t, k):
    x = _stream(g, t, k)
    scale = x.abs().amax(1) / 127.0
    return torch.round(x / scale[:, None]).to(torch.int8), scale


class Product:
    """Operands of a projection and its exact sums."""

    def __init__(self, rs, t, n, k, packed, seed=0):
        g = _gen(seed + t * 131 + n * 7 + k)
        self.rs, self.t, self.n, self.k, self.packed = rs, t, n, k, packed
        self.a, self.a_scale = _codes(g, t, k)
        self.w, self.w_scale = _codes(g, n, k)
        self.w_scale *= 0.02 / self.w_scale.mean() / np.sqrt(k) / 3.0
        self.held = rs.pack_codes(self.w) if packed else self.w
        self.y = (self.a.double() @ self.w.double().t()) * self.a_scale.double()[:, None] * self.w_scale.double()
        self.g = g

    def call(self, epilogue, residual, out, workspace=None, stream=None):
        self.rs.relserve_linear_i8(self.a, self.a_scale, self.held, self.w_scale, epilogue, residual, out, n=self.n if self.packed else 0,
                                   workspace=workspace, stream=stream)

    def workspace(self):
        return torch.empty(self.rs.relserve_linear_i8_workspace_bytes(self.t, self.n), dtype=torch.uint8, device="cuda")

    def check(self, epilogue, workspace=None, with_residual=True):
        t, n, y = self.t, self.n, self.y
        what = f"T={t} N={n} K={self.k} packed={self.packed} epilogue {epilogue}"
        dtype = torch.float32 if epilogue == 1 else torch.bfloat16
        full, out = _with_guard(t, n // 2 if epilogue == 3 else n, dtype=dtype, fill=9.0)
        res = None
        if epilogue == 2 or (epilogue == 1 and with_residual):
            res = _randn(self.g, t, n).to(torch.bfloat16 if epilogue == 1 else torch.float32)
        self.call(epilogue, res, out, workspace)
        torch.cuda.synchronize()
        assert _untouched(full, t, 9.0), what
        # the sum's conversion and two products: 3 U; the addition U; bf16 B
        if epilogue == 3:
            gate, up = y[:, :n // 2], y[:, n // 2:]
            want = gate * torch.sigmoid(gate) * up
            # e^-g from an argument off by 4 U of g, the hardware's exponential and reciprocal (2 U each), 1 + e, two products, up: 3 U
            tol = (B + (4 * gate.abs() + 16) * U) * want.abs() + 1e-30
        else:
            want = y if res is None else y + res.double()
            tol = 3.03 * U * y.abs() + (U if epilogue == 1 else U + B) * 1.01 * want.abs()
        bad = ((out.double() - want).abs() > tol) | ~torch.isfinite(out.double())
        assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} values off, first at {bad.nonzero()[0].tolist()}"
        return out.clone()


LINEAR_SIZES = [(1, 4, 128), (1, 5120, 5120), (3, 16, 256), (24, 15360, 1024), (31, 260, 384), (33, 1004, 1152), (64, 256, 5120),
                (65, 512, 2048), (128, 5120, 13824), (129, 132, 640), (192, 1024, 4096), (200, 2048, 128), (256, 640, 2560), (257, 512, 5120),
                (300, 1000, 512), (385, 7168, 2560), (640, 5120, 1024), (1282, 5120, 640), (1384, 1536, 1024), (2100, 1088, 128), (17, 5120, 13824), (8, 4096, 28672), (50, 12288, 4096), (70, 10240, 640),
                (12, 20480, 5120)]


@pytest.mark.parametrize("packed", [False, True], ids=["rowmajor", "packed"])
@pytest.mark.parametrize("t,n,k", LINEAR_SIZES)
def test_linear(rs, t, n, k, packed):
    print(f"[case] linear i8 T={t} N={n} K={k} packed={packed}", flush=True)
    p = Product(rs, t, n, k, packed)
    ws = p.workspace()
    for epilogue in (0, 1, 2):
        p.check(epilogue, ws)
    # without scratch: the same bits
    assert torch.equal(p.check(1, None, with_residual=False), p.check(1, ws, with_residual=False))


@pytest.mark.parametrize("packed", [False, True], ids=["rowmajor", "packed"])
@pytest.mark.parametrize("t,inner,k", [(1, 8, 128), (1, 13824, 1024), (9, 128, 128), (33, 1000, 256), (64, 13824, 512), (130, 768, 640), (250, 14336, 256),
                                       (300, 1000, 512), (1384, 5504, 256), (2100, 2808, 128)])
def test_linear_swiglu(rs, t, inner, k, packed):
    print(f"[case] linear i8 swiglu T={t} I={inner} K={k} packed={packed}", flush=True)
    p = Product(rs, t, 2 * inner, k, packed)
    assert torch.equal(p.check(3, p.workspace()), p.check(3, None))


@pytest.mark.parametrize("splits", [0, 2, 4])
@pytest.mark.parametrize("tile", range(5))
def test_every_tile_and_split_gives_the_same_bits(rs, tile, splits):
    p, q = Product(rs, 700, 1284, 4096, True), Product(rs, 333, 1008, 4096, False)
    want = [(x, e, x.check(e, x.workspace())) for x, e in ((p, 0), (p, 1), (p, 2), (q, 3), (q, 0))]
    try:
        for x, e, w in want:
            print(f"[case] linear i8 T={x.t} N={x.n} epilogue {e} tile {tile} splits {splits}", flush=True)
            rs.relserve_debug_force_gemm_plan(tile, splits)
            got = x.check(e, x.workspace())
            rs.relserve_debug_force_gemm_plan()
            if e in (0, 3):     # (the others' residuals are drawn anew)
                assert torch.equal(got, w)
    finally:
        rs.relserve_debug_force_gemm_plan()


@pytest.mark.parametrize("t,n,k,e", [(640, 1280, 5120, 1), (265, 2564, 13824, 2), (320, 8192, 13824, 0), (900, 2564, 8192, 0), (1900, 20480, 2048, 3),
                                     (780, 10240, 1024, 0), (500, 20480, 1024, 3), (780, 15360, 2048, 0)])
def test_plans_of_more_tokens(rs, t, n, k, e):
    """Tails and whole problems in k ranges, two tile shapes side by side, whole tiles of each shape: a forced tile's bits, with scratch and without."""
    print(f"[case] linear i8 T={t} N={n} K={k} epilogue {e}", flush=True)
    p = Product(rs, t, n, k, True)
    dtype = torch.float32 if e == 1 else torch.bfloat16
    res = _randn(p.g, t, n).to(torch.bfloat16 if e == 1 else torch.float32) if e in (1, 2) else None
    got = []
    p.check(e, p.workspace())
    for force, workspace in ((False, p.workspace()), (False, None), (True, None)):
        out = torch.empty(t, n // 2 if e == 3 else n, dtype=dtype, device="cuda")
        try:
            if force:
                rs.relserve_debug_force_gemm_plan(2, 0)
            p.call(e, res, out, workspace)
        finally:
            rs.relserve_debug_force_gemm_plan()
        got.append(out)
    torch.cuda.synchronize()
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[2])


@pytest.mark.parametrize("splits", [0, 2, 4])
@pytest.mark.parametrize("t,n,k", [(1, 512, 128), (159, 1284, 256), (160, 1008, 384), (161, 512, 512), (320, 1284, 640), (333, 1008, 4096), (700, 1284, 4096)])
def test_the_tile_of_160_tokens_gives_the_same_bits(rs, t, n, k, splits):
    """An odd number of token fragments a wave, of all lengths of its ring of three stages."""
    for packed in (False, True):
        p = Product(rs, t, n, k, packed)
        for e in (0, 1, 2, 3):
            if e == 3 and n % 16:
                continue
            print(f"[case] linear i8 T={t} N={n} K={k} epilogue {e} packed={packed} splits {splits}", flush=True)
            want = p.check(e, p.workspace())
            try:
                rs.relserve_debug_force_gemm_plan(5, splits)
                got = p.check(e, p.workspace())
            finally:
                rs.relserve_debug_force_gemm_plan()
            if e in (0, 3):     # (the others' residuals are drawn anew)
                assert torch.equal(got, want)


@pytest.mark.parametrize("t,n,k,e", [(1, 5120, 5120, 0), (16, 1004, 1280, 0), (24, 2056, 2048, 0), (32, 27648, 4096, 3), (33, 512, 384, 0), (64, 10240, 2048, 0),
                                     (60, 5124, 4096, 0), (100, 6000, 128, 0), (200, 2816, 1152, 3), (900, 520, 640, 0), (2, 57344, 2048, 3), (130, 10000, 2176, 0), (128, 11264, 5120, 3),
                                     (75, 7172, 4096, 0), (250, 3600, 5120, 3), (640, 2560, 4096, 0)])
def test_small_problems_give_the_tiled_kernels_bits(rs, t, n, k, e):
    """A forced tile sends these to the kernels of larger problems."""
    for packed in (False, True):
        print(f"[case] linear i8 T={t} N={n} K={k} epilogue {e} packed={packed}", flush=True)
        p = Product(rs, t, n, k, packed)
        got = p.check(e)
        try:
            rs.relserve_debug_force_gemm_plan(4, 0)
            assert torch.equal(got, p.check(e))
        finally:
            rs.relserve_debug_force_gemm_plan()


@pytest.mark.parametrize("t", [1, 40, 300])
def test_largest_sums(rs, t):
    """Codes at the ends of their range, k as long as 32 bits allow: sums up to 2^31 - 2^21."""
    k, n = 130944, 8
    a = torch.full((t, k), 127, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), 127, dtype=torch.int8, device="cuda")
    w[1], w[2], a[t // 2], w[3, ::2], w[4, k // 2:] = -128, -127, -128, -127, -128
    a_scale, w_scale = torch.full((t,), 2.0 ** -10, device="cuda"), torch.full((n,), 2.0 ** -12, device="cuda")
    want = (a.double() @ w.double().t()) * 2.0 ** -22
    for held, rows in ((w, 0), (rs.pack_codes(w), n)):
        for workspace in (None, torch.empty(rs.relserve_linear_i8_workspace_bytes(t, n), dtype=torch.uint8, device="cuda")):
            out = torch.zeros((t, n), device="cuda")
            rs.relserve_linear_i8(a, a_scale, held, w_scale, 1, None, out, n=rows, workspace=workspace)
            torch.cuda.synchronize()
            assert bool(((out.double() - want).abs() <= U * want.abs()).all())     # the conversion to fp32 alone


def test_scales_that_are_not_finite(rs):
    p = Product(rs, 70, 128, 256, True)
    clean = p.check(0, p.workspace())
    p.a_scale[5], p.a_scale[69] = float("nan"), float("inf")
    p.a[69, :] = 0
    out = torch.zeros((70, 128), dtype=torch.bfloat16, device="cuda")
    p.call(0, None, out, p.workspace())
    torch.cuda.synchronize()
    assert bool(torch.isnan(out[5]).all()) and bool(torch.isnan(out[69]).all())
    rest = [i for i in range(69) if i != 5]
    assert torch.equal(out[rest], clean[rest])


def _mlp(rs, bufs, stream=None):
    """norm, gate/up, quantise, down: a feed-forward block as a serving step runs it."""
    b = bufs
    rs.relserve_add_rmsnorm_i8(b["x"], b["w_norm"], 1e-5, b["codes"], b["scale"], delta=b["delta"], sum_out=b["sum"], stream=stream)
    rs.relserve_linear_i8(b["codes"], b["scale"], b["gu"].held, b["gu"].w_scale, 3, None, b["act"], n=b["gu"].n, workspace=b["ws"], stream=stream)
    rs.relserve_quantise_rows_i8(b["act"], b["act_codes"], b["act_scale"], stream=stream)
    rs.relserve_linear_i8(b["act_codes"], b["act_scale"], b["down"].held, b["down"].w_scale, 2, b["sum"], b["out"], n=b["down"].n,
                          workspace=b["ws"], stream=stream)


def _mlp_buffers(rs, t, h, inner, seed):
    g = _gen(seed)

    def empty(*size, dtype=torch.bfloat16):
        return torch.empty(*size, dtype=dtype, device="cuda")

    gu, down = Product(rs, 1, 2 * inner, h, True, seed), Product(rs, 1, h, inner, True, seed + 1)
    # weights of RMS about 0.02 and 0.01: the block's output is a fraction of the stream
    gu.w_scale *= 0.02 * 3 * np.sqrt(h)
    down.w_scale *= 0.01 * 3 * np.sqrt(inner)
    ws = max(rs.relserve_linear_i8_workspace_bytes(t, 2 * inner), rs.relserve_linear_i8_workspace_bytes(t, h))
    return {"x": _stream(g, t, h), "delta": (_randn(g, t, h) * 0.5).to(torch.bfloat16), "w_norm": (1 + 0.1 * _randn(g, h)).to(torch.bfloat16),
            "sum": empty(t, h, dtype=torch.float32), "codes": empty(t, h, dtype=torch.int8), "scale": empty(t, dtype=torch.float32),
            "gu": gu, "down": down, "act": empty(t, inner), "act_codes": empty(t, inner, dtype=torch.int8),
            "act_scale": empty(t, dtype=torch.float32), "out": empty(t, h), "ws": empty(ws, dtype=torch.uint8)}


@pytest.mark.parametrize("t,h,inner", [(1, 256, 384), (29, 1024, 2816), (150, 512, 1408), (640, 1024, 2816)])
def test_feed_forward_block(rs, t, h, inner):
    """The four calls as they are used, each step against 64 bits on the inputs it had."""
    print(f"[case] feed-forward block i8 T={t} H={h} I={inner}", flush=True)
    b = _mlp_buffers(rs, t, h, inner, t + h)
    _mlp(rs, b)
    torch.cuda.synchronize()
    s = b["sum"].double()
    assert torch.equal(b["sum"], b["x"] + b["delta"].float())
    _check_codes(b["codes"], b["scale"], s * b["w_norm"].double() / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5),
                 ((h / 64 + 16) / 2 + 7) * U, 4.04 * U, "norm")
    y = (b["codes"].double() @ b["gu"].w.double().t()) * b["scale"].double()[:, None] * b["gu"].w_scale.double()
    gate, up = y.chunk(2, 1)
    want = gate * torch.sigmoid(gate) * up
    assert bool(((b["act"].double() - want).abs() <= (B + (4 * gate.abs() + 16) * U) * want.abs() + 1e-30).all())
    _check_codes(b["act_codes"], b["act_scale"], b["act"].double(), 1.01 * U, 2.02 * U, "quantise")
    y = (b["act_codes"].double() @ b["down"].w.double().t()) * b["act_scale"].double()[:, None] * b["down"].w_scale.double()
    want = y + s
    assert bool(((b["out"].double() - want).abs() <= 3.03 * U * y.abs() + (U + B) * 1.01 * want.abs()).all())
    # and the whole against the block without any rounding: codes are within half a step, 1 / 254 of a row's largest magnitude
    exact = s * b["w_norm"].double() / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5)
    gate, up = ((exact @ b["gu"].w.double().t()) * b["gu"].w_scale.double()).chunk(2, 1)
    delta = ((gate * torch.sigmoid(gate) * up) @ b["down"].w.double().t()) * b["down"].w_scale.double()
    got = b["out"].double() - s
    rel = float((got - delta).norm() / delta.norm())
    print(f"[parity] block's own contribution rel-L2 {rel:.2e}", flush=True)


def test_feed_forward_block_captured_and_on_streams(rs):
    """Two blocks captured into graphs on a side stream, replayed in turn with eager work between; each replay equals the eager run."""
    blocks = [_mlp_buffers(rs, 24, 512, 1408, 3), _mlp_buffers(rs, 300, 512, 1408, 4)]
    want = []
    for b in blocks:
        _mlp(rs, b)
        torch.cuda.synchronize()
        want.append(b["out"].clone())
    side = torch.cuda.Stream()
    graphs = []
    for b in blocks:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            _mlp(rs, b, stream=side)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            _mlp(rs, b, stream=side)
        graphs.append(graph)
    for turn in range(3):
        for b, graph, out in zip(blocks, graphs, want):
            b["out"].fill_(0.0)
            b["ws"].fill_(0xff)          # what an earlier call left there does not matter
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(b["out"], out), turn
        _mlp(rs, blocks[turn % 2])
        torch.cuda.synchronize()


def test_no_rows(rs):
    def empty(*size, dtype=torch.bfloat16):
        return torch.empty(*size, dtype=dtype, device="cuda")

    codes, scales = empty(0, 256, dtype=torch.int8), empty(0, dtype=torch.float32)
    rs.relserve_quantise_rows_i8(empty(0, 256), codes, scales)
    rs.relserve_add_rmsnorm_i8(empty(0, 256), empty(256), 1e-5, codes, scales, delta=empty(0, 256), sum_out=empty(0, 256))
    w, ws = empty(64, 256, dtype=torch.int8), empty(64, dtype=torch.float32)
    for epilogue, n, dtype in ((0, 64, torch.bfloat16), (1, 64, torch.float32), (2, 64, torch.bfloat16), (3, 32, torch.bfloat16)):
        rs.relserve_linear_i8(codes, scales, w, ws, epilogue, empty(0, 64, dtype=torch.float32) if epilogue == 2 else None, empty(0, n, dtype=dtype))
    torch.cuda.synchronize()


def test_two_calls_at_once(rs):
    """Calls on two streams, each with a workspace of its own."""
    ps = [Product(rs, 24, 5120, 5120, True, seed=i) for i in range(2)]
    outs = [torch.zeros((24, 5120), dtype=torch.bfloat16, device="cuda") for _ in ps]
    want = [p.check(0, p.workspace()) for p in ps]
    spaces, streams = [p.workspace() for p in ps], [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, out, ws, s in zip(ps, outs, spaces, streams):
            p.call(0, None, out, ws, stream=s)
    torch.cuda.synchronize()
    for out, w in zip(outs, want):
        np.testing.assert_array_equal(host_f32(out), host_f32(w))
