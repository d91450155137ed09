"""Block-scaled operators and log probabilities on more than the caches hold, on more rows than one launch takes, and behind element 2^32: paths that only
such sizes take.  Compared on the device, in 64 bits; tolerances as beside the smaller sizes."""
import pytest
import torch

from tests import f8b_far
from tests import test_gpu_f8b as small
from tests import test_gpu_f8b_precision as precision

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
CODE = torch.float8_e4m3fn
FAR = 256 << 20       # bytes that the last-level cache holds


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def _fill(x, g, scale=1.0):
    """normal values, every 61st channel eight times as large, each row on its own scale, a few hundred MB at a time"""
    step = max(1, (1 << 26) // x.shape[1])
    for at in range(0, x.shape[0], step):
        part = x[at:at + step]
        v = torch.randn(part.shape, generator=g, device="cuda") * scale
        v[:, ::61] *= 8.0
        part.copy_(v * torch.exp(torch.randn(part.shape[0], 1, generator=g, device="cuda")))


def _nearest(q):
    e = torch.frexp(q)[1]
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return torch.round(q / step) * step


def _check_codes(codes, scales, v, block_rows, exact=True, tol=1.01 * U, factor=None):
    """codes and scales [rows' blocks, blocks of a row] of v (64 bits), whose first row begins a block"""
    rows, n = v.shape
    top = v.abs().unflatten(1, (-1, 128)).amax(2)
    if block_rows > 1:
        full = torch.zeros(-(-rows // 128) * 128, n // 128, dtype=torch.float64, device="cuda")
        full[:rows] = top
        top = full.unflatten(0, (-1, 128)).amax(1)
    each = top.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)
    q = v * 448.0 / torch.where(each > 0, each, torch.ones_like(each))
    got, want = codes.view(CODE).double(), _nearest(q)
    if exact:
        assert torch.equal(got, want), f"{int((got != want).sum())} codes are not the nearest"
    else:
        assert bool(((got - q).abs() <= (want - q).abs() + 8 * U * q.abs()).all())
    want = top / 448.0 * (1.0 if factor is None else factor[:, None])
    assert bool(((scales.double() - want).abs() <= tol * want + 2.0 ** -149).all())


def _pieces(rows, n):
    step = max(128, (1 << 24) // n // 128 * 128)
    return [(at, min(rows, at + step)) for at in range(0, rows, step)]


@pytest.mark.parametrize("t,n", [(4099, 28672), (17001, 5504), (4003, 23808), (90011, 1152), (524288 + 17, 128)],
                         ids=["whole fours of blocks", "three left", "two left", "one left", "two launches"])
def test_rows(rs, t, n):
    assert t * n * 3 > FAR or t > 524288
    print(f"[case] far rows {t} x {n}", flush=True)
    x = torch.empty(t, n, dtype=torch.bfloat16, device="cuda")
    _fill(x, small._gen(n))
    full_c, codes = small._with_guard(t, n, dtype=torch.uint8, fill=77)
    full_s, scales = small._with_guard(n // 128, t, dtype=torch.float32, fill=-3.0)
    rs.relserve_quantise_f8b(x, codes, scales)
    assert bool((full_c[t:] == 77).all()) and bool((full_s[n // 128:] == -3.0).all())
    for a, b in _pieces(t, n):
        _check_codes(codes[a:b], scales[:, a:b].t(), x[a:b].double(), 1)


FIRST = 32768 * 128      # rows of blocks of 128 x 128 that one launch takes


def test_square_blocks_of_two_launches(rs):
    t, n = FIRST + 300, 128
    print(f"[case] far square blocks {t} x {n}", flush=True)
    x = torch.empty(t, n, dtype=torch.bfloat16, device="cuda")
    _fill(x, small._gen(5))
    full_c, codes = small._with_guard(t, n, dtype=torch.uint8, fill=77)
    full_s, scales = small._with_guard(-(-t // 128), 1, dtype=torch.float32, fill=-3.0)
    rs.relserve_quantise_f8b(x, codes, scales, block_rows=128)
    assert bool((full_c[t:] == 77).all()) and bool((full_s[-(-t // 128):] == -3.0).all())
    for a, b in ((0, 4096), (FIRST - 4096, FIRST), (FIRST, t)):
        _check_codes(codes[a:b], scales[a // 128:-(-b // 128)], x[a:b].double(), 128)


def _check_norm(rs, t, n, f32, delta, kept, pieces):
    g = small._gen(t + n)
    dtype = torch.float32 if f32 else torch.bfloat16
    full_x = torch.full((t + 3, n), 5.0, dtype=dtype, device="cuda")
    x = full_x[:t]
    _fill(x, g)
    d = None
    if delta:
        d = torch.empty(t, n, dtype=torch.bfloat16, device="cuda")
        _fill(d, g, 0.5)
    w = (1.0 + 0.1 * torch.randn(n, generator=g, device="cuda")).to(torch.bfloat16)
    before = [x[a:b].clone() for a, b in pieces]
    full_c, codes = small._with_guard(t, n, dtype=torch.uint8, fill=77)
    full_s, scales = small._with_guard(n // 128, t, dtype=torch.float32, fill=-3.0)
    out = x if kept == "in place" else torch.empty_like(x) if kept else None
    rs.relserve_add_rmsnorm_f8b(x, w, 1e-5, codes, scales, delta=d, sum_out=out)
    assert bool((full_c[t:] == 77).all()) and bool((full_s[n // 128:] == -3.0).all()) and bool((full_x[t:] == 5.0).all())
    for (a, b), was in zip(pieces, before):
        s = was if d is None else (was.float() + d[a:b].float()).to(dtype)
        if out is not None:
            assert torch.equal(out[a:b], s)
        if kept != "in place":
            assert torch.equal(x[a:b], was)
        s = s.double()
        factor = 1.0 / (s.square().mean(1) + 1e-5).sqrt()
        _check_codes(codes[a:b], scales[:, a:b].t(), s * w.double(), 1, exact=not f32, tol=((n / 64 + 16) / 2 + 8) * U, factor=factor)


@pytest.mark.parametrize("f32,delta,kept", [(False, True, "sum"), (True, True, "in place"), (False, False, None), (True, False, "sum"), (False, True, None)],
                         ids=["bf16+delta", "f32+delta in place", "bf16", "f32 copied", "bf16+delta not kept"])
@pytest.mark.parametrize("n", [3968, 5248, 7808, 12416, 28800])
def test_norm(rs, n, f32, delta, kept):
    """Rows of each length class, as many as are just more than the cache holds."""
    size = 4 if f32 else 2
    row = n * (size * (2 if delta and kept else 1) + (2 if delta else 0) + 1)
    t = FAR // row + 3
    print(f"[case] far norm {t} x {n} f32={f32} delta={delta} sum={kept}", flush=True)
    _check_norm(rs, t, n, f32, delta, kept, _pieces(t, n))


def test_norm_of_two_launches_and_rows_behind_element_2_32(rs):
    """Short rows have a wave each: 2^25 of them in a launch."""
    first, t = 1 << 25, (1 << 25) + 37
    print(f"[case] far norm {t} x 128", flush=True)
    _check_norm(rs, t, 128, False, True, "in place", [(0, 1024), (first - 1024, first), (first, t)])


def test_rows_behind_element_2_32(rs):
    t, n = (1 << 25) + 37, 128
    print(f"[case] far rows {t} x {n}", flush=True)
    x = torch.empty(t, n, dtype=torch.bfloat16, device="cuda")
    _fill(x, small._gen(8))
    codes, scales = torch.empty(t, n, dtype=torch.uint8, device="cuda"), torch.empty(1, t, device="cuda")
    rs.relserve_quantise_f8b(x, codes, scales)
    for a, b in ((0, 1024), (524288 - 64, 524288 + 64), ((1 << 25) - 1024, t)):
        _check_codes(codes[a:b], scales[:, a:b].t(), x[a:b].double(), 1)


@pytest.mark.parametrize("size", f8b_far.SIZES, ids=str)
def test_linear(rs, size):
    t, n, k, epilogue = size
    print(f"[case] far linear {f8b_far.SIZES[size]}: {size}", flush=True)
    p = small._problem(small._gen(t + n + k), t, n, k, epilogue, False)
    y, bound = small._reference(*p, epilogue)
    got = small._run_linear(rs, p, epilogue, False, True, n)
    small._check_linear(got, y, bound, p[4], epilogue, k, str(size))
    assert torch.equal(got, small._run_linear(rs, p, epilogue, True, True, n))
    if epilogue != 1:
        precision.check_path(rs, size)


@pytest.mark.parametrize("epilogue", [0, 1])
def test_linear_outputs_behind_element_2_32(rs, epilogue):
    t, n, k = (1 << 20) + 5, 4608, 128
    print(f"[case] far linear {t} x {n} x {k} epilogue {epilogue}", flush=True)
    a, a_scale, w, w_scale, _ = small._problem(small._gen(2), t, n, k, 0, False)
    full, out = small._with_guard(t, n, dtype=torch.float32 if epilogue else torch.bfloat16, fill=7.0)
    ws = torch.empty(rs.relserve_linear_f8b_workspace_bytes(t, n), dtype=torch.uint8, device="cuda")
    rs.relserve_linear_f8b(a, a_scale, w, w_scale, epilogue, None, out, workspace=ws)
    assert bool((full[t:] == 7.0).all())
    for i in (0, (1 << 32) // n - 100, t - 200):
        rows = slice(i, i + 200)
        y, bound = small._reference(a[rows].contiguous(), a_scale[:, rows].contiguous(), w, w_scale, None, 0)
        small._check_linear(out[rows], y, bound, None, epilogue, k, f"rows from {i}")


@pytest.mark.parametrize("n_top", [0, 7])
def test_logits_behind_element_2_32(rs, n_top):
    """The largest vocabulary."""
    t, v = 258, 1 << 24
    print(f"[case] far log probabilities {t} x {v} top {n_top}", flush=True)
    g = small._gen(4)
    x = torch.empty(t, v, dtype=torch.bfloat16, device="cuda")
    for row in x:
        row.copy_(torch.randn(v, generator=g, device="cuda") * 2.0)
    ids = torch.randint(0, v, (t, 2), generator=g, device="cuda", dtype=torch.int32)
    lp, h = torch.empty(t, 2, device="cuda"), torch.empty(t, device="cuda")
    top, tlp = torch.empty(t, n_top, dtype=torch.int32, device="cuda"), torch.empty(t, n_top, device="cuda")
    rs.relserve_logprobs(x, ids, lp, h, top if n_top else None, tlp if n_top else None)
    for r in (0, 127, 128, t - 1):
        d = x[r].double() - x[r].double().max()
        e = d.exp()
        z = e.sum()
        lz, mean = float(z.log()), float((-d * e).sum() / z)
        # S: an exponential and its argument, 31 additions of a chunk, 2048 chunks, 24 behind them; a term's argument is off by 3 |d| U, e^d |d| of all terms: mean z
        s = 2 + 3 * mean + 31 + 2048 + 24
        want = d[ids[r].long()] - lz
        assert bool(((lp[r].double() - want).abs() <= U * (s + 4 * lz + 2 * want.abs())).all())
        assert abs(float(h[r]) - (lz + mean)) <= U * (s + 4 * lz + (2 * s + 4) * mean + 2 * (lz + mean))
        if n_top:
            value, at = torch.sort(x[r].float(), descending=True, stable=True)
            assert torch.equal(top[r].long(), at[:n_top])
            assert bool(((tlp[r].double() - (d[at[:n_top]] - lz)).abs() <= U * (s + 4 * lz + 2 * lz)).all())
