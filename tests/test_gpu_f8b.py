"""The block-scaled operators (matrices as 8-bit floating point codes with a scale for each block of 128, the norm that writes them, the projections
that multiply them) against plain 64-bit arithmetic on the same inputs, through the C-ABI binding.

Tolerances count roundings: one of fp32 is off by at most U = 2^-24 of its value, one to bf16 by B = 2^-8.
"""
import numpy as np
import pytest
import torch

from tests import f8b_paths

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
GUARD = 3     # rows behind the last one, which no call may touch
CODE = torch.float8_e4m3fn


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


def _values(codes):
    return codes.view(CODE).cpu().double().numpy()


def _nearest(q):
    """The number of the format nearest to each q, ties to the even one, by whole numbers of the format's step there (numpy's arithmetic is exact)."""
    _, e = np.frexp(q)
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    return np.round(q / step) * step


def _largest(v, block_rows):
    t, n = v.shape
    blocks = -(-t // block_rows)
    top = np.zeros((blocks * block_rows, n // 128))
    top[:t] = np.abs(v).reshape(t, n // 128, 128).max(2)
    return top.reshape(blocks, block_rows, n // 128).max(1)


def _check_codes(codes, scales, v, block_rows, what, exact=True, scale_tol=1.01 * U, factor=None):
    """codes, scales of v (64 bits): every code the nearest one to v * 448 / m, or (exact false) one that roundings of 4 U of the quotient can reach;
    scales m / 448 (times factor, a row's)."""
    top = _largest(v, block_rows)
    each = top.repeat(block_rows, 0)[:v.shape[0]].repeat(128, 1)
    q = v * 448.0 / np.where(each > 0, each, 1.0)
    got, want = _values(codes), _nearest(q)
    if exact:
        assert np.array_equal(got, want), f"{what}: {(got != want).sum()} codes are not the nearest"
    else:
        assert (np.abs(got - q) <= np.abs(want - q) + 8 * U * np.abs(q)).all(), what
    want = top / 448.0
    if factor is not None:
        want = want * factor[:, None]
    got = scales.cpu().double().numpy()
    got = got.T if block_rows == 1 else got
    assert (np.abs(got - want) <= scale_tol * want + 2.0 ** -149).all(), f"{what}: a scale is off by {(np.abs(got - want) / np.maximum(want, 1e-300)).max()}"


ROW_SIZES = [(1, 128), (5, 256), (300, 384), (24, 2048), (17, 5120), (1282, 5120), (7, 8192), (33, 13824), (3, 28672), (1, 65664), (2050, 1024), (1029, 2048)]


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("t,n", ROW_SIZES + [(128, 128), (129, 640), (255, 256)])
def test_quantise(rs, t, n, block_rows):
    print(f"[case] quantise {t} x {n} in blocks of {block_rows}", flush=True)
    g = _gen(t * 31 + n)
    x = (_stream(g, t, n) * torch.exp(4 * _randn(g, t, 1))).to(torch.bfloat16)
    x[:, :128][::3] = 0                                             # blocks of zeros, and of one value
    if n > 128:
        x[:, 128:256] = x[:, 128:129]
    full_c, codes = _with_guard(t, n, dtype=torch.uint8, fill=77)
    blocks = -(-t // 128) if block_rows == 128 else n // 128
    full_s, scales = _with_guard(blocks, n // 128 if block_rows == 128 else t, dtype=torch.float32, fill=-3.0)
    rs.relserve_quantise_f8b(x, codes, scales, block_rows=block_rows)
    torch.cuda.synchronize()
    assert bool((full_c[t:] == 77).all()) and bool((full_s[blocks:] == -3.0).all())
    _check_codes(codes, scales, x.cpu().double().numpy(), block_rows, f"{t} x {n}")


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantise_halfway_and_far_values(rs, block_rows):
    """Quotients exactly between two codes, blocks near either end of the type's range, and blocks with nothing to scale by."""
    t = 128
    v = torch.zeros(t, 128 * 9)
    ties = torch.tensor([1 + i / 16 for i in range(16)] + [2.0 ** -6 * (i + 0.5) / 8 for i in range(8)])
    for b, m in enumerate((448.0, 7.0, 2.0 ** -126 * 448, 2.0 ** 119 * 448)):
        v[:, 128 * b:128 * b + 24] = ties * (m / 448)
        v[:, 128 * b + 24:128 * b + 48] = -ties * (m / 448)
        v[:, 128 * b + 100] = m
    v[:, 512:640] = 2.0 ** -133                                      # bf16's smallest
    v[:, 640 + 5] = 3.3895e38                                        # and largest
    v[:, 768:896] = 1.0
    v[:, 896:1024] = 2.0
    v[0, 770], v[0, 900] = float("nan"), float("inf")
    x = v.to(torch.bfloat16).cuda()
    codes, scales = torch.empty(t, v.shape[1], dtype=CODE, device="cuda"), torch.empty((1, 9) if block_rows == 128 else (9, t), device="cuda")
    rs.relserve_quantise_f8b(x, codes, scales, block_rows=block_rows)
    s = scales if block_rows == 128 else scales.t()
    assert not bool(torch.isfinite(s[0, 6:8]).any()) and bool((codes.view(torch.uint8)[0, 768:1024] == 0).all())
    keep = list(range(0, 768)) + list(range(1024, 1152))
    _check_codes(codes[:, keep], (s[:, [0, 1, 2, 3, 4, 5, 8]] if block_rows == 128 else scales[[0, 1, 2, 3, 4, 5, 8]]).contiguous(),
                 x.cpu().double().numpy()[:, keep], block_rows, "halfway")
    assert bool((s[:, 8] == 0).all())


@pytest.mark.parametrize("t,n", ROW_SIZES)
@pytest.mark.parametrize("f32,delta,kept", [(False, True, "sum"), (True, False, None), (True, True, "in place"), (False, False, None),
                                            (False, True, None), (True, False, "sum")],
                         ids=["bf16+delta", "f32", "f32+delta in place", "bf16", "bf16+delta not kept", "f32 copied"])
def test_add_rmsnorm(rs, t, n, f32, delta, kept):
    if t * n > 1 << 22 and (f32, delta) not in ((False, True), (True, True)):
        pytest.skip("covered at the smaller sizes")
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
    full_c, codes = _with_guard(t, n, dtype=torch.uint8, fill=77)
    full_s, scales = _with_guard(n // 128, t, dtype=torch.float32, fill=-3.0)
    full_o, out = _with_guard(t, n, dtype=dtype, fill=9.0)
    rs.relserve_add_rmsnorm_f8b(x, w, 1e-5, codes, scales, delta=d, sum_out={"sum": out, "in place": x, None: None}[kept])
    torch.cuda.synchronize()
    assert bool((full_c[t:] == 77).all()) and bool((full_s[n // 128:] == -3.0).all()) and bool((full_x[t:] == 5.0).all()) and bool((full_o[t:] == 9.0).all())
    if kept:
        assert torch.equal(out if kept == "sum" else x, want)
    if kept != "in place":
        assert torch.equal(x, before)
    s = want.cpu().double().numpy()
    factor = 1.0 / np.sqrt((s * s).mean(1) + 1e-5)
    # scales: at most n / 64 squares in one chain, a tree of the rest, of which the root halves the error; the quotient, root, reciprocal, s w, its
    # product with the factor, the division by 448
    _check_codes(codes, scales, s * w.cpu().double().numpy(), 1, f"{t} x {n}", exact=not f32, scale_tol=((n / 64 + 16) / 2 + 8) * U, factor=factor)


def _problem(g, t, n, k, epilogue, packed, pow2=False):
    a = torch.randint(0, 256, (t, k), generator=g, device="cuda", dtype=torch.uint8)
    w = torch.randint(0, 256, (n, k), generator=g, device="cuda", dtype=torch.uint8)
    for c in (a, w):          # any code but the two that are no number, smaller magnitudes more often
        c[(c & 127) == 127] = 0
        c[(c & 127) > 100] &= 0xdf
    blocks = 2 * (-(-(n // 2) // 128)) if epilogue == 3 else -(-n // 128)
    a_scale = torch.exp(_randn(g, k // 128, t)) * 1e-3
    w_scale = torch.exp(_randn(g, blocks, k // 128)) * (1e-3 / k ** 0.5)
    residual = {1: _randn(g, t, n).to(torch.bfloat16), 2: _randn(g, t, n)}.get(epilogue)
    return a, a_scale, w, w_scale, residual


def _reference(a, a_scale, w, w_scale, residual, epilogue):
    """(result, what the products' magnitudes add up to) in 64 bits."""
    n, k = w.shape
    half = n // 2 if epilogue == 3 else n
    row = torch.arange(n, device=w.device)
    block = torch.where(row < half, row // 128, -(-half // 128) + (row - half) // 128)
    av = a.view(CODE).double() * a_scale.double().t().repeat_interleave(128, 1)
    wv = (w.view(CODE).double() * w_scale.double()[block].repeat_interleave(128, 1)).t().contiguous()
    y, size = av @ wv, av.abs() @ wv.abs()
    if residual is not None:
        y = y + residual.double()
    return y, size


def _check_linear(got, y, size, residual, epilogue, k, what):
    blocks = k // 128
    if epilogue == 1:
        # codes as bf16 are exact, 128 products and 4 partial sums a block, a scale's and a sum's rounding each, then the residual's
        tol = (132 + 3 + blocks + 8) * U * size + 2 * U * y.abs()
    else:
        # the instruction on codes keeps 13 bits below the largest of a group of eight products at least
        tol = 2.0 ** -10 * size + (blocks + 8) * U * size
    if epilogue == 3:
        half = y.shape[1] // 2
        gate, up, tg, tu = y[:, :half], y[:, half:], tol[:, :half], tol[:, half:]
        y = gate * torch.sigmoid(gate) * up
        # |d silu| <= 1.1, |silu(g)| <= |g|; the hardware's exponential and reciprocal: 4 U
        tol = 1.1 * tg * (up.abs() + tu) + (gate.abs() + tg) * tu + 8 * U * y.abs()
    if epilogue != 1:
        tol = tol + B * (y.abs() + tol) + 2.0 ** -133
    off = (got.double() - y).abs()
    bad = off > tol
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} values, the worst {float((off / tol).max())} of its tolerance"
    rel = float((got.double() - y).norm() / y.norm())
    assert rel <= (1e-6 if epilogue == 1 else B), f"{what}: {rel} of the norm"


def _run_linear(rs, p, epilogue, packed, scratch, n, stream=None):
    a, a_scale, w, w_scale, residual = p
    t = a.shape[0]
    full, out = _with_guard(t, n // 2 if epilogue == 3 else n, dtype=torch.float32 if epilogue == 1 else torch.bfloat16, fill=7.0)
    ws = torch.full((max(256, rs.relserve_linear_f8b_workspace_bytes(t, n)),), 255, dtype=torch.uint8, device="cuda") if scratch else None
    if packed:
        w = rs.pack_codes(w)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())   # the fills above too
    rs.relserve_linear_f8b(a, a_scale, w, w_scale, epilogue, residual, out, n=n if packed else 0, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    assert bool((full[t:] == 7.0).all())
    return out


LINEAR_SIZES = [(1, 4, 128), (1, 5120, 1024), (3, 132, 384), (16, 1000, 2048), (17, 260, 640), (24, 1536, 5120), (33, 4096, 256), (64, 2052, 1152),
                (65, 512, 4096), (100, 256, 8192), (129, 1004, 1152), (200, 8192, 512), (257, 300, 2048), (333, 1004, 1152), (512, 516, 640),
                (700, 2304, 128), (1000, 1028, 1280), (1282, 640, 2560), (2050, 1280, 384)]


@pytest.mark.parametrize("epilogue", [0, 1, 2, 3])
@pytest.mark.parametrize("t,n,k", LINEAR_SIZES)
def test_linear(rs, t, n, k, epilogue):
    if epilogue == 3:
        n = (n + 15) // 16 * 16
    packed = (t + n + k // 128 + epilogue) % 2 == 0
    print(f"[case] linear {t} x {n} x {k} epilogue {epilogue} packed={packed}", flush=True)
    p = _problem(_gen(t * 7 + n + k), t, n, k, epilogue, packed)
    y, size = _reference(*p, epilogue)
    results = [_run_linear(rs, p, epilogue, packed, scratch, n) for scratch in (True, False)]
    for got in results:
        _check_linear(got, y, size, p[4], epilogue, k, f"{t} x {n} x {k}")
    assert torch.equal(results[0], _run_linear(rs, p, epilogue, packed, True, n))            # the same bits every time
    assert torch.equal(results[0], _run_linear(rs, p, epilogue, not packed, True, n))        # and from either layout


@pytest.mark.parametrize("size", f8b_paths.SIZES, ids=str)
def test_paths(rs, size):
    """Every tile, whole and in k ranges, in either layout of the weights."""
    t, n, k, epilogue = size
    print(f"[case] path {f8b_paths.SIZES[size]}: {size}", flush=True)
    p = _problem(_gen(t + n + k), t, n, k, epilogue, False)
    y, bound = _reference(*p, epilogue)
    got = _run_linear(rs, p, epilogue, False, True, n)
    _check_linear(got, y, bound, p[4], epilogue, k, str(size))
    assert torch.equal(got, _run_linear(rs, p, epilogue, True, True, n))


def test_no_residual_is_a_residual_of_zeros(rs):
    for t in (3, 300):
        p = _problem(_gen(5), t, 516, 512, 0, False)
        q = (*p[:4], torch.zeros(t, 516, dtype=torch.bfloat16, device="cuda"))
        assert torch.equal(_run_linear(rs, p, 1, False, True, 516), _run_linear(rs, q, 1, False, True, 516))


@pytest.mark.parametrize("epilogue", [0, 1])
@pytest.mark.parametrize("t", [2, 24, 60, 200, 600])
def test_blocks_that_are_not_finite(rs, t, epilogue):
    """A token with such a block has no finite output; the others keep theirs."""
    n, k = 640, 1024
    p = _problem(_gen(t), t, n, k, epilogue, False)
    clean = _run_linear(rs, p, epilogue, False, True, n)
    a, a_scale = p[0].clone(), p[1].clone()
    a[1, 256:384] = 0
    a_scale[2, 1] = float("nan")
    got = _run_linear(rs, (a, a_scale, *p[2:]), epilogue, False, True, n)
    assert bool(torch.isnan(got[1]).all())
    rest = [i for i in range(t) if i != 1]
    assert torch.equal(got[rest], clean[rest])


def test_feed_forward_block(rs):
    """The calls of a feed-forward block one behind the other: off the same block in 64 bits (codes made by the same rule) by its roundings to bf16
    and the codes that those move."""
    for t in (5, 60, 700):
        g, h, m = _gen(t), 1024, 1408
        x = _stream(g, t, h)
        d = (_randn(g, t, h) * 0.5).to(torch.bfloat16)
        wn = (1.0 + 0.1 * _randn(g, h)).to(torch.bfloat16)

        def codes_of(v, rows):
            c = torch.empty(*v.shape, dtype=torch.uint8, device="cuda")
            s = torch.empty(-(-v.shape[0] // 128) if rows == 128 else v.shape[1] // 128, v.shape[1] // 128 if rows == 128 else v.shape[0], device="cuda")
            rs.relserve_quantise_f8b(v, c, s, block_rows=rows)
            return c, s

        gate, up, down = ((_randn(g, r, c) * 0.03).to(torch.bfloat16) for r, c in ((m, h), (m, h), (h, m)))
        (gc, gs), (uc, us), (dc, ds) = codes_of(gate, 128), codes_of(up, 128), codes_of(down, 128)
        wc, wsc = torch.cat([gc, uc]), torch.cat([gs, us])
        c, s = torch.empty(t, h, dtype=torch.uint8, device="cuda"), torch.empty(h // 128, t, device="cuda")
        ws = torch.empty(rs.relserve_linear_f8b_workspace_bytes(t, 2 * m), dtype=torch.uint8, device="cuda")
        rs.relserve_add_rmsnorm_f8b(x, wn, 1e-5, c, s, delta=d, sum_out=x)
        act = torch.empty(t, m, dtype=torch.bfloat16, device="cuda")
        rs.relserve_linear_f8b(c, s, rs.pack_codes(wc), wsc, 3, None, act, n=2 * m, workspace=ws)
        ac, asc = codes_of(act, 1)
        out = torch.empty(t, h, dtype=torch.bfloat16, device="cuda")
        ws2 = torch.empty(rs.relserve_linear_f8b_workspace_bytes(t, h), dtype=torch.uint8, device="cuda")
        rs.relserve_linear_f8b(ac, asc, rs.pack_codes(dc), ds, 2, x, out, n=h, workspace=ws2)
        y, _ = _reference(c, s, wc, wsc, None, 3)
        plain = y[:, :m] * torch.sigmoid(y[:, :m]) * y[:, m:]
        assert float((act.double() - plain).norm() / plain.norm()) <= B
        y2, _ = _reference(ac, asc, dc, ds, x, 2)
        assert float((out.double() - y2).norm() / y2.norm()) <= B


def test_replays_of_a_captured_chain(rs):
    """Norm, projection and log probabilities captured into a graph: every replay gives the eager call's bits, with other work between."""
    t, h, v = 24, 1024, 4000
    g = _gen(1)
    x, wn = _stream(g, t, h).to(torch.bfloat16), (1.0 + 0.1 * _randn(g, h)).to(torch.bfloat16)
    _, _, w, w_scale, _ = _problem(g, t, v, h, 0, False)
    ids = torch.randint(0, v, (t, 2), generator=g, device="cuda", dtype=torch.int32)
    c, s = torch.empty(t, h, dtype=torch.uint8, device="cuda"), torch.empty(h // 128, t, device="cuda")
    logits, lp, ent = torch.empty(t, v, device="cuda"), torch.empty(t, 2, device="cuda"), torch.empty(t, device="cuda")
    top, tlp = torch.empty(t, 5, dtype=torch.int32, device="cuda"), torch.empty(t, 5, device="cuda")
    ws = torch.empty(rs.relserve_linear_f8b_workspace_bytes(t, v) + 4096, dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(max(256, rs.relserve_logprobs_workspace_bytes(t, v, 5)), dtype=torch.uint8, device="cuda")

    def chain():
        rs.relserve_add_rmsnorm_f8b(x, wn, 1e-5, c, s)
        rs.relserve_linear_f8b(c, s, w, w_scale, 1, None, logits, workspace=ws)
        rs.relserve_logprobs(logits, ids, lp, ent, top, tlp, workspace=ws2)

    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for seed in range(3):
        x.copy_(_stream(_gen(10 + seed), t, h).to(torch.bfloat16))
        chain()
        torch.cuda.synchronize()
        want = [o.clone() for o in (c, s, logits, lp, ent, top, tlp)]
        for o in (c, s, logits, lp, ent, top, tlp, ws, ws2):
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for o, e in zip((c, s, logits, lp, ent, top, tlp), want):
            assert torch.equal(o, e)


def test_another_stream(rs):
    p = _problem(_gen(3), 40, 768, 2048, 1, False)
    want = _run_linear(rs, p, 1, False, True, 768)
    assert torch.equal(_run_linear(rs, p, 1, False, True, 768, stream=torch.cuda.Stream()), want)
