"""int8 projections at sizes where scratch is used or k is cut: few tokens in k ranges and whole, all tiles in k ranges, cut tails, two shapes
(tests/i8_paths.py, whose plans a CPU test holds), against 64 bits; the q/k/v projection on each of them too, and the largest sums on the tiled kernels.

Tolerances as in test_gpu_i8.py: U = 2^-24 a rounding of fp32, B = 2^-8 one to bf16."""
import numpy as np
import pytest
import torch

from paper_2601_11546_amd import workloads as W
from tests import i8_paths
from tests.test_gpu_i8 import B, U, Product, _gen, _randn
from tests.test_gpu_i8_layer import _bytes, _pools, _rotated

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


@pytest.mark.parametrize("t,n,k", list(i8_paths.LINEAR))
def test_linear(rs, t, n, k):
    print(f"[case] linear i8 T={t} N={n} K={k}", flush=True)
    p = Product(rs, t, n, k, True)
    for epilogue in (0, 1, 2):
        p.check(epilogue, p.workspace().fill_(0xff))      # what an earlier call left in the scratch does not matter


@pytest.mark.parametrize("t,n,k", list(i8_paths.SWIGLU))
def test_linear_swiglu(rs, t, n, k):
    print(f"[case] linear i8 swiglu T={t} N={n} K={k}", flush=True)
    p = Product(rs, t, n, k, True)
    p.check(3, p.workspace().fill_(0xff))


class Qkv:
    """Operands of a q/k/v projection of t tokens: decode rows up to 64, above that a chunk behind ten of them."""

    def __init__(self, rs, t, nq, nkv, d, hidden, seed=0):
        self.rs, self.t = rs, t
        self.shape = s = W.LayerShape(hidden, nq, nkv, d, 128)
        n_dec = t if t <= 64 else 10
        lengths, ctx = [1] * n_dec, [40 + 3 * i for i in range(n_dec)]
        if t > n_dec:
            lengths, ctx = lengths + [t - n_dec], ctx + [t - n_dec + 5]
        self.batch = W.build_batch(s, lengths, ctx, seed=t)
        self.layer = rs.relserve_layer_create(s)
        self.pb = rs.relserve_batch_prepare(self.layer, self.batch)
        g = _gen(seed + t + hidden)
        self.h = torch.randint(-127, 128, (t, hidden), generator=g, device="cuda", dtype=torch.int8)
        self.w = torch.randint(-127, 128, (s.qkv_dim, hidden), generator=g, device="cuda", dtype=torch.int8)
        self.hs = (0.5 + torch.rand(t, generator=g, device="cuda")) * 0.02
        self.ws = (0.5 + torch.rand(s.qkv_dim, generator=g, device="cuda")) * 0.02 / np.sqrt(hidden)
        self.packed = rs.pack_codes(self.w)

    def call(self, scratch, pools):
        q = torch.full((self.t + 3, self.shape.q_dim), 9.0, dtype=torch.bfloat16, device="cuda")
        workspace = None
        if scratch:
            workspace = torch.empty(self.rs.relserve_linear_i8_workspace_bytes(self.t, self.shape.qkv_dim), dtype=torch.uint8, device="cuda").fill_(0xff)
        self.rs.relserve_qkv_rope_append_i8(self.layer, self.pb, self.h, self.hs, self.packed, self.ws, q[:self.t], *pools, packed=True, workspace=workspace)
        torch.cuda.synchronize()
        assert bool((q[self.t:] == 9.0).all())
        return [q[:self.t].clone()] + [_bytes(p) for p in pools]

    def check(self, pools, before):
        """q and the pools' new rows against 64 bits, the pools' other rows as they were."""
        s, t, b = self.shape, self.t, self.batch
        nq, nkv, d = s.n_q_heads, s.n_kv_heads, s.head_dim
        q = self.call(True, pools)[0]
        y = ((self.h.double() @ self.w.double().t()) * self.hs.double()[:, None] * self.ws.double()).view(t, nq + 2 * nkv, d)
        pos = torch.tensor(np.concatenate([np.arange(c - n, c) for n, c in zip(np.diff(b.q_start), b.ctx_len)]), device="cuda")
        rot, size = _rotated(y[:, :nq + nkv], pos, s.rope_base), y[:, :nq + nkv].abs()
        # sums 3 U, the angle's cosine and sine 4 U, two products: of both partners; then bf16
        tol = (size + torch.cat([size[..., d // 2:], size[..., :d // 2]], -1)) * 10 * U + B * 1.01 * rot.abs()
        slots = torch.from_numpy(self.rs.relserve_batch_slots(s, b)).long().cuda()
        k, v = (p.view(-1, nkv, d)[slots].double() for p in pools)
        assert bool(((q.view(t, nq, d).double() - rot[:, :nq]).abs() <= tol[:, :nq]).all())
        assert bool(((k - rot[:, nq:]).abs() <= tol[:, nq:]).all())
        assert bool(((v - y[:, nq + nkv:]).abs() <= (B * 1.01 + 4 * U) * y[:, nq + nkv:].abs()).all())
        for pool, old in zip(pools, before):
            now, was = _bytes(pool).view(-1, nkv * d), old.view(-1, nkv * d)
            now[slots] = was[slots]
            assert torch.equal(now, was)


@pytest.mark.parametrize("t,nq,nkv,d,hidden", list(i8_paths.QKV))
def test_qkv_rope_append(rs, t, nq, nkv, d, hidden):
    """With scratch against 64 bits, and bit for bit what it gives without (where nothing is cut), over pools of either type."""
    print(f"[case] q/k/v i8 T={t} heads {nq}/{nkv} of {d}, hidden {hidden}", flush=True)
    x = Qkv(rs, t, nq, nkv, d, hidden)
    pools = _pools(x.shape, x.batch, 9, False, rs)
    x.check(pools, [_bytes(p) for p in pools])
    for fp8 in (False, True):
        got = [x.call(scratch, _pools(x.shape, x.batch, 9, fp8, rs)) for scratch in (True, False)]
        assert all(torch.equal(a, c) for a, c in zip(*got))
    x.pb.close()


@pytest.mark.parametrize("splits", [2, 4])
@pytest.mark.parametrize("tile", [0, 1, 2, 5])
def test_qkv_tails_of_every_tile(rs, tile, splits):
    """The last round of each tile shape in k ranges, which one pass adds up, scales and rotates: the bits of whole tiles."""
    for d, nq, nkv in ((128, 16, 2), (64, 24, 8)):
        x = Qkv(rs, 340, nq, nkv, d, 4096)
        want = x.call(False, _pools(x.shape, x.batch, 9, False, rs))
        print(f"[case] q/k/v i8 T=340 head_dim {d} tile {tile} tails in {splits}", flush=True)
        try:
            rs.relserve_debug_force_gemm_plan(tile, splits)
            got = x.call(True, _pools(x.shape, x.batch, 9, False, rs))
        finally:
            rs.relserve_debug_force_gemm_plan()
        assert all(torch.equal(a, c) for a, c in zip(got, want))
        x.pb.close()


@pytest.mark.parametrize("t,tile,splits", [(40, 0, 0), (100, 0, 0), (200, 0, 0)] + [(300, tile, splits) for tile in range(6) for splits in (0, 4)])
def test_largest_sums_of_the_tiled_kernels(rs, t, tile, splits):
    """Sums up to 2^31 - 2^21 and of either sign, whole and in k ranges; a forced tile keeps these few outputs off the waves' kernel, and up to 256
    tokens scratch cuts k.  (Between kernels the sums lie where floats would: small negative ones have the bits of NaNs.)"""
    k, n = 130944, 8
    a = torch.full((t, k), 127, dtype=torch.int8, device="cuda")
    w = torch.full((n, k), 127, dtype=torch.int8, device="cuda")
    w[1], w[2], a[t // 2], w[3, ::2], w[4, k // 2:] = -128, -127, -128, -127, -128
    w[5], w[5, ::64], w[6], w[6, 1::128] = 0, -1, 0, 1
    a_scale, w_scale = torch.full((t,), 2.0 ** -10, device="cuda"), torch.full((n,), 2.0 ** -12, device="cuda")
    want = (a.double() @ w.double().t()) * 2.0 ** -22
    workspace = torch.empty(rs.relserve_linear_i8_workspace_bytes(t, n), dtype=torch.uint8, device="cuda").fill_(0xff)
    out = torch.zeros((t, n), device="cuda")
    print(f"[case] largest sums T={t} tile {tile} splits {splits}", flush=True)
    try:
        rs.relserve_debug_force_gemm_plan(tile, splits)
        rs.relserve_linear_i8(a, a_scale, rs.pack_codes(w), w_scale, 1, None, out, n=n, workspace=workspace)
    finally:
        rs.relserve_debug_force_gemm_plan()
    torch.cuda.synchronize()
    assert bool(((out.double() - want).abs() <= U * want.abs()).all())     # the conversion to fp32 alone
