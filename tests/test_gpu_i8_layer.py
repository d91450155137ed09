"""The int8 layer step: bit for bit the composition of its exported stages, each of which is compared with 64 bits here or in test_gpu_i8.py;
and the whole against a 64-bit recomputation of the layer with the same quantisers."""
import numpy as np
import pytest
import torch

from paper_2601_11546_amd import workloads as W
from tests.dense_reference import rope_complex
from tests.gpu_harness import dev_bf16, gen_cache

pytestmark = pytest.mark.gpu

U, B = 2.0 ** -24, 2.0 ** -8
SHAPES = {"mha": W.LayerShape(256, 4, 4, 64, 768), "gqa": W.LayerShape(256, 4, 2, 64, 384), "g4d128": W.LayerShape(512, 4, 1, 128, 640),
          "wide": W.LayerShape(256, 2, 2, 64, 896)}     # mlp_dim as large as the step takes: 2 * 256 + 4 * 128 - 128


@pytest.fixture(scope="module")
def rs():
    from paper_2601_11546_amd import binding
    return binding


def _weights(rs, shape, seed, packed):
    w = rs.quantise_layer_weights_i8({k: dev_bf16(v) for k, v in W.make_weights(shape, seed).items()})
    return (rs.pack_layer_weights_w8a8(w) if packed else w), w


def _pools(shape, batch, seed, fp8, rs):
    if fp8:
        kp, vp = W.make_cache_fp8(shape, batch.num_pages, seed)
        return [rs.QuantPool(torch.from_numpy(np.ascontiguousarray(p)).cuda(), s) for p, s in ((kp, 0.05), (vp, 0.04))]
    kp, vp = gen_cache(shape, batch.num_pages, seed)
    return [dev_bf16(kp), dev_bf16(vp)]


def _bytes(pool):
    return (pool.codes if hasattr(pool, "codes") else pool.view(torch.int16)).clone()


def _composed(rs, layer, pb, w, x, pools, ws):
    s, t, n = layer.shape, pb.T, lambda name: w["s_" + name].shape[0] if w.get("packed") else 0

    def rows(width):
        return torch.empty(t, width, dtype=torch.int8, device="cuda"), torch.empty(t, dtype=torch.float32, device="cuda")

    def linear(codes, name, epilogue, residual, out):
        rs.relserve_linear_i8(*codes, w["w_" + name], w["s_" + name], epilogue, residual, out, n=n(name))

    h, a, act_c = rows(s.hidden), rows(s.q_dim), rows(s.mlp_dim)
    q, attn = (torch.empty(t, s.q_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x1 = torch.empty(t, s.hidden, device="cuda")
    act, y = torch.empty(t, s.mlp_dim, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    rs.relserve_add_rmsnorm_i8(x, w["w_in_norm"], s.rms_eps, *h)
    rs.relserve_qkv_rope_append_i8(layer, pb, *h, w["w_qkv"], w["s_qkv"], q, *pools, packed=bool(w.get("packed")))
    rs.relserve_attention(layer, pb, q, s.q_dim, *pools, attn, ws)
    rs.relserve_quantise_rows_i8(attn, *a)
    linear(a, "o", 1, x, x1)
    rs.relserve_add_rmsnorm_i8(x1, w["w_post_norm"], s.rms_eps, *h)
    linear(h, "gate_up", 3, None, act)
    rs.relserve_quantise_rows_i8(act, *act_c)
    linear(act_c, "down", 2, x1, y)
    torch.cuda.synchronize()
    return y


def _step_is_its_stages(rs, shape, batch, seed, packed, fp8):
    layer = rs.relserve_layer_create(shape)
    pb = rs.relserve_batch_prepare(layer, batch)
    w, _ = _weights(rs, shape, seed, packed)
    x = dev_bf16(W.make_activations(batch.T, shape.hidden, seed))
    ws = torch.empty(rs.relserve_workspace_bytes(layer, batch.T), dtype=torch.uint8, device="cuda")
    ws.fill_(0xff)
    pools = _pools(shape, batch, seed, fp8, rs)
    y = torch.empty_like(x)
    rs.relserve_layer_step_i8(layer, pb, w, x, y, *pools, ws)
    torch.cuda.synchronize()
    ref_pools = _pools(shape, batch, seed, fp8, rs)
    want = _composed(rs, layer, pb, w, x, ref_pools, ws)
    assert bool(torch.isfinite(y.float()).all())
    assert torch.equal(y, want)
    for got, ref in zip(pools, ref_pools):
        assert torch.equal(_bytes(got), _bytes(ref))
    rs.relserve_layer_step_i8(layer, pb, w, x, x, *pools, ws)      # in place; the appended rows are the same again
    torch.cuda.synchronize()
    assert torch.equal(x, want)
    pb.close()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16 cache", "8-bit cache"])
@pytest.mark.parametrize("packed", [False, True], ids=["rowmajor", "packed"])
@pytest.mark.parametrize("name", list(SHAPES))
def test_step_is_its_stages(rs, name, packed, fp8):
    shape = SHAPES[name]
    for make in (W.workload_tiny, W.workload_tiny_prefix, W.workload_tiny_long_prefixes):
        wl = make(shape=shape)
        print(f"[case] int8 step {wl.name} {name} packed={packed} fp8={fp8}: T={wl.batch.T}", flush=True)
        _step_is_its_stages(rs, shape, wl.batch, wl.seed, packed, fp8)


@pytest.mark.parametrize("n_dec,chunk", [(1, 0), (5, 0), (40, 0), (64, 0), (100, 28), (130, 126), (40, 300), (3, 700)])
def test_step_is_its_stages_at_other_sizes(rs, n_dec, chunk):
    shape = W.LayerShape(512, 4, 2, 128, 1024)
    b = W.build_batch(shape, [1] * n_dec + ([chunk] if chunk else []), [40 + 3 * i for i in range(n_dec)] + ([chunk] if chunk else []), seed=n_dec)
    print(f"[case] int8 step: {n_dec} decode rows + chunk {chunk}: T={b.T}", flush=True)
    _step_is_its_stages(rs, shape, b, 40 + n_dec, True, False)


def test_step_on_a_stream_and_captured(rs):
    shape = SHAPES["gqa"]
    wl = W.workload_tiny_prefix(shape=shape)
    layer = rs.relserve_layer_create(shape)
    pb = rs.relserve_batch_prepare(layer, wl.batch)
    w, _ = _weights(rs, shape, wl.seed, True)
    x = dev_bf16(W.make_activations(wl.batch.T, shape.hidden, wl.seed))
    pools = _pools(shape, wl.batch, wl.seed, False, rs)
    ws = torch.empty(rs.relserve_workspace_bytes(layer, wl.batch.T), dtype=torch.uint8, device="cuda")
    want, y = torch.empty_like(x), torch.empty_like(x)
    rs.relserve_layer_step_i8(layer, pb, w, x, want, *pools, ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rs.relserve_layer_step_i8(layer, pb, w, x, y, *pools, ws, stream=side)
    for _ in range(3):
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        rs.relserve_layer_step_i8(layer, pb, w, x, y, *pools, ws)
        torch.cuda.synchronize()
        assert torch.equal(y, want)


@pytest.mark.parametrize("packed", [False, True], ids=["rowmajor", "packed"])
def test_model_step_is_its_layers(rs, packed):
    """Embedding, three int8 layers, final norm and output layer of the last tokens: bit for bit the calls one by one."""
    shape, vocab, n = SHAPES["gqa"], 512, 3
    wl = W.workload_tiny_prefix(shape=shape)
    b = wl.batch
    layer = rs.relserve_layer_create(shape)
    pb = rs.relserve_batch_prepare(layer, b)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)

    def randn(*size, std=1.0, mean=0.0):
        return (torch.randn(*size, generator=g, device="cuda") * std + mean).bfloat16()

    model = {"embedding": randn(vocab, shape.hidden), "layers": [_weights(rs, shape, 50 + i, packed)[0] for i in range(n)],
             "w_final_norm": randn(shape.hidden, std=0.02, mean=1.0), "w_lm_head": randn(vocab, shape.hidden, std=0.02)}
    ids = torch.randint(0, vocab, (b.T,), generator=g, device="cuda", dtype=torch.int32)
    ws = torch.empty(rs.relserve_model_workspace_bytes(layer, b.T, b.num_reqs), dtype=torch.uint8, device="cuda")
    logits, pools = [], []
    for whole in (True, False):
        caches = [_pools(shape, b, 60 + i, False, rs) for i in range(n)]
        out = torch.empty(b.num_reqs, vocab, device="cuda")
        if whole:
            rs.relserve_model_step(layer, pb, {**model, "caches": caches}, ids, out, ws)
        else:
            x = model["embedding"][ids.long()].contiguous()
            for w, (k, v) in zip(model["layers"], caches):
                rs.relserve_layer_step_i8(layer, pb, w, x, x, k, v, ws)
            last = x[torch.from_numpy(np.asarray(b.q_start[1:], np.int64) - 1).cuda()].contiguous()
            normed = torch.empty_like(last)
            rs.relserve_rmsnorm(last, model["w_final_norm"], shape.rms_eps, normed)
            rs.relserve_linear(normed, model["w_lm_head"], 1, None, out)
        torch.cuda.synchronize()
        logits.append(out)
        pools.append([_bytes(p) for c in caches for p in c])
    pb.close()
    assert bool(torch.isfinite(logits[0]).all()) and torch.equal(*logits)
    assert all(torch.equal(a, c) for a, c in zip(*pools))


def test_refusals_launch_nothing(rs):
    """A layer that cannot be stepped is refused before the model step touches anything, and so are shapes and buffers that do not fit."""
    shape = SHAPES["gqa"]
    b = W.build_batch(shape, [3, 1], [3, 9], seed=1)
    layer = rs.relserve_layer_create(shape)
    pb = rs.relserve_batch_prepare(layer, b)
    w, _ = _weights(rs, shape, 1, True)
    x = dev_bf16(W.make_activations(b.T, shape.hidden, 1))
    pools = _pools(shape, b, 2, False, rs)
    ws = torch.zeros(rs.relserve_model_workspace_bytes(layer, b.T, b.num_reqs), dtype=torch.uint8, device="cuda")
    out = torch.full((b.num_reqs, 512), 7.0, device="cuda")
    ids = torch.zeros(b.T, dtype=torch.int32, device="cuda")
    odd = dict(w)
    odd["s_down"] = torch.zeros(shape.hidden + 1, device="cuda")[1:]     # not 16-byte aligned
    model = {"embedding": x[:1].repeat(512, 1), "layers": [w, odd], "caches": [tuple(pools)] * 2, "w_final_norm": w["w_in_norm"],
             "w_lm_head": x[:1].repeat(512, 1)}
    before = [_bytes(p) for p in pools]
    with pytest.raises(rs.RelserveError) as e:
        rs.relserve_model_step(layer, pb, model, ids, out, ws)
    assert e.value.status == -14
    # (relserve_workspace_bytes counts 256 bytes more than a step takes)
    for bad, status in ((ws[:rs.relserve_workspace_bytes(layer, b.T) - 512], -9), (ws[128:], -9)):
        with pytest.raises(rs.RelserveError) as e:
            rs.relserve_layer_step_i8(layer, pb, w, x, x, *pools, bad)
        assert e.value.status == status
    with pytest.raises(ValueError, match="w_o"):
        rs.relserve_layer_step_i8(layer, pb, {**w, "w_o": w["w_o"][:-1]}, x, x, *pools, ws)
    with pytest.raises(ValueError, match="x must"):
        rs.relserve_layer_step_i8(layer, pb, w, x[:-1], x, *pools, ws)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and bool((ws == 0).all()) and all(torch.equal(_bytes(p), o) for p, o in zip(pools, before))
    pb.close()
    for bad in (W.LayerShape(256, 4, 4, 64, 688), W.LayerShape(256, 2, 2, 64, 1024)):     # mlp_dim no multiple of 128; 2 * 256 + 4 * 128
        layer = rs.relserve_layer_create(bad)
        b = W.build_batch(bad, [2], [2], seed=1)
        pb = rs.relserve_batch_prepare(layer, b)
        wt = {n: torch.zeros(s, dtype=dt, device="cuda") for n, s, dt in [
            ("w_in_norm", (256,), torch.bfloat16), ("w_post_norm", (256,), torch.bfloat16), ("w_qkv", (bad.qkv_dim, 256), torch.int8),
            ("s_qkv", (bad.qkv_dim,), torch.float32), ("w_o", (256, bad.q_dim), torch.int8), ("s_o", (256,), torch.float32),
            ("w_gate_up", (2 * bad.mlp_dim, 256), torch.int8), ("s_gate_up", (2 * bad.mlp_dim,), torch.float32),
            ("w_down", (256, bad.mlp_dim), torch.int8), ("s_down", (256,), torch.float32)]}
        x = torch.zeros(2, 256, dtype=torch.bfloat16, device="cuda")
        pools = [torch.zeros(b.num_pages, bad.page_size, bad.n_kv_heads, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        ws = torch.zeros(rs.relserve_workspace_bytes(layer, 2), dtype=torch.uint8, device="cuda")
        with pytest.raises(rs.RelserveError) as e:
            rs.relserve_layer_step_i8(layer, pb, wt, x, x, *pools, ws)
        assert e.value.status == -14
        pb.close()


def _rotated(v, pos, base):
    """[T, heads, d] by the angles fp32(pos) * fp32(base^(-2 i / d)) in fp32, cosines in 64 bits."""
    d = v.shape[-1]
    freq = torch.tensor([float(np.float32(base)) ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64).float().cuda()
    ang = (pos.float()[:, None] * freq).double()[:, None, :]
    lo, hi = v[..., :d // 2], v[..., d // 2:]
    return torch.cat([lo * ang.cos() - hi * ang.sin(), lo * ang.sin() + hi * ang.cos()], -1)


@pytest.mark.parametrize("packed", [False, True], ids=["rowmajor", "packed"])
@pytest.mark.parametrize("name,n_dec,chunk", [("mha", 3, 0), ("g4d128", 20, 0), ("gqa", 50, 0), ("g4d128", 10, 130), ("gqa", 7, 600), ("mha", 1, 2000)])
def test_qkv_rope_append(rs, name, n_dec, chunk, packed):
    shape = SHAPES[name]
    b = W.build_batch(shape, [1] * n_dec + ([chunk] if chunk else []), [40 + 3 * i for i in range(n_dec)] + ([chunk] if chunk else []), seed=n_dec)
    print(f"[case] int8 qkv {name} T={b.T} packed={packed}", flush=True)
    layer = rs.relserve_layer_create(shape)
    pb = rs.relserve_batch_prepare(layer, b)
    w, plain = _weights(rs, shape, 7, packed)
    x = dev_bf16(W.make_activations(b.T, shape.hidden, 8))
    h, hs = torch.empty(b.T, shape.hidden, dtype=torch.int8, device="cuda"), torch.empty(b.T, device="cuda")
    rs.relserve_quantise_rows_i8(x, h, hs)
    pools = _pools(shape, b, 9, False, rs)
    before = [_bytes(p) for p in pools]
    q = torch.full((b.T + 3, shape.q_dim), 9.0, dtype=torch.bfloat16, device="cuda")
    rs.relserve_qkv_rope_append_i8(layer, pb, h, hs, w["w_qkv"], w["s_qkv"], q[:b.T], *pools, packed=packed)
    torch.cuda.synchronize()
    assert bool((q[b.T:] == 9.0).all())
    nq, nkv, d = shape.n_q_heads, shape.n_kv_heads, shape.head_dim
    y = (h.double() @ plain["w_qkv"].double().t()) * hs.double()[:, None] * plain["s_qkv"].double()
    y = y.view(b.T, nq + 2 * nkv, d)
    pos = torch.tensor(np.concatenate([np.arange(c - n, c) for n, c in zip(np.diff(b.q_start), b.ctx_len)]), device="cuda")
    rot, size = _rotated(y[:, :nq + nkv], pos, shape.rope_base), y[:, :nq + nkv].abs()
    # the second opinion's angles, in 64 bits throughout: apart by the angle's rounding, U of an angle of at most 2000
    assert torch.allclose(rot.cpu(), rope_complex(y[:, :nq + nkv].cpu(), pos.cpu(), shape.rope_base), atol=float(size.max()) * 2000 * 4 * U)
    # sums 3 U, the angle's cosine and sine 4 U, two products: of both partners; then bf16
    tol = (size + torch.cat([size[..., d // 2:], size[..., :d // 2]], -1)) * 10 * U + B * 1.01 * rot.abs()
    slots = torch.from_numpy(rs.relserve_batch_slots(shape, b)).long().cuda()
    k, v = (p.view(-1, nkv, d)[slots].double() for p in pools)
    assert bool(((q[:b.T].view(b.T, nq, d).double() - rot[:, :nq]).abs() <= tol[:, :nq]).all())
    assert bool(((k - rot[:, nq:]).abs() <= tol[:, nq:]).all())
    assert bool(((v - y[:, nq + nkv:]).abs() <= (B * 1.01 + 4 * U) * y[:, nq + nkv:].abs()).all())
    for pool, old in zip(pools, before):     # no other byte of the pools
        now, was = _bytes(pool).view(-1, nkv * d), old.view(-1, nkv * d)
        now[slots] = was[slots]
        assert torch.equal(now, was)
    # an 8-bit cache and the tiled kernels: the same bits either way
    got = []
    for force in (False, True):
        eight = _pools(shape, b, 9, True, rs)
        try:
            if force:
                rs.relserve_debug_force_gemm_plan(0, 0)
            rs.relserve_qkv_rope_append_i8(layer, pb, h, hs, w["w_qkv"], w["s_qkv"], q[:b.T], *eight, packed=packed)
        finally:
            rs.relserve_debug_force_gemm_plan()
        torch.cuda.synchronize()
        got.append([q[:b.T].clone()] + [_bytes(p) for p in eight])
    assert all(torch.equal(a, c) for a, c in zip(*got))
    pb.close()


@pytest.mark.parametrize("name,n_dec,chunk", [("mha", 3, 100), ("g4d128", 10, 150), ("gqa", 7, 600)])
def test_qkv_rope_append_on_the_tile_of_160_tokens(rs, name, n_dec, chunk):
    shape = SHAPES[name]
    b = W.build_batch(shape, [1] * n_dec + [chunk], [5 + i for i in range(n_dec)] + [chunk + 3], seed=n_dec + chunk)
    layer = rs.relserve_layer_create(shape)
    pb = rs.relserve_batch_prepare(layer, b)
    w, _ = _weights(rs, shape, 1, True)
    x = dev_bf16(W.make_activations(b.T, shape.hidden, 1))
    h, hs = torch.empty(b.T, shape.hidden, dtype=torch.int8, device="cuda"), torch.empty(b.T, device="cuda")
    rs.relserve_quantise_rows_i8(x, h, hs)
    got = []
    for tile in (0, 5):
        pools, q = _pools(shape, b, 9, False, rs), torch.zeros(b.T, shape.q_dim, dtype=torch.bfloat16, device="cuda")
        print(f"[case] q/k/v i8 {name} T={b.T} tile {tile}", flush=True)
        try:
            rs.relserve_debug_force_gemm_plan(tile, 0)
            rs.relserve_qkv_rope_append_i8(layer, pb, h, hs, w["w_qkv"], w["s_qkv"], q, *pools, packed=True)
        finally:
            rs.relserve_debug_force_gemm_plan()
        torch.cuda.synchronize()
        got.append([q] + [_bytes(p) for p in pools])
    assert all(torch.equal(a, c) for a, c in zip(*got))
    pb.close()


def _rows64(v):
    m = v.abs().amax(1, keepdim=True) / 127.0
    return torch.round(v / m) * m


def _dense_layer(shape, w, x, quantised):
    """One request's whole sequence in 64 bits on dequantised weights; quantised: every projection's input through its row quantiser, the
    attention's output and the SwiGLU product through bf16 before it."""
    def proj(a, name, sixteen=False):
        if quantised:
            a = _rows64(a.float().bfloat16().double() if sixteen else a)
        return (a @ w["w_" + name].double().t()) * w["s_" + name].double()

    def norm(a, g):
        return a / torch.sqrt(a.square().mean(1, keepdim=True) + shape.rms_eps) * g.double()

    nq, nkv, d, n = shape.n_q_heads, shape.n_kv_heads, shape.head_dim, x.shape[0]
    qkv = proj(norm(x, w["w_in_norm"]), "qkv").view(n, nq + 2 * nkv, d)
    rot = _rotated(qkv[:, :nq + nkv], torch.arange(n, device="cuda"), shape.rope_base)
    q, k, v = rot[:, :nq], rot[:, nq:].bfloat16().double(), qkv[:, nq + nkv:].bfloat16().double()
    k, v = (t.repeat_interleave(nq // nkv, 1).transpose(0, 1).contiguous() for t in (k, v))
    score = torch.bmm(q.transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) / np.sqrt(d)
    score.masked_fill_(torch.triu(torch.ones(n, n, dtype=torch.bool, device="cuda"), 1), float("-inf"))
    out = torch.bmm(torch.softmax(score, -1), v).transpose(0, 1).reshape(n, nq * d)
    x1 = x + proj(out, "o", True)
    gate, up = proj(norm(x1, w["w_post_norm"]), "gate_up").chunk(2, 1)
    return x1 + proj(gate * torch.sigmoid(gate) * up, "down", True)


@pytest.mark.parametrize("name", list(SHAPES))
def test_step_against_64_bits(rs, name):
    """Prompts prefilled, then a token each decoded.  What the two sides may differ by is the quantisers' own noise: an attention output that
    differs by a bf16 rounding, 2^-9 of it, goes to the other code in a share of that over a step (1 / 127 of the row's largest, some four
    RMS, so about one in twenty), each time by a whole step: 0.7 % of the RMS, where the quantiser's own error is 0.9 %; and the stages
    behind it see inputs that far apart.  So the deviation from the 64-bit layer with the same quantisers is held to 1.5 times the distance that
    this layer has from the one without quantisers; an unquantised or wrongly scaled input, or a lost term, is far outside."""
    shape = SHAPES[name]
    lengths = [65, 9, 130]
    w, plain = _weights(rs, shape, 3, True)
    for s_name in ("s_o", "s_down"):
        w[s_name] *= 8.0          # (both dicts hold the same tensors) a contribution of the stream's own size
    layer = rs.relserve_layer_create(shape)
    xs = [dev_bf16(W.make_activations(n, shape.hidden, 20 + i)) for i, n in enumerate(lengths)]
    whole = W.build_batch(shape, lengths, lengths, seed=1)
    pools = _pools(shape, whole, 2, False, rs)
    ws = torch.empty(rs.relserve_workspace_bytes(layer, sum(lengths)), dtype=torch.uint8, device="cuda")
    got = [torch.empty(n, shape.hidden, dtype=torch.bfloat16, device="cuda") for n in lengths]
    for part in ("prefill", "decode"):
        ctx = [n - 1 for n in lengths] if part == "prefill" else lengths
        q_len = ctx if part == "prefill" else [1] * len(lengths)
        b = W.build_batch(shape, q_len, ctx, seed=1)
        b.block_table, b.num_pages = whole.block_table, whole.num_pages
        pb = rs.relserve_batch_prepare(layer, b)
        x = torch.cat([v[:-1] if part == "prefill" else v[-1:] for v in xs]).contiguous()
        y = torch.empty_like(x)
        rs.relserve_layer_step_i8(layer, pb, w, x, y, *pools, ws)
        torch.cuda.synchronize()
        for i, rows in enumerate(torch.split(y, q_len)):
            got[i][:-1 if part == "prefill" else None][-len(rows):] = rows
        pb.close()
    for x, y in zip(xs, got):
        with_q, without = _dense_layer(shape, plain, x.double(), True), _dense_layer(shape, plain, x.double(), False)
        noise, off = float((with_q - without).norm()), float((y.double() - with_q).norm())
        own = float((without - x.double()).norm())
        bf16 = float(y.double().norm()) * B / np.sqrt(3)       # the output's own rounding
        print(f"[parity] int8 layer {name} {len(y)} tokens: off {off / own:.2e} of the layer's contribution, quantisers {noise / own:.2e}", flush=True)
        assert noise < 0.05 * own and off <= 1.5 * noise + bf16, (off, noise, bf16, own)

