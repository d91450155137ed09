"""The operators of 8-bit integer serving (W8A8 with a scale for each token and each output channel), as measurable cases.

A projection whose weights are held in 8-bit integers multiplies codes by codes; what stands around it is the making of the codes:

  op "norm"      s = x + delta (kept as the residual stream), codes of rmsnorm(s) * w with one scale per token   (relserve_add_rmsnorm_i8)
  op "quantise"  codes of the rows of a bf16 matrix with one scale per token                                    (relserve_quantise_rows_i8)
  op "linear"    out[t, n] = sum_k a[t, k] w[n, k] * (a_scale[t] * w_scale[n]), plain, onto a residual or as SwiGLU  (relserve_linear_i8)
  op "mlp"       the four calls of a feed-forward block: norm, gate/up with SwiGLU, quantise, down onto the stream

A row's scale is its largest magnitude / 127, a code the nearest integer to value / scale.  Codes are returned as the values they stand for.

Fields of a case: "tokens"; "features" = the row's length (norm, quantise), the outputs (linear; of a SwiGLU projection gate and up
together), the MLP's inner size (mlp); "k" = the depth of a product, the hidden size of an MLP; "f32": the stream is fp32 instead of bf16;
"delta": there is an addend; "epilogue": 0 bf16, 1 bf16 residual and fp32 out, 2 fp32 residual and bf16 out, 3 SwiGLU to bf16;
"packed": the weights lie in the tiled streaming layout, else row by row.
"""
import math
import random

import torch

own = False

EPS = 1e-5


def _case(name, op, tokens, features, k=0, **kw):
    c = {"name": name, "op": op, "tokens": tokens, "features": features, "k": k, "f32": False, "delta": False, "epilogue": 0, "packed": True}
    c.update(kw)
    return c


def listed():
    return [
        # four rows of a relQuery's tail decode: the launch is everything
        _case("norm_decode4", "norm", 4, 5120, delta=True),
        # the post-attention norm of a 13B layer over the headline batch (1282 tokens, fp32 stream)
        _case("norm_relquery", "norm", 1282, 5120, f32=True),
        # a prefill batch of the 70B shape with the attention's output still to be added
        _case("norm_prefill_70b", "norm", 8192, 8192, delta=True),
        # SwiGLU products of a small decode batch on their way into the down projection
        _case("quantise_decode24", "quantise", 24, 13824),
        # the same of a long prefill chunk on the 70B shape, an odd number of tokens
        _case("quantise_prefill_70b", "quantise", 4099, 28672),
        # one decoding row: the weights' stream and the latency of a nearly idle server
        _case("linear_decode1", "linear", 1, 5120, 5120, epilogue=1),
        # q/k/v of a 13B layer for a decode batch
        _case("linear_decode24_qkv", "linear", 24, 15360, 5120),
        # a shape of no model, weights as they come: odd tokens and outputs
        _case("linear_odd", "linear", 333, 1004, 1152, packed=False),
        # W_o of the headline batch
        _case("linear_relquery_o", "linear", 1282, 5120, 5120, epilogue=1),
        # the down projection of the 70B shape, decode rows beside a prefill chunk
        _case("linear_mixed_70b_down", "linear", 2304, 8192, 28672, epilogue=2),
        # gate/up of a prefill batch: the largest product of a 13B layer
        _case("linear_prefill_gate_up", "linear", 8192, 27648, 5120, epilogue=3),
        # a feed-forward block of 128 decode rows and a 512-token chunk
        _case("mlp_chunk512", "mlp", 640, 13824, 5120, f32=True, delta=True, epilogue=2),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random) -> dict:
    """The same operators at 1 .. 8192 tokens, rows of 256 .. 28672 values and products of the layers' sizes, odd ones among them."""
    op = rng.choice(["norm", "norm", "quantise", "linear", "linear", "linear", "mlp"])
    tokens = _log_int(rng, 1, 8192)
    if op == "norm":
        c = _case("", op, tokens, 8 * _log_int(rng, 32, 1024), f32=rng.random() < 0.4, delta=rng.random() < 0.6)
    elif op == "quantise":
        c = _case("", op, tokens, 8 * _log_int(rng, 32, 3584))
    elif op == "linear":
        epilogue = rng.randint(0, 3)
        c = _case("", op, tokens, 16 * _log_int(rng, 16, 3584) if epilogue == 3 else 4 * _log_int(rng, 64, 14336), 128 * _log_int(rng, 2, 224),
                  epilogue=epilogue, packed=rng.random() < 0.75)
    else:
        c = _case("", op, min(tokens, _log_int(rng, 1, 2048)), 128 * _log_int(rng, 4, 224), 128 * _log_int(rng, 2, 64), f32=True,
                  delta=rng.random() < 0.7, epilogue=2)
    del c["name"]
    top = max(_cost(x) for x in listed())
    while _cost(c) > top:    # never dearer than the largest listed case
        c["tokens"] = max(1, c["tokens"] * 3 // 4)
    return c


def work(case):
    """Every input read once, every output written once; the products' multiplications and additions (and for rows some ten operations a value)."""
    t, n, k, op = case["tokens"], case["features"], case["k"], case["op"]
    if op in ("norm", "quantise"):
        size = 4 if case["f32"] else 2
        per = size + 1 + ((2 + size) if case["delta"] else 0)
        return {"bytes": t * n * per + 4 * t + (2 * n if op == "norm" else 0), "flops": 10 * t * n}
    if op == "linear":
        out = t * n // 2 * 2 if case["epilogue"] == 3 else t * n * (4 if case["epilogue"] == 1 else 2)
        res = {0: 0, 1: 2, 2: 4, 3: 0}[case["epilogue"]] * t * n
        return {"bytes": t * k + n * k + 4 * (t + n) + out + res, "flops": 2 * t * n * k}
    stream = t * k * (4 + (2 + 4 if case["delta"] else 0) + 2)      # x, the addend and the sum, the block's output
    return {"bytes": stream + 3 * n * k + 4 * (2 * n + k) + 2 * k, "flops": 6 * t * n * k}


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 2e15)


# ---- inputs ---------------------------------------------------------------------------------------------------------------------------


def _rand(g, *size, std=1.0, mean=0.0, dtype=torch.bfloat16):
    return (torch.randn(*size, generator=g, device="cuda", dtype=torch.float32) * std + mean).to(dtype)


def _activations(g, t, n, dtype=torch.bfloat16):
    """A residual stream: normal, with every 61st channel eight times as large, as trained models have it."""
    x = torch.randn(t, n, generator=g, device="cuda", dtype=torch.float32)
    x[:, ::61] *= 8.0
    return x.to(dtype)


def _made_codes(v):
    """A program's stored codes of rows and their scales."""
    scale = v.float().abs().amax(1) / 127.0
    return torch.round(v.float() / scale[:, None]).to(torch.int8), scale


def _tiled(w):
    """[N, K] codes in the library's streaming layout: of 256 rows one after the other the slices of 128 codes, rows past N zero."""
    n, k = w.shape
    full = torch.zeros(-(-n // 256) * 256, k, dtype=w.dtype, device=w.device)
    full[:n] = w
    return full.view(-1, 256, k // 128, 128).permute(0, 2, 1, 3).contiguous().view(-1)


def _weights(g, n, k, packed, std=0.02):
    codes, scale = _made_codes(_rand(g, n, k, std=std))
    return {"codes": codes, "scale": scale, "held": _tiled(codes) if packed else codes, "n": n, "packed": packed}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t, n, k, op = case["tokens"], case["features"], case["k"], case["op"]
    stream = torch.float32 if case["f32"] else torch.bfloat16

    def empty(*size, dtype=torch.bfloat16):
        return torch.empty(*size, dtype=dtype, device="cuda")

    st = {"case": case}
    if op in ("norm", "mlp"):
        h = n if op == "norm" else k
        st["x"], st["w_norm"] = _activations(g, t, h, stream), _rand(g, h, std=0.02, mean=1.0)
        st["delta"] = _rand(g, t, h, std=0.5) if case["delta"] else None
        st["sum"] = empty(t, h, dtype=stream) if case["delta"] else None
        st["codes"], st["scale"] = empty(t, h, dtype=torch.int8), empty(t, dtype=torch.float32)
    if op == "quantise":
        st["x"] = _activations(g, t, n)
        st["codes"], st["scale"] = empty(t, n, dtype=torch.int8), empty(t, dtype=torch.float32)
    if op in ("norm", "quantise"):
        st["values"] = empty(t, n)
    if op in ("linear", "mlp"):
        st["workspace"] = empty(64 << 20, dtype=torch.uint8)      # the program's one scratch for its projections
    if op == "linear":
        st["a"], st["a_scale"] = _made_codes(_activations(g, t, k))
        st["w"] = _weights(g, n, k, case["packed"])
        e = case["epilogue"]
        st["residual"] = _rand(g, t, n, dtype=torch.bfloat16 if e == 1 else torch.float32) if e in (1, 2) else None
        st["out"] = empty(t, n // 2 if e == 3 else n, dtype=torch.float32 if e == 1 else torch.bfloat16)
    if op == "mlp":
        st["gate_up"], st["down"] = _weights(g, 2 * n, k, case["packed"]), _weights(g, k, n, case["packed"], std=0.02 / math.sqrt(80))
        st["act"], st["act_codes"], st["act_scale"] = empty(t, n), empty(t, n, dtype=torch.int8), empty(t, dtype=torch.float32)
        st["out"] = empty(t, k)
    return st


# ---- the operators in elementary operations ---------------------------------------------------------------------------------------------


def _plain_rows(v):
    """Codes (as fp32 integers) and scales of fp32 rows."""
    scale = v.abs().amax(1, keepdim=True) / 127.0
    return torch.round(v / scale), scale


def _plain_norm(x, delta, w):
    s = x if delta is None else (x.float() + delta.float()).to(x.dtype)
    f = s.float()
    return s, f * torch.rsqrt(f.square().mean(1, keepdim=True) + EPS) * w.float()


def _plain_linear(a, a_scale, w, epilogue, residual):
    y = (a @ w["codes"].float().t()) * (a_scale * w["scale"])
    if epilogue == 3:
        gate, up = y.chunk(2, 1)
        return (gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16)
    if residual is not None:
        y = y + residual.float()
    return y if epilogue == 1 else y.to(torch.bfloat16)


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "linear":
        return {"out": _plain_linear(st["a"].float(), st["a_scale"][:, None], st["w"], case["epilogue"], st["residual"])}
    if op == "quantise":
        codes, scale = _plain_rows(st["x"].float())
        return {"values": (codes * scale).to(torch.bfloat16), "scale": scale.flatten()}
    s, normed = _plain_norm(st["x"], st["delta"], st["w_norm"])
    codes, scale = _plain_rows(normed)
    kept = {} if st["delta"] is None else {"sum": s}
    if op == "norm":
        return {"values": (codes * scale).to(torch.bfloat16), "scale": scale.flatten(), **kept}
    act = _plain_linear(codes, scale, st["gate_up"], 3, None)
    codes, scale = _plain_rows(act.float())
    return {"out": _plain_linear(codes, scale, st["down"], 2, s), **kept}


# ---- the framework's calls ------------------------------------------------------------------------------------------------------------


def _own(st):
    from paper_2601_11546_amd import binding as rs
    case, op = st["case"], st["case"]["op"]

    def linear(a, a_scale, w, epilogue, residual, out):
        rs.relserve_linear_i8(a, a_scale, w["held"], w["scale"], epilogue, residual, out, n=w["n"] if w["packed"] else 0,
                              workspace=st["workspace"])

    if op == "linear":
        linear(st["a"], st["a_scale"], st["w"], case["epilogue"], st["residual"], st["out"])
        return {"out": st["out"]}
    if op == "quantise":
        rs.relserve_quantise_rows_i8(st["x"], st["codes"], st["scale"])
        return {"values": torch.mul(st["codes"], st["scale"][:, None], out=st["values"]), "scale": st["scale"]}
    rs.relserve_add_rmsnorm_i8(st["x"], st["w_norm"], EPS, st["codes"], st["scale"], delta=st["delta"], sum_out=st["sum"])
    kept = {} if st["delta"] is None else {"sum": st["sum"]}
    if op == "norm":
        return {"values": torch.mul(st["codes"], st["scale"][:, None], out=st["values"]), "scale": st["scale"], **kept}
    stream = st["x"] if st["delta"] is None else st["sum"]
    linear(st["codes"], st["scale"], st["gate_up"], 3, None, st["act"])
    rs.relserve_quantise_rows_i8(st["act"], st["act_codes"], st["act_scale"])
    linear(st["act_codes"], st["act_scale"], st["down"], 2, stream, st["out"])
    return {"out": st["out"], **kept}


def run(st):
    return _own(st) if own else _plain(st)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------------------


def _exact_rows(v):
    top = torch.maximum(v.max(dim=1).values, -v.min(dim=1).values).unsqueeze(1)
    step = top / 127
    return step, (v * 127 / top).round()


def _exact_product(codes, step, w):
    sums = torch.matmul(codes, w["codes"].to(torch.float64).transpose(0, 1).contiguous())
    return sums.mul_(step).mul_(w["scale"].to(torch.float64)[None])


def _exact_swiglu(y):
    half = y.shape[1] // 2
    gate = y[:, :half]
    return gate * torch.sigmoid(gate) * y[:, half:]


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "linear":
        y = _exact_product(st["a"].to(torch.float64), st["a_scale"].to(torch.float64).unsqueeze(1), st["w"])
        if case["epilogue"] == 3:
            y = _exact_swiglu(y)
        elif st["residual"] is not None:
            y += st["residual"].to(torch.float64)
        return {"out": y}
    if op == "quantise":
        step, codes = _exact_rows(st["x"].to(torch.float64))
        return {"values": codes * step, "scale": step.squeeze(1)}
    total = st["x"].to(torch.float64)
    if st["delta"] is not None:
        total = total + st["delta"].to(torch.float64)
    stored = total.to(st["x"].dtype).to(torch.float64)      # the norm reads the stream as it is kept
    root = torch.sqrt((stored * stored).sum(dim=1, keepdim=True) / stored.shape[1] + EPS)
    step, codes = _exact_rows(stored * st["w_norm"].to(torch.float64)[None] / root)
    kept = {} if st["delta"] is None else {"sum": total}
    if op == "norm":
        return {"values": codes * step, "scale": step.squeeze(1), **kept}
    act = _exact_swiglu(_exact_product(codes, step, st["gate_up"]))
    step, codes = _exact_rows(act.to(torch.bfloat16).to(torch.float64))
    return {"out": _exact_product(codes, step, st["down"]) + stored, **kept}
