"""The operators that answer from a checkpoint held in 8-bit floating point with a scale for each block of 128, as measurable cases.

Matrices of such a checkpoint hold codes of 1 sign, 4 exponent and 3 mantissa bits with one fp32 scale per block of 128 outputs x 128 inputs;
activations get a scale for each 128 values of a token on the way.  A serving program makes codes, multiplies them, and reads from the
logits how sure the model is of its answers:

  op "quantise"  codes and scales of the rows of a bf16 matrix, in blocks of 1 or 128 rows x 128 values           (relserve_quantise_f8b)
  op "norm"      s = x + delta (kept as the residual stream), codes and scales of rmsnorm(s) * w in blocks of 128  (relserve_add_rmsnorm_f8b)
  op "linear"    out[t, n] = sum over blocks b of k of (sum of a[t, k] w[n, k]) * a_scale[b, t] * w_scale[n / 128, b], plain, onto a residual or
                 as SwiGLU                                                                                        (relserve_linear_f8b)
  op "logprobs"  of rows of logits: log probabilities of given tokens, entropy, the top alternatives              (relserve_logprobs)
  op "answers"   the end of a model over a relQuery's rows: final norm, output layer, log probabilities of each row's labels

A block's scale is its largest magnitude / 448, a code the nearest number of the format to value / scale.  Scales of tokens lie block by block,
[k / 128, tokens].  Codes are returned as numbers of torch's type of that format, beside their scales.

Fields of a case: "tokens" = rows; "features" = the row's length (quantise, norm), the outputs (linear; of a SwiGLU projection gate and up
together), the vocabulary (logprobs, answers); "k" = the depth of a product, the hidden size; "block_rows" = rows of a quantised block; "f32":
the stream, or the logits, are fp32 instead of bf16; "delta": there is an addend; "epilogue": 0 bf16, 1 bf16 residual (answers: none) and fp32
out, 2 fp32 residual and bf16 out, 3 SwiGLU to bf16; "packed": weights in the tiled streaming layout, else row by row; "given", "top": tokens
a row is asked for, alternatives a row returns.
"""
import math
import random

import torch

own = False

EPS = 1e-5
LARGEST = 448.0
CODE = torch.float8_e4m3fn


def _case(name, op, tokens, features, k=0, **kw):
    c = {"name": name, "op": op, "tokens": tokens, "features": features, "k": k, "block_rows": 1, "f32": False, "delta": False, "epilogue": 0,
         "packed": True, "given": 0, "top": 0}
    c.update(kw)
    return c


def listed():
    return [
        # four rows of a relQuery's tail decode: the launch is everything
        _case("norm_decode4", "norm", 4, 5120, delta=True),
        # the post-attention norm of a prefill batch on the 70B shape, an odd number of tokens, fp32 stream
        _case("norm_prefill_70b", "norm", 4099, 8192, f32=True, delta=True),
        # SwiGLU products of the headline batch on their way into the down projection of a 13B layer
        _case("quantise_relquery", "quantise", 1282, 13824),
        # a 16-bit gate/up matrix converted when a model is loaded
        _case("quantise_weights", "quantise", 27648, 5120, block_rows=128),
        # one decoding row: the weights' stream and the latency of a nearly idle server
        _case("linear_decode1", "linear", 1, 5120, 5120, epilogue=1),
        # q/k/v of a 13B layer for a decode batch
        _case("linear_decode24_qkv", "linear", 24, 15360, 5120),
        # a shape of no model, weights as they come: odd tokens, outputs that end inside a block
        _case("linear_odd", "linear", 333, 1004, 1152, packed=False, epilogue=2),
        # W_o of the headline batch
        _case("linear_relquery_o", "linear", 1282, 5120, 5120, epilogue=1),
        # gate/up of a prefill batch: the largest product of a 13B layer
        _case("linear_prefill_gate_up", "linear", 8192, 27648, 5120, epilogue=3),
        # the next tokens of a decode batch with five alternatives each, logits as a model step leaves them
        _case("logprobs_decode24", "logprobs", 24, 32000, f32=True, given=1, top=5),
        # a prompt scored token by token, 16-bit logits of an odd vocabulary
        _case("logprobs_prompt", "logprobs", 2048, 50257, given=1, top=20),
        # 200 rows of a relQuery: how likely each of the query's four labels is
        _case("answers_relquery", "answers", 200, 32000, 5120, delta=True, epilogue=1, given=4),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random) -> dict:
    """The same operators at 1 .. 8192 tokens, rows of 256 .. 28672 values, products of the layers' sizes and vocabularies of 1000 .. 160000."""
    op = rng.choice(["norm", "quantise", "linear", "linear", "linear", "linear", "logprobs", "logprobs", "answers"])
    tokens = _log_int(rng, 1, 8192)
    if op == "norm":
        c = _case("", op, tokens, 128 * _log_int(rng, 2, 64), f32=rng.random() < 0.5, delta=rng.random() < 0.6)
    elif op == "quantise":
        c = _case("", op, tokens, 128 * _log_int(rng, 2, 224), block_rows=rng.choice([1, 1, 128]))
    elif op == "linear":
        epilogue = rng.randint(0, 3)
        c = _case("", op, tokens, 16 * _log_int(rng, 16, 3584) if epilogue == 3 else 4 * _log_int(rng, 64, 14336), 128 * _log_int(rng, 2, 224),
                  epilogue=epilogue, packed=rng.random() < 0.75)
    elif op == "logprobs":
        c = _case("", op, min(tokens, 4096), _log_int(rng, 1000, 160000), f32=rng.random() < 0.7, given=rng.choice([1, 1, 2, 4]), top=rng.choice([0, 1, 5, 20]))
    else:
        c = _case("", op, min(tokens, 512), 4 * _log_int(rng, 2000, 40000), 128 * _log_int(rng, 8, 64), delta=rng.random() < 0.7,
                  epilogue=1, given=rng.choice([1, 2, 4]))
    del c["name"]
    top = max(_cost(x) for x in listed())
    while _cost(c) > top:    # never dearer than the largest listed case
        c["tokens"] = max(1, c["tokens"] * 3 // 4)
    return c


def work(case):
    """Every input read once, every output written once; the products' multiplications and additions (and some ten operations a value elsewhere)."""
    t, n, k, op = case["tokens"], case["features"], case["k"], case["op"]
    size = 4 if case["f32"] else 2

    def norm(h):
        return t * h * (size + 1 + (2 + size if case["delta"] else 0)) + t * h // 32 + 2 * h

    def linear(residual):
        out = t * n // 2 * 2 if case["epilogue"] == 3 else t * n * (4 if case["epilogue"] == 1 else 2)
        return t * k + n * k + t * k // 32 + n * k // 4096 + out + residual

    if op == "norm":
        return {"bytes": norm(n), "flops": 10 * t * n}
    if op == "quantise":
        return {"bytes": 3 * t * n + 4 * t * n // (128 * case["block_rows"]), "flops": 10 * t * n}
    if op == "linear":
        return {"bytes": linear({0: 0, 1: 2, 2: 4, 3: 0}[case["epilogue"]] * t * n), "flops": 2 * t * n * k}
    few = 8 * t * (case["given"] + case["top"]) + 4 * t
    if op == "logprobs":
        return {"bytes": t * n * size + few, "flops": 10 * t * n}
    return {"bytes": norm(k) + linear(0) + 4 * t * n + few, "flops": 2 * t * n * k + 10 * t * n}


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


def _logits(g, t, n, dtype):
    """Rows as a model leaves them: most tokens alike, some sixty far ahead, and rows from nearly undecided to nearly sure."""
    x = torch.randn(t, n, generator=g, device="cuda", dtype=torch.float32) * 1.5 - 4.0
    ahead = torch.randint(0, n, (t, 60), generator=g, device="cuda")
    sure = torch.rand(t, 1, generator=g, device="cuda") * 4.0
    x.scatter_add_(1, ahead, torch.randn(t, 60, generator=g, device="cuda") * sure + 6.0)
    return x.to(dtype)


def _made_codes(v):
    """A program's stored codes of a token's blocks and their scales, [k / 128, tokens]."""
    t, k = v.shape
    b = v.float().view(t, k // 128, 128)
    scale = b.abs().amax(2) / LARGEST
    return (b / scale[:, :, None]).clamp(-LARGEST, LARGEST).to(CODE).view(t, k), scale.t().contiguous()


def _tiled(w):
    """[N, K] codes in the library's streaming layout: of 256 rows one after the other the slices of 128 codes, rows past N zero."""
    n, k = w.shape
    full = torch.zeros(-(-n // 256) * 256, k, dtype=torch.uint8, device=w.device)
    full[:n] = w.view(torch.uint8)
    return full.view(-1, 256, k // 128, 128).permute(0, 2, 1, 3).contiguous().view(-1)


def _block_codes(w):
    n, k = w.shape
    full = torch.zeros(-(-n // 128) * 128, k, dtype=torch.float32, device=w.device)
    full[:n] = w.float()
    b = full.view(-1, 128, k // 128, 128)
    scale = b.abs().amax((1, 3)) / LARGEST
    return (b / scale[:, None, :, None]).clamp(-LARGEST, LARGEST).to(CODE).view(-1, k)[:n].contiguous(), scale


def _weights(g, n, k, packed, swiglu=False, std=0.02):
    """Codes of a matrix in blocks of 128 x 128; of a gate and an up matrix one behind the other, each in blocks of its own."""
    if swiglu:
        gate, up = _block_codes(_rand(g, n // 2, k, std=std)), _block_codes(_rand(g, n // 2, k, std=std))
        codes, scale = torch.cat([gate[0].view(torch.uint8), up[0].view(torch.uint8)]).view(CODE), torch.cat([gate[1], up[1]])
    else:
        codes, scale = _block_codes(_rand(g, n, k, std=std))
    return {"codes": codes, "scale": scale, "held": _tiled(codes) if packed else codes, "n": n, "packed": packed}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t, n, k, op = case["tokens"], case["features"], case["k"], case["op"]
    stream = torch.float32 if case["f32"] else torch.bfloat16

    def empty(*size, dtype=torch.bfloat16):
        return torch.empty(*size, dtype=dtype, device="cuda")

    st = {"case": case}
    if op in ("norm", "answers"):
        h = n if op == "norm" else k
        st["x"], st["w_norm"] = _activations(g, t, h, stream), _rand(g, h, std=0.02, mean=1.0)
        st["delta"] = _rand(g, t, h, std=0.5) if case["delta"] else None
        st["sum"] = empty(t, h, dtype=stream) if case["delta"] else None
        st["codes"], st["scale"] = empty(t, h, dtype=CODE), empty(h // 128, t, dtype=torch.float32)
    if op == "quantise":
        st["x"] = _rand(g, t, n, std=0.02) if case["block_rows"] == 128 else _activations(g, t, n)
        st["codes"] = empty(t, n, dtype=CODE)
        st["scale"] = empty(*((-(-t // 128), n // 128) if case["block_rows"] == 128 else (n // 128, t)), dtype=torch.float32)
    if op in ("linear", "answers", "logprobs"):
        st["workspace"] = empty(64 << 20, dtype=torch.uint8)      # the program's one scratch
    if op == "linear":
        e = case["epilogue"]
        st["a"], st["a_scale"] = _made_codes(_activations(g, t, k))
        st["w"] = _weights(g, n, k, case["packed"], swiglu=e == 3)
        st["residual"] = _rand(g, t, n, dtype=torch.bfloat16 if e == 1 else torch.float32) if e in (1, 2) else None
        st["out"] = empty(t, n // 2 if e == 3 else n, dtype=torch.float32 if e == 1 else torch.bfloat16)
    if op == "answers":
        st["w"] = _weights(g, n, k, case["packed"])
        st["logits"] = empty(t, n, dtype=torch.float32)
    if op == "logprobs":
        st["logits"] = _logits(g, t, n, stream)
    if op in ("logprobs", "answers"):
        st["ids"] = torch.randint(0, n, (t, case["given"]), generator=g, device="cuda", dtype=torch.int32)
        st["logprob"], st["entropy"] = empty(t, case["given"], dtype=torch.float32), empty(t, dtype=torch.float32)
        st["top_ids"], st["top_logprob"] = empty(t, case["top"], dtype=torch.int32), empty(t, case["top"], dtype=torch.float32)
    return st


# ---- the operators in elementary operations ---------------------------------------------------------------------------------------------


def _plain_codes(v, block_rows):
    """Of fp64 values: a quotient halfway between two codes has to come out as that, and 32-bit division is not exact everywhere."""
    t, n = v.shape
    if block_rows == 1:
        b = v.view(t, n // 128, 128)
        top = b.abs().amax(2, keepdim=True)
        return (b * LARGEST / top).float().to(CODE).view(t, n), (top.squeeze(2) / LARGEST).t().float().contiguous()
    rows = -(-t // 128) * 128
    b = torch.cat([v, v.new_zeros(rows - t, n)]).view(-1, 128, n // 128, 128) if rows > t else v.view(-1, 128, n // 128, 128)
    top = b.abs().amax((1, 3), keepdim=True)
    return (b * LARGEST / top).float().to(CODE).view(rows, n)[:t], (top.view(-1, n // 128) / LARGEST).float()


def _plain_norm(x, delta, w):
    """The stream, and its codes: the values less the factor that a whole row shares, which goes into the scales."""
    s = x if delta is None else (x.float() + delta.float()).to(x.dtype)
    f = s.float()
    codes, scale = _plain_codes((f * w.float()).double(), 1)
    return s, codes, scale * torch.rsqrt(f.square().mean(1) + EPS)[None]


def _plain_linear(a, a_scale, w, epilogue, residual):
    t, k = a.shape
    n = w["n"]
    half = n // 2 if epilogue == 3 else n
    scale = w["scale"].view(n // half, -1, k // 128).repeat_interleave(128, 1)[:, :half].reshape(n, k // 128)
    held = (w["codes"].float().view(n, k // 128, 128) * scale[:, :, None]).view(n, k)
    y = (a.float().view(t, k // 128, 128) * a_scale.t()[:, :, None]).view(t, k) @ held.t()
    if epilogue == 3:
        gate, up = y.chunk(2, 1)
        return (gate / (1.0 + torch.exp(-gate)) * up).to(torch.bfloat16)
    if residual is not None:
        y = y + residual.float()
    return y if epilogue == 1 else y.to(torch.bfloat16)


def _plain_logprobs(logits, ids, top):
    x = logits.float()
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    lse = m.double() + total.log()
    out = {"logprob": (x.gather(1, ids.long()).double() - lse).float(),
           "entropy": (total.log().squeeze(1) - ((x - m).double() * e).sum(1) / total.squeeze(1)).float()}
    if top:
        values, order = torch.sort(x, dim=1, descending=True, stable=True)
        out["top_ids"], out["top_logprob"] = order[:, :top].to(torch.int32), (values[:, :top].double() - lse).float()
    return out


def _plain(st):
    case, op = st["case"], st["case"]["op"]
    if op == "quantise":
        codes, scale = _plain_codes(st["x"].double(), case["block_rows"])
        return {"codes": codes, "scale": scale}
    if op == "linear":
        return {"out": _plain_linear(st["a"], st["a_scale"], st["w"], case["epilogue"], st["residual"])}
    if op == "logprobs":
        return _plain_logprobs(st["logits"], st["ids"], case["top"])
    s, codes, scale = _plain_norm(st["x"], st["delta"], st["w_norm"])
    kept = {} if st["delta"] is None else {"sum": s}
    if op == "norm":
        return {"codes": codes, "scale": scale, **kept}
    logits = _plain_linear(codes, scale, st["w"], 1, None)
    return {"logits": logits, **_plain_logprobs(logits, st["ids"], case["top"]), **kept}


# ---- the framework's calls ------------------------------------------------------------------------------------------------------------


def _own(st):
    from paper_2601_11546_amd import binding as rs
    case, op = st["case"], st["case"]["op"]

    def linear(a, a_scale, w, epilogue, residual, out):
        rs.relserve_linear_f8b(a, a_scale, w["held"], w["scale"], epilogue, residual, out, n=w["n"] if w["packed"] else 0,
                               workspace=st["workspace"])

    def logprobs():
        rs.relserve_logprobs(st["logits"], ids=st["ids"], logprobs=st["logprob"], entropy=st["entropy"],
                             top_ids=st["top_ids"] if case["top"] else None, top_logprobs=st["top_logprob"] if case["top"] else None,
                             workspace=st["workspace"])
        out = {"logprob": st["logprob"], "entropy": st["entropy"]}
        return {**out, "top_ids": st["top_ids"], "top_logprob": st["top_logprob"]} if case["top"] else out

    if op == "quantise":
        rs.relserve_quantise_f8b(st["x"], st["codes"], st["scale"], block_rows=case["block_rows"])
        return {"codes": st["codes"], "scale": st["scale"]}
    if op == "linear":
        linear(st["a"], st["a_scale"], st["w"], case["epilogue"], st["residual"], st["out"])
        return {"out": st["out"]}
    if op == "logprobs":
        return logprobs()
    rs.relserve_add_rmsnorm_f8b(st["x"], st["w_norm"], EPS, st["codes"], st["scale"], delta=st["delta"], sum_out=st["sum"])
    kept = {} if st["delta"] is None else {"sum": st["sum"]}
    if op == "norm":
        return {"codes": st["codes"], "scale": st["scale"], **kept}
    linear(st["codes"], st["scale"], st["w"], 1, None, st["logits"])
    return {"logits": st["logits"], **logprobs(), **kept}


def run(st):
    return _own(st) if own else _plain(st)


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------------------------


def _nearest_code(v):
    """The number of 4 exponent and 3 mantissa bits nearest to each value of [-448, 448], ties to the even one."""
    _, exponent = torch.frexp(v)
    step = torch.tensor([2.0 ** i for i in range(-9, 6)], dtype=torch.float64, device=v.device)[(exponent.long() - 4).clamp(-9, 5) + 9]
    return torch.round(v / step) * step


def _exact_codes(v, block_rows):
    rows, n = v.shape
    blocks = -(-rows // block_rows)
    top = torch.zeros(blocks * block_rows, n // 128, dtype=torch.float64, device=v.device)
    top[:rows] = torch.maximum(v.unflatten(1, (-1, 128)).max(dim=2).values, -v.unflatten(1, (-1, 128)).min(dim=2).values)
    top = top.unflatten(0, (-1, block_rows)).max(dim=1).values
    each = top.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)
    return _nearest_code(v * 448 / each), top / 448


def _exact_values(w, k, half):
    """A matrix as the numbers that its codes and scales stand for."""
    row = torch.arange(w["n"], device=w["codes"].device)
    block = torch.where(row < half, row // 128, -(-half // 128) + (row - half) // 128)
    return w["codes"].to(torch.float64) * w["scale"].to(torch.float64)[block].repeat_interleave(128, 1)


def _exact_product(codes, step, w, half):
    values = codes * step.transpose(0, 1).repeat_interleave(128, 1)
    return torch.matmul(values, _exact_values(w, codes.shape[1], half).transpose(0, 1).contiguous())


def _exact_answers(logits, ids, top):
    p = torch.log_softmax(logits, dim=1)
    at = {"logprob": torch.gather(p, 1, ids.to(torch.int64)), "entropy": torch.special.entr(p.exp()).sum(dim=1)}
    if top:
        at["top_ids"], at["top_logprob"] = None, torch.topk(p, top, dim=1).values
    return at


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "quantise":
        codes, scale = _exact_codes(st["x"].to(torch.float64), case["block_rows"])
        return {"codes": codes, "scale": scale.transpose(0, 1).contiguous() if case["block_rows"] == 1 else scale}
    if op == "linear":
        half = st["w"]["n"] // 2 if case["epilogue"] == 3 else st["w"]["n"]
        y = _exact_product(st["a"].to(torch.float64), st["a_scale"].to(torch.float64), st["w"], half)
        if case["epilogue"] == 3:
            y = y[:, :half] * torch.sigmoid(y[:, :half]) * y[:, half:]
        elif st["residual"] is not None:
            y += st["residual"].to(torch.float64)
        return {"out": y}
    if op == "logprobs":
        return _exact_answers(st["logits"].to(torch.float64), st["ids"], case["top"])
    total = st["x"].to(torch.float64)
    if st["delta"] is not None:
        total = total + st["delta"].to(torch.float64)
    stored = total.to(st["x"].dtype).to(torch.float64)      # the norm reads the stream as it is kept
    root = torch.sqrt((stored * stored).sum(dim=1, keepdim=True) / stored.shape[1] + EPS)
    codes, scale = _exact_codes(stored * st["w_norm"].to(torch.float64)[None], 1)     # (the root is of a whole row: it leaves the codes alone)
    scale = (scale / root).transpose(0, 1).contiguous()
    kept = {} if st["delta"] is None else {"sum": total}
    if op == "norm":
        return {"codes": codes, "scale": scale, **kept}
    logits = _exact_product(codes, scale, st["w"], st["w"]["n"])
    return {"logits": logits, **_exact_answers(logits, st["ids"], case["top"]), **kept}
