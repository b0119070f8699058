"""Cases for the operators around a linear layer in microscaled 4-bit floating point: quantization in blocks of 32 with a power-of-two scale,
the product of such operands with the layer's forward and backward pass, and the root-mean-square norm with the residual's addition that
hands a layer its rows, quantized or not.  Their inputs, the work they cannot do without, the same results in elementary torch operations
in 32 bits, and from the definition in 64.

Kinds of cases (`op`):
  quantize    ssg_mx4_quantize and ssg_mx4_dequantize: a matrix, or its transpose, in 4 bits; the values that its codes stand for
  linear      ssg_mx4_linear: rows of x quantized in the call, times 4-bit weights
  linear_bwd  ssg_mx4_linear_bwd: the gradients with respect to x and the weights
  norm        ssg_rmsnorm_fwd: residual's addition, norm, and rows as bf16, E4M3 with a given scale, or 8- and 4-bit rows that a product reads
  norm_bwd    ssg_rmsnorm_bwd: the gradients with respect to x, the residual and the weights
All inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
BLOCK = 32                                   # neighbours that share a scale
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


# ---------------------------------------------------------------- the cases
def _quantize_case(rows, K, x="bf16", transposed=0, rule="floor"):
    return {"op": "quantize", "rows": rows, "K": K, "x": x, "transposed": transposed, "rule": rule}


def _linear(M, K, N, x="bf16", y="bf16", rule="floor"):
    return {"op": "linear", "M": M, "K": K, "N": N, "x": x, "y": y, "rule": rule}


def _linear_bwd(M, K, N, dy="bf16", x="bf16", dw="f32", rule="floor"):
    return {"op": "linear_bwd", "M": M, "K": K, "N": N, "dy": dy, "x": x, "dw": dw, "rule": rule}


def _norm(T, d, x="bf16", r="none", w="bf16", out="bf16", N=0, gap=0, offset=0.0, rule="floor"):
    """r: the residual's type, or none; N: columns of the product that reads 8- or 4-bit rows; gap: elements between two rows of x."""
    return {"op": "norm", "T": T, "d": d, "x": x, "r": r, "w": w, "out": out, "N": N, "gap": gap, "offset": offset, "rule": rule}


def _norm_bwd(T, d, x="bf16", r="none", w="bf16", dy="bf16", offset=0.0):
    return {"op": "norm_bwd", "T": T, "d": d, "x": x, "r": r, "w": w, "dy": dy, "offset": offset}


def listed():
    return [
        # activations of a decode batch, odd sizes: nothing but latency
        {"name": "quantize_batch", **_quantize_case(75, 2736, "f32")},
        # an operand of a weight gradient at the 7B widths: activations of a micro-batch in blocks along the tokens
        {"name": "quantize_transposed", **_quantize_case(11008, 4096, transposed=1)},
        # decoding at the 7B widths, up projection: one token, the weights' bytes
        {"name": "mx4_token", **_linear(1, 4096, 11008)},
        # a mixed batch of odd size and odd widths, scales that let nothing saturate, results in fp32
        {"name": "mx4_odd", **_linear(333, 2736, 1040, "f32", "f32", "ceil")},
        # a prefill at the 7B widths, down projection
        {"name": "mx4_prefill", **_linear(4096, 11008, 4096)},
        # the backward pass of a short ragged micro-batch through a narrow layer, weight gradients kept in bf16
        {"name": "mx4_bwd_odd", **_linear_bwd(777, 1376, 2064, x="f32", dw="bf16")},
        # the backward pass of a micro-batch at the 7B widths, up projection
        {"name": "mx4_bwd_large", **_linear_bwd(4096, 4096, 11008)},
        # one token's residual and norm before a product in E4M3 under delayed scaling: nothing but latency
        {"name": "norm_token", **_norm(1, 4096, r="bf16", out="e4m3")},
        # the heads' norm of queries inside wider rows: many short rows
        {"name": "norm_heads", **_norm(131072, 128, w="f32", gap=128)},
        # a prefill at the 7B widths: residual in fp32, norm, 4-bit rows and the up projection that reads them
        {"name": "norm_mx4_prefill", **_norm(4096, 4096, r="f32", out="mx4", N=11008)},
        # the gradient in a short ragged micro-batch, all in fp32, weights stored around zero
        {"name": "norm_bwd_odd", **_norm_bwd(1023, 2736, "f32", "f32", "f32", "f32", 1.0)},
        # the gradient in a micro-batch at the 7B widths
        {"name": "norm_bwd_large", **_norm_bwd(16384, 4096, r="bf16")},
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "linear", "linear_bwd", "linear_bwd", "norm", "norm", "norm", "norm_bwd", "norm_bwd"])
    two, rule = ["bf16", "bf16", "f32"], rng.choice(["floor", "ceil"])
    if op == "quantize":
        t = rng.randrange(2)
        return _quantize_case(_log(rng, 16, 11008, 16) if t else _log(rng, 1, 11008), _log(rng, 1, 4096) if t else _log(rng, 64, 4096, 16), rng.choice(two), t, rule)
    if op == "linear":
        return _linear(_log(rng, 1, 4096), _log(rng, 256, 11008, rng.choice([16, 128])), _log(rng, 256, 4096, rng.choice([16, 128])), rng.choice(two),
                       rng.choice(two), rule)
    if op == "linear_bwd":
        return _linear_bwd(_log(rng, 16, 4096), _log(rng, 256, 4096, rng.choice([16, 128])), _log(rng, 256, 11008, rng.choice([16, 128])), rng.choice(two),
                           rng.choice(two), rng.choice(two), rule)
    r, offset = rng.choice(["none", "bf16", "f32"]), rng.choice([0.0, 1.0])
    d = _log(rng, 64, 8192, rng.choice([16, 64]))
    if op == "norm_bwd":
        return _norm_bwd(_log(rng, 1, min(131072, 16384 * 4096 // d)), d, rng.choice(two), r, rng.choice(two), rng.choice(two), offset)
    out = rng.choice(["bf16", "f32", "e4m3", "e4m3", "i8", "mx4", "mx4"])
    product = out in ("i8", "mx4")
    return _norm(_log(rng, 1, 4096 if product else min(131072, 16384 * 4096 // d)), d, rng.choice(two), r, rng.choice(two), out,
                 _log(rng, 256, 4096, 16) if product else 0, rng.choice([0, 0, 64]), offset, rule)


# ---------------------------------------------------------------- inputs, from the seed alone
def _activations(gen, rows, cols, dtype, gap=0):
    """Rows of different magnitude, a few of the channels far larger than the others."""
    x = torch.randn((rows, cols), generator=gen, device=DEV)
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device=DEV))
    x[:, torch.randperm(cols, generator=gen, device=DEV)[:4]] *= 8.0
    wide = torch.zeros((rows, cols + gap), device=DEV, dtype=DTYPE[dtype])
    wide[:, :cols] = x
    return wide


def _fill(x, to):
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % to))


def _mx4(x, rule):
    """Values 0, .5, 1, 1.5, 2, 3, 4, 6 with their signs, and a power of two for 32 neighbours along the last axis, in 32 bits."""
    v = _fill(x.float(), BLOCK).unflatten(-1, (-1, BLOCK))
    amax = v.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(amax)                                 # amax = m 2^e, m from .5 to 1
    e = torch.where(amax > 0, e - 3 + (m > 0.75) * (rule == "ceil"), torch.full_like(e, -127)).clamp(-127, 125)
    scale = torch.ldexp(torch.ones_like(amax), e)
    a = (v.abs() / scale).clamp_max(6.0)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return torch.copysign(torch.round(a / step) * step, v), scale


def _through_mx4(x, rule):
    """The values that x in 4 bits stands for."""
    v, scale = _mx4(x, rule)
    return (v * scale).flatten(-2)[..., :x.shape[-1]]


def _weights(gen, rows, cols, transposed=False):
    """Codes, two to a byte, the even column's in the low half, and the scales' bytes, as a checkpoint holds them: of W [rows, cols], or of its
    transpose."""
    W = torch.randn((rows, cols), generator=gen, device=DEV).mul_(cols ** -0.5)
    v, scale = _mx4(W.t().contiguous() if transposed else W, "floor")
    code = (2 * v.abs()).long()
    code = torch.where(code > 4, torch.where(code == 6, 5, torch.where(code == 8, 6, 7)), code) + 8 * torch.signbit(v)
    code = code.flatten(-2)[:, :rows if transposed else cols].to(torch.uint8)
    return code[:, ::2] + code[:, 1::2] * 16, (torch.frexp(scale[..., 0])[1] + 126).to(torch.uint8)


def _values_of(weights):
    codes, scales = weights
    level = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    level = torch.cat([level, -level])
    v = torch.stack([level[(codes & 15).long()], level[(codes >> 4).long()]], -1).flatten(-2)
    K = v.shape[-1]
    return (_fill(v, BLOCK).unflatten(-1, (-1, BLOCK)) * torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)[..., None]).flatten(-2)[:, :K]


def _i8_weights(gen, rows, cols):
    W = torch.randn((rows, cols), generator=gen, device=DEV).mul_(cols ** -0.5)
    scale = W.abs().amax(-1, keepdim=True) / 127.0
    return torch.round(W / scale).clamp(-127, 127).to(torch.int8), scale[:, 0].contiguous()


def _norm_inputs(case, gen, s):
    T, d = case["T"], case["d"]
    s["w"] = (1.0 - case["offset"] + 0.1 * torch.randn(d, generator=gen, device=DEV)).to(DTYPE[case["w"]])
    s["x"] = _activations(gen, T, d, case["x"], case.get("gap", 0))
    if case["r"] != "none":
        s["r"] = (4.0 * _activations(gen, T, d, "f32")).to(DTYPE[case["r"]])


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s, op = {"case": case}, case["op"]
    if op == "quantize":
        s["x"] = _activations(gen, case["K"], case["rows"], case["x"]) if case["transposed"] else _activations(gen, case["rows"], case["K"], case["x"])
    elif op == "linear":
        s["x"] = _activations(gen, case["M"], case["K"], case["x"])
        s["W"] = _weights(gen, case["N"], case["K"])
    elif op == "linear_bwd":
        s["x"] = _activations(gen, case["M"], case["K"], case["x"])
        s["dy"] = _activations(gen, case["M"], case["N"], "f32").mul_(1e-4).to(DTYPE[case["dy"]])
        s["Wt"] = _weights(gen, case["N"], case["K"], transposed=True)
    elif op == "norm":
        _norm_inputs(case, gen, s)
        if case["out"] == "e4m3":
            s["scale"] = torch.full((1,), 40.0, device=DEV)          # a factor from the ranges of earlier steps
        if case["out"] in ("i8", "mx4"):
            s["W"] = (_weights if case["out"] == "mx4" else _i8_weights)(gen, case["N"], case["d"])
    else:
        _norm_inputs(case, gen, s)
        T, d = case["T"], case["d"]
        if case["r"] != "none":                              # what the forward pass kept: the sum; and the gradient that comes down the residual
            s["x"] = (s["x"].float() + s.pop("r").float()).to(DTYPE[case["r"]])
            s["ds"] = (1e-4 * torch.randn((T, d), generator=gen, device=DEV)).to(DTYPE[case["r"]])
        s["rstd"] = torch.rsqrt(s["x"].double().square().mean(-1) + EPS).float()
        s["dy"] = _activations(gen, T, d, "f32").mul_(1e-4).to(DTYPE[case["dy"]])
    return s


def _buffer(nbytes):
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)


def _laid_out(weights, i8=False):
    import paper_2409_12517_amd as ssg
    codes, scales = weights
    rows, K = codes.shape[0], codes.shape[1] * (1 if i8 else 2)
    q = _buffer((ssg.ssg_i8_bytes if i8 else ssg.ssg_mx4_bytes)(rows, K))
    (ssg.ssg_i8_pack if i8 else ssg.ssg_mx4_pack)(codes, scales, rows, K, q)
    return q


def _norm_desc(case):
    import paper_2409_12517_amd as ssg
    dt = {"bf16": ssg.SSG_BF16, "f32": ssg.SSG_F32}
    out = {"bf16": ssg.SSG_NORM_BF16, "f32": ssg.SSG_NORM_F32, "e4m3": ssg.SSG_NORM_E4M3, "i8": ssg.SSG_NORM_I8, "mx4": ssg.SSG_NORM_MX4}
    return ssg.make_rmsnorm_desc(case["T"], case["d"], EPS, x_dtype=dt[case["x"]], residual=int(case["r"] != "none"), r_dtype=dt.get(case["r"], ssg.SSG_BF16),
                                 w_dtype=dt[case["w"]], w_offset=case["offset"], y_format=out[case.get("out", "bf16")], ldx=case["d"] + case.get("gap", 0),
                                 rule=_rule(case))


def _rule(case):
    import paper_2409_12517_amd as ssg
    return ssg.SSG_MX_CEIL if case.get("rule") == "ceil" else ssg.SSG_MX_FLOOR


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:                                                  # a program keeps its weights as its path reads them, a plan and scratch
        import paper_2409_12517_amd as ssg
        op = case["op"]
        for n in ("W", "Wt"):
            if n in s:
                s[n] = _laid_out(s[n], case.get("out") == "i8")
        if op == "quantize":
            s["q"] = _buffer(ssg.ssg_mx4_bytes(case["rows"], case["K"]))
        elif op == "linear":
            s["work"] = _buffer(ssg.ssg_mx4_linear_workspace_bytes(case["M"], case["K"]))
        elif op == "linear_bwd":
            s["work"] = _buffer(ssg.ssg_mx4_linear_bwd_workspace_bytes(case["M"], case["N"], case["K"]))
        else:
            s["desc"] = _norm_desc(case)
            if op == "norm_bwd":
                s["work"] = _buffer(ssg.ssg_rmsnorm_bwd_workspace_bytes(s["desc"]))
            elif case["N"]:
                s["q"] = _buffer((ssg.ssg_i8_bytes if case["out"] == "i8" else ssg.ssg_mx4_bytes)(case["T"], case["d"]))
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


# the framework's operators
def _dt(name):
    import paper_2409_12517_amd as ssg
    return ssg.SSG_BF16 if name == "bf16" else ssg.SSG_F32


def _own_quantize(s):
    import paper_2409_12517_amd as ssg
    case = s["case"]
    rows, K = case["rows"], case["K"]
    ssg.ssg_mx4_quantize(s["x"], _dt(case["x"]), rows, K, rows if case["transposed"] else K, case["transposed"], _rule(case), s["q"])
    y = torch.empty((rows, K), dtype=torch.bfloat16, device=DEV)
    if K % 8 == 0:
        ssg.ssg_mx4_dequantize(s["q"], rows, K, y, ssg.SSG_BF16, K)
        return y
    wide = torch.empty((rows, K + -K % 8), dtype=torch.bfloat16, device=DEV)     # rows start on 16 bytes
    ssg.ssg_mx4_dequantize(s["q"], rows, K, wide, ssg.SSG_BF16, wide.shape[1])
    return wide[:, :K]


def _own_linear(s):
    import paper_2409_12517_amd as ssg
    case = s["case"]
    M, K, N = (case[n] for n in ("M", "K", "N"))
    y = torch.empty((M, N), dtype=DTYPE[case["y"]], device=DEV)
    ssg.ssg_mx4_linear(s["x"], _dt(case["x"]), M, K, K, _rule(case), s["W"], N, y, _dt(case["y"]), N, s["work"])
    return y


def _own_linear_bwd(s):
    import paper_2409_12517_amd as ssg
    case = s["case"]
    M, K, N = (case[n] for n in ("M", "K", "N"))
    dx = torch.empty((M, K), dtype=DTYPE[case["x"]], device=DEV)
    dW = torch.empty((N, K), dtype=DTYPE[case["dw"]], device=DEV)
    ssg.ssg_mx4_linear_bwd(s["dy"], _dt(case["dy"]), N, s["x"], _dt(case["x"]), K, M, N, K, _rule(case), s["Wt"], dx, _dt(case["x"]), K, dW, _dt(case["dw"]), K,
                           s["work"])
    return {"dx": dx, "dW": dW}


def _own_norm(s):
    import paper_2409_12517_amd as ssg
    case, out = s["case"], {}
    T, d, N = case["T"], case["d"], case["N"]
    if "r" in s:
        out["residual"] = torch.empty_like(s["r"])
    out["rstd"] = torch.empty(T, device=DEV)
    if N:
        y = s["q"]
    else:
        y = out["y"] = torch.empty((T, d), dtype=torch.float8_e4m3fn if case["out"] == "e4m3" else DTYPE[case["out"]], device=DEV)
    if case["out"] == "e4m3":
        out["amax"] = torch.empty(T, device=DEV)
    ssg.ssg_rmsnorm_fwd(s["desc"], s["x"], s.get("r"), s["w"], out.get("residual"), y, s.get("scale"), out.get("amax"), out["rstd"])
    if N:
        out["y"] = torch.empty((T, N), dtype=torch.bfloat16, device=DEV)
        (ssg.ssg_i8_gemm if case["out"] == "i8" else ssg.ssg_mx4_gemm)(y, T, s["W"], N, d, out["y"], ssg.SSG_BF16, N)
    return out


def _own_norm_bwd(s):
    import paper_2409_12517_amd as ssg
    case = s["case"]
    out = {"dx": torch.empty((case["T"], case["d"]), dtype=DTYPE[case["x"]], device=DEV), "dw": torch.empty(case["d"], device=DEV)}
    if case["r"] != "none":
        out["dr"] = torch.empty_like(s["ds"])
    ssg.ssg_rmsnorm_bwd(s["desc"], s["dy"], _dt(case["dy"]), case["d"], s["x"], s["rstd"], s["w"], s.get("ds"), out["dx"], out.get("dr"), out["dw"], s["work"])
    return out


_run_own = {"quantize": _own_quantize, "linear": _own_linear, "linear_bwd": _own_linear_bwd, "norm": _own_norm, "norm_bwd": _own_norm_bwd}


# the plain forms
def _plain_quantize(s):
    x = s["x"].t() if s["case"]["transposed"] else s["x"]
    return _through_mx4(x, s["case"]["rule"]).to(torch.bfloat16)


def _plain_linear(s):
    return (_through_mx4(s["x"], s["case"]["rule"]) @ _values_of(s["W"]).t()).to(DTYPE[s["case"]["y"]])


def _plain_linear_bwd(s):
    case = s["case"]
    dx = _through_mx4(s["dy"], case["rule"]) @ _values_of(s["Wt"]).t()
    dW = _through_mx4(s["dy"].t(), case["rule"]) @ _through_mx4(s["x"].t(), case["rule"]).t()
    return {"dx": dx.to(DTYPE[case["x"]]), "dW": dW.to(DTYPE[case["dw"]])}


def _plain_norm(s):
    case, out = s["case"], {}
    v = s["x"][:, :case["d"]].float()
    if "r" in s:
        out["residual"] = (v + s["r"].float()).to(s["r"].dtype)
        v = out["residual"].float()
    out["rstd"] = 1.0 / torch.sqrt(v.square().mean(-1) + EPS)
    y = v * out["rstd"][:, None] * (s["w"].float() + case["offset"])
    if case["out"] == "e4m3":
        out["amax"] = y.abs().amax(-1)
        out["y"] = (y * s["scale"]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    elif case["out"] == "mx4":
        out["y"] = (_through_mx4(y, case["rule"]) @ _values_of(s["W"]).t()).to(torch.bfloat16)
    elif case["out"] == "i8":
        amax = y.abs().amax(-1, keepdim=True)
        codes, scale = s["W"]
        out["y"] = (torch.round(y * (127.0 / amax)) @ codes.float().t() * (amax / 127.0) * scale).to(torch.bfloat16)
    else:
        out["y"] = y.to(DTYPE[case["out"]])
    return out


def _plain_norm_bwd(s):
    case, dy = s["case"], s["dy"].float()
    n = s["x"].float() * s["rstd"][:, None]
    a = dy * (s["w"].float() + case["offset"])
    g = s["rstd"][:, None] * (a - n * (a * n).mean(-1, keepdim=True))
    out = {"dw": (dy * n).sum(0)}
    if "ds" in s:
        g = g + s["ds"].float()
        out["dr"] = g.to(s["ds"].dtype)
    out["dx"] = g.to(DTYPE[case["x"]])
    return out


_run_plain = {"quantize": _plain_quantize, "linear": _plain_linear, "linear_bwd": _plain_linear_bwd, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd}


# ---------------------------------------------------------------- the work of one pass
def _bytes(name):
    return {"bf16": 2, "f32": 4, "e4m3": 1, "i8": 1, "mx4": 17 / 32, "none": 0}[name]


def work(case):
    op = case["op"]
    if op == "quantize":
        n = case["rows"] * case["K"]
        # the matrix read, its codes and scales written; they read again and the values written
        return {"bytes": n * (_bytes(case["x"]) + 2 * _bytes("mx4") + 2), "flops": 0}
    if op == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * K * _bytes(case["x"]) + N * K * _bytes("mx4") + M * N * _bytes(case["y"]), "flops": 2 * M * N * K}
    if op == "linear_bwd":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * N * _bytes(case["dy"]) + 2 * M * K * _bytes(case["x"]) + N * K * (_bytes("mx4") + _bytes(case["dw"])), "flops": 4 * M * N * K}
    n, d = case["T"] * case["d"], case["d"]
    if op == "norm":
        N = case["N"]
        rows = n * (_bytes(case["x"]) + 2 * _bytes(case["r"]) + (0 if N else _bytes(case["out"])))
        return {"bytes": rows + d * _bytes(case["w"]) + 4 * case["T"] + N * d * _bytes(case["out"]) + 2 * case["T"] * N, "flops": 2 * case["T"] * N * d + 4 * n}
    # dy and the normed rows; the residual's gradient in and out; dx; weights and their gradient
    kept = _bytes(case["x"]) if case["r"] == "none" else _bytes(case["r"])
    return {"bytes": n * (_bytes(case["dy"]) + kept + 2 * _bytes(case["r"]) + _bytes(case["x"])) + d * (_bytes(case["w"]) + 4) + 4 * case["T"], "flops": 10 * n}


# ---------------------------------------------------------------- from the definition, in 64 bits
def _exact_mx4(x, rule):
    """The nearest of the fifteen values by comparison with the midpoints between them; between two, the one whose code is even."""
    level = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=DEV)
    mid = (level[1:] + level[:-1]) / 2
    x = x.double()
    out = torch.zeros_like(x)
    for k in range(0, x.shape[1], BLOCK):
        v = x[:, k:k + BLOCK]
        amax = v.abs().amax(1, keepdim=True)
        e = torch.floor(torch.log2(amax.clamp_min(2.0 ** -1000)))
        e = e - (torch.exp2(e) > amax).double() + (torch.exp2(e + 1) <= amax).double()
        e = (e - 2 + (amax > 1.5 * torch.exp2(e)) if rule == "ceil" else e - 2).clamp(-127, 125)
        a = v.abs() / torch.exp2(e)
        at = torch.zeros_like(a, dtype=torch.long)
        for i in range(7):
            at += (a > mid[i]) if i % 2 == 0 else (a >= mid[i])
        out[:, k:k + BLOCK] = level[at] * torch.sign(v) * torch.exp2(e)
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "quantize":
        return _exact_mx4(s["x"].t() if case["transposed"] else s["x"], case["rule"])
    if op == "linear":
        return _exact_mx4(s["x"], case["rule"]) @ _values_of(s["W"]).double().t()
    if op == "linear_bwd":
        dy = s["dy"]
        dW = _exact_mx4(dy.t(), case["rule"]) @ _exact_mx4(s["x"].t(), case["rule"]).t()
        return {"dx": _exact_mx4(dy, case["rule"]) @ _values_of(s["Wt"]).double().t(), "dW": dW}
    w = s["w"].double() + case["offset"]
    if op == "norm_bwd":
        v = s["x"].double()
        rstd = s["rstd"].double()[:, None]
        dy = s["dy"].double()
        inner = (dy * w * v).sum(-1, keepdim=True)
        g = dy * w * rstd - v * rstd.pow(3) * inner / case["d"]
        out = {"dw": (dy * v * rstd).sum(0)}
        if "ds" in s:
            g = out["dr"] = g + s["ds"].double()
        out["dx"] = g
        return out
    v, out = s["x"][:, :case["d"]].double(), {}
    if "r" in s:
        total = v + s["r"].double()
        out["residual"] = total
        v = total.float().to(s["r"].dtype).double()          # what is normed is what is kept
    rstd = (v.pow(2).sum(-1) / case["d"] + EPS).pow(-0.5)
    out["rstd"] = rstd
    y = v * rstd[:, None] * w
    if case["out"] == "e4m3":
        out["amax"] = y.abs().max(-1).values
        z = (y * s["scale"].double()).clamp(-448.0, 448.0)
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp_min(2.0 ** -6))) - 3)
        y = torch.round(z / step) * step
    elif case["out"] == "mx4":
        y = _exact_mx4(y, case["rule"]) @ _values_of(s["W"]).double().t()
    elif case["out"] == "i8":
        unit = y.abs().max(-1, keepdim=True).values / 127.0
        codes, scale = s["W"]
        y = (torch.round(y / unit) @ codes.double().t()) * unit * scale.double()
    out["y"] = y
    return out
