"""Cases for the operators of a mixture of experts served in 8-bit integers: routing with its gradient, the int8 matrix
product with a scale for each token and channel, and the layer that runs them together.  Their inputs, the work they cannot do
without, the same results in elementary torch operations in 32 bits, and from the definition in 64.

Kinds of cases (`op`):
  route      ssg_route: chosen experts, their weights, and the order in which grouped products take the rows
  route_bwd  ssg_route_bwd: the gradient of the weights with respect to the logits
  linear     ssg_i8_linear: rows of x quantized with a scale each, times int8 weights with a scale for each channel
  moe        ssg_moe_fwd: routing, the experts' SwiGLU MLPs on int8 products, the weighted sum
All inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DEV = "cuda"
ALIGN = 16                                   # an expert's rows start at a multiple of this
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- the cases
def _route(T, E, k, dtype="f32", score="softmax", bias=0, groups=1, top_groups=1, group_top=1, renorm=1, scale=1.0, pad=0, gap=0):
    """pad: every pad-th token of the batch is padding, all experts closed to it; gap: elements between two tokens' logits."""
    return {"op": "route", "T": T, "E": E, "k": k, "dtype": dtype, "score": score, "bias": bias, "groups": groups,
            "top_groups": top_groups, "group_top": group_top, "renorm": renorm, "scale": scale, "pad": pad, "gap": gap}


def _linear(M, K, N, x="bf16", y="bf16"):
    return {"op": "linear", "M": M, "K": K, "N": N, "x": x, "y": y}


def _moe(d, f, **route):
    return {**_route(**route), "op": "moe", "d": d, "f": f}


BALANCED = dict(score="sigmoid", bias=1, groups=8, top_groups=4, group_top=2, scale=2.5)


def listed():
    return [
        # a decode step of one sequence: nothing but latency
        {"name": "route_token", **_route(1, 64, 8)},
        # a ragged batch with padding tokens in it, plain probabilities as weights, logits inside a wider buffer
        {"name": "route_batch", **_route(331, 160, 6, "bf16", groups=8, top_groups=3, renorm=0, scale=16.0, pad=16, gap=32)},
        # the tokens of a training micro-batch or of a long prefill: sigmoid scores with a balance bias, groups, renormalised
        {"name": "route_prefill", **_route(16384, 256, 8, **BALANCED)},
        # the gradient in a micro-batch with softmax weights as they are: every expert's logit has one
        {"name": "route_bwd_dense", **_route(4099, 64, 2, "bf16", renorm=0), "op": "route_bwd"},
        # the gradient of the long micro-batch: the chosen experts' only
        {"name": "route_bwd_prefill", **_route(16384, 256, 8, **BALANCED), "op": "route_bwd"},
        # decoding at the 7B widths, up projection: one token, the weights' bytes
        {"name": "linear_token", **_linear(1, 4096, 11008)},
        # a mixed batch of odd size and odd widths, results for a sum in fp32
        {"name": "linear_odd", **_linear(333, 2736, 1040, "f32", "f32")},
        # a prefill at the 7B widths, down projection
        {"name": "linear_prefill", **_linear(4096, 11008, 4096)},
        # one token through small experts
        {"name": "moe_token", **_moe(2048, 1376, T=1, E=64, k=8)},
        # a decode batch: a few rows for each expert
        {"name": "moe_batch", **_moe(2048, 1376, T=75, E=64, k=8, dtype="bf16", pad=16, **BALANCED)},
        # few large experts at the 7B widths, an odd number of tokens
        {"name": "moe_large_experts", **_moe(4096, 11008, T=1041, E=8, k=2, dtype="bf16")},
        # a prefill through small experts
        {"name": "moe_prefill", **_moe(2048, 1376, T=4096, E=64, k=8, **BALANCED)},
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def _draw_route(rng, T, E, k):
    groups = rng.choice([g for g in (1, 1, 2, 4, 8) if E % g == 0])
    top_groups = rng.randint(max(1, -(-k * groups // E)), groups)
    return _route(T, E, k, rng.choice(["bf16", "f32"]), rng.choice(["softmax", "sigmoid"]), rng.randrange(2), groups, top_groups,
                  rng.choice([1, 2]), rng.randrange(2), rng.choice([1.0, 2.5]), rng.choice([0, 0, 7]), rng.choice([0, 0, 16]))


def draw(rng):
    op = rng.choice(["route", "route", "route_bwd", "linear", "linear", "linear", "moe", "moe", "moe"])
    if op in ("route", "route_bwd"):
        E = _log(rng, 8, 256, rng.choice([1, 8]))
        r = {**_draw_route(rng, _log(rng, 1, 16384), E, rng.randint(1, min(8, E // 2))), "op": op}
        if op == "route_bwd" and r["k"] == 1:
            r["renorm"] = 0                                  # a single renormalised weight is constant: no gradient
        return r
    if op == "linear":
        return _linear(_log(rng, 1, 4096), _log(rng, 256, 11008, rng.choice([16, 128])), _log(rng, 256, 4096, rng.choice([16, 128])),
                       rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bf16", "bf16", "f32"]))
    E = rng.choice([8, 16, 32, 64, 96])
    k = rng.randint(1, min(8, E // 4))
    d = _log(rng, 512, 4096, rng.choice([16, 128]))
    f = _log(rng, 256, min(11008, 8 * 4096 * 11008 // (E * d)), rng.choice([16, 128]))
    T = _log(rng, 1, min(4096, max(1, int(4096 * 8 * 2048 * 1376 / (k * d * f)))))
    return {**_draw_route(rng, T, E, k), "op": "moe", "d": d, "f": f}


# ---------------------------------------------------------------- inputs, from the seed alone
def _quantize(x):
    """Whole numbers from -127 to 127 and a scale for each row, in 32 bits."""
    amax = x.abs().amax(-1, keepdim=True)
    scale = torch.where(amax > 0, (amax / 127.0).clamp_min(2.0 ** -126), amax)
    inv = torch.where(amax / 127.0 >= 2.0 ** -126, 127.0 / amax, torch.full_like(amax, 2.0 ** 126))
    return torch.round(x * inv).clamp(-127, 127), scale


def _gaps64(case, z, bias):
    """How far apart the keys are that decide a token's choice, in 64 bits: of neighbours among the best experts, and of the last group
    that stays and the first that does not."""
    z = z.double()
    closed = torch.isneginf(z)
    if case["score"] == "softmax":
        s = torch.softmax(z.masked_fill(closed, -1e300), -1)
    else:
        s = torch.sigmoid(z)
    key = (s if bias is None else s + bias.double()).masked_fill(closed, -math.inf)
    groups, top = case["groups"], case["top_groups"]
    found = []
    if top < groups:
        by = key.unflatten(-1, (groups, -1)).sort(-1, descending=True).values
        g = by[..., 0] + (by[..., 1].clamp_min(-1e9) if case["group_top"] == 2 and by.shape[-1] > 1 else 0.0)
        g, order = g.sort(-1, descending=True)
        found.append(g[:, top - 1:top] - g[:, top:top + 1])
        key = key.masked_fill(torch.ones_like(g, dtype=torch.bool).scatter_(1, order[:, :top], False).repeat_interleave(case["E"] // groups, 1), -math.inf)
    best = key.sort(-1, descending=True).values[:, :case["k"] + 1]
    found.append((best[:, :-1] - best[:, 1:]) / (1.0 if bias is not None else best[:, :-1].clamp_min(1e-30)))
    return torch.cat(found, 1)


def _router(case, gen):
    """Logits as a trained router gives them, a balance bias of many small steps.  Tokens whose choice hangs on the last bits of
    a score are drawn again: the order of two experts that differ by less than the rounding of 32 bits has no right answer."""
    T, E = case["T"], case["E"]
    dt = DTYPE[case["dtype"]]
    offset = torch.randn((1, E), generator=gen, device=DEV) * 0.5
    bias = torch.randint(-100, 101, (E,), generator=gen, device=DEV).float() * 1e-3 if case["bias"] else None

    def fresh():
        return (torch.randn((T, E), generator=gen, device=DEV) * 1.5 + offset).to(dt)

    def bad(z):
        gap = _gaps64(case, z, bias)
        return ((gap > 0) & (gap < 4e-6)).any(-1)

    z = fresh()
    if case["pad"]:
        z[::case["pad"]] = -math.inf
    for _ in range(12):
        again = bad(z)
        z = torch.where(again[:, None], fresh(), z)
    z = torch.where(bad(z)[:, None], torch.arange(E, device=DEV).mul(-0.0625).to(dt)[None], z)
    wide = torch.zeros((T, E + case["gap"]), device=DEV, dtype=dt)
    wide[:, :E] = z
    return wide, bias


def _activations(gen, rows, cols, dtype):
    """Rows of different magnitude, a few of the channels far larger than the others."""
    x = torch.randn((rows, cols), generator=gen, device=DEV)
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device=DEV))
    x[:, torch.randperm(cols, generator=gen, device=DEV)[:4]] *= 8.0
    return x.to(DTYPE[dtype])


def _weights(gen, rows, cols):
    """Codes [rows, cols] int8 and a scale for each row, as a checkpoint holds them."""
    codes, scale = _quantize(torch.randn((rows, cols), generator=gen, device=DEV).mul_(cols ** -0.5))
    return codes.to(torch.int8), scale[:, 0].contiguous()


def _laid_out(weights):
    import paper_2409_12517_amd as ssg
    codes, scale = weights
    q = torch.empty(ssg.ssg_i8_bytes(*codes.shape), dtype=torch.uint8, device=DEV)
    ssg.ssg_i8_pack(codes, scale, codes.shape[0], codes.shape[1], q)
    return q


def _route_desc(case):
    import paper_2409_12517_amd as ssg
    return ssg.make_route_desc(
        case["T"], case["E"], case["k"], ld=case["E"] + case["gap"],
        logits_dtype=ssg.SSG_BF16 if case["dtype"] == "bf16" else ssg.SSG_F32,
        score=ssg.SSG_ROUTE_SIGMOID if case["score"] == "sigmoid" else ssg.SSG_ROUTE_SOFTMAX,
        groups=case["groups"], top_groups=case["top_groups"], group_top=case["group_top"], renorm=case["renorm"],
        scale=case["scale"], row_align=ALIGN)


def _workspace(nbytes):
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=DEV)


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = {"case": case}
    if case["op"] == "linear":
        s["x"] = _activations(gen, case["M"], case["K"], case["x"])
        s["W"] = _weights(gen, case["N"], case["K"])
        return s
    s["logits"], s["bias"] = _router(case, gen)
    if case["op"] == "route_bwd":
        s.update(_plain_scores(case, s["logits"], s["bias"]))
        s["dweights"] = torch.randn(s["weights"].shape, generator=gen, device=DEV) * 1e-2
    if case["op"] == "moe":
        E, d, f = case["E"], case["d"], case["f"]
        s["x"] = _activations(gen, case["T"], d, "bf16")
        s["W1"], s["W2"], s["W3"] = _weights(gen, E * f, d), _weights(gen, E * f, d), _weights(gen, E * d, f)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:                                                  # a program keeps its weights as its path reads them, a plan and scratch
        import paper_2409_12517_amd as ssg
        for n in ("W", "W1", "W2", "W3"):
            if n in s:
                s[n] = _laid_out(s[n])
        if case["op"] == "linear":
            s["work"] = _workspace(ssg.ssg_i8_linear_workspace_bytes(case["M"], case["K"]))
        else:
            s["desc"] = _route_desc(case)
        if case["op"] == "route":
            s["work"] = _workspace(ssg.ssg_route_workspace_bytes(s["desc"]))
        if case["op"] == "moe":
            s["desc"] = ssg.make_moe_desc(s["desc"], case["d"], case["f"])
            s["work"] = _workspace(ssg.ssg_moe_workspace_bytes(s["desc"]))
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


# the framework's operators
def _own_route(s):
    import paper_2409_12517_amd as ssg
    T, E, k = (s["case"][n] for n in ("T", "E", "k"))
    rows = ssg.ssg_route_rows(s["desc"])
    out = {n: torch.empty(shape, dtype=torch.float32 if n == "weights" else torch.int32, device=DEV)
           for n, shape in (("ids", (T, k)), ("weights", (T, k)), ("counts", (E,)), ("offsets", (E + 1,)), ("place", (T * k,)), ("source", (rows,)))}
    ssg.ssg_route(s["desc"], s["logits"], s["bias"], out["ids"], out["weights"], out["counts"], out["offsets"], out["place"],
                  out["source"], s["work"])
    return out


def _own_route_bwd(s):
    import paper_2409_12517_amd as ssg
    dlogits = torch.empty((s["case"]["T"], s["case"]["E"]), dtype=s["logits"].dtype, device=DEV)
    ssg.ssg_route_bwd(s["desc"], s["logits"], s["ids"], s["weights"], s["dweights"], dlogits)
    return dlogits


def _own_linear(s):
    import paper_2409_12517_amd as ssg
    M, K, N = (s["case"][n] for n in ("M", "K", "N"))
    dt = {"bf16": ssg.SSG_BF16, "f32": ssg.SSG_F32}
    y = torch.empty((M, N), dtype=DTYPE[s["case"]["y"]], device=DEV)
    ssg.ssg_i8_linear(s["x"], dt[s["case"]["x"]], M, K, K, s["W"], N, y, dt[s["case"]["y"]], N, s["work"])
    return y


def _own_moe(s):
    import paper_2409_12517_amd as ssg
    y = torch.empty((s["case"]["T"], s["case"]["d"]), dtype=torch.bfloat16, device=DEV)
    ssg.ssg_moe_fwd(s["desc"], s["x"], s["logits"], s["bias"], s["W1"], s["W2"], s["W3"], y, s["work"])
    return y


_run_own = {"route": _own_route, "route_bwd": _own_route_bwd, "linear": _own_linear, "moe": _own_moe}


# the plain forms
def _scores(case, logits):
    z = logits[:, :case["E"]].float()
    open_ = z > -math.inf
    z = z.clamp_max(torch.finfo(torch.float32).max)
    if case["score"] == "softmax":
        m = torch.where(open_, z, torch.full_like(z, -math.inf)).amax(-1, keepdim=True)
        e = torch.where(open_, torch.exp(z - torch.where(torch.isneginf(m), torch.zeros_like(m), m)), torch.zeros_like(z))
        s = e / e.sum(-1, keepdim=True).clamp_min(1e-38)
    else:
        s = torch.where(open_, 1.0 / (1.0 + torch.exp(-z)), torch.zeros_like(z))
    return z, open_, s


def _plain_scores(case, logits, bias):
    T, E, k, groups = case["T"], case["E"], case["k"], case["groups"]
    z, open_, s = _scores(case, logits)
    closed = torch.full_like(s, -math.inf)
    key = torch.where(open_, z if bias is None else s + bias, closed)
    if case["top_groups"] < groups:
        by = key if case["group_top"] == 1 else torch.where(open_, s if bias is None else s + bias, closed)
        by = torch.sort(by.reshape(T, groups, -1), dim=-1, descending=True).values
        g = by[..., 0]
        if case["group_top"] == 2 and by.shape[-1] > 1:
            g = g + torch.where(torch.isneginf(by[..., 1]), torch.zeros_like(g), by[..., 1])
        kept = torch.sort(g, dim=-1, descending=True, stable=True).indices[:, :case["top_groups"]]
        mask = torch.zeros((T, groups), dtype=torch.bool, device=DEV).scatter_(1, kept, True)
        key = torch.where(mask.repeat_interleave(E // groups, dim=1), key, closed)
    key, ids = torch.sort(key, dim=-1, descending=True, stable=True)
    ids, chosen = ids[:, :k], key[:, :k] > -math.inf
    w = torch.where(chosen, s.gather(1, ids), torch.zeros((), device=DEV))
    if case["renorm"]:
        w = w / w.sum(-1, keepdim=True).clamp_min(1e-38)
    return {"ids": torch.where(chosen, ids, torch.full_like(ids, -1)).int(), "weights": w * case["scale"]}


def _rows(case):
    n = case["T"] * case["k"]
    return (n + min(case["E"], n) * (ALIGN - 1)) // ALIGN * ALIGN


def _plain_route(s):
    case = s["case"]
    T, E, k = case["T"], case["E"], case["k"]
    r = _plain_scores(case, s["logits"], s["bias"])
    flat = r["ids"].reshape(-1).long()
    e = torch.where(flat < 0, torch.full_like(flat, E), flat)
    e_sorted, order = torch.sort(e, stable=True)
    counts = torch.zeros(E + 1, dtype=torch.long, device=DEV).scatter_add_(0, e, torch.ones_like(e))
    padded = (counts + ALIGN - 1) // ALIGN * ALIGN
    offsets = torch.cumsum(padded, 0) - padded
    row = offsets[e_sorted] + torch.arange(T * k, device=DEV) - (torch.cumsum(counts, 0) - counts)[e_sorted]
    row = torch.where(e_sorted < E, row, torch.full_like(row, -1))
    place = torch.empty(T * k, dtype=torch.long, device=DEV).scatter_(0, order, row)
    rows = _rows(case)
    source = torch.full((rows + 1,), -1, dtype=torch.long, device=DEV).scatter_(0, torch.where(row < 0, torch.full_like(row, rows), row), order)
    return {**r, "counts": counts[:E].int(), "offsets": offsets.int(), "place": place.int(), "source": source[:rows].int()}


def _plain_route_bwd(s):
    case, ids, w, dw = s["case"], s["ids"].long(), s["weights"], s["dweights"]
    _, _, p = _scores(case, s["logits"])
    chosen = ids >= 0
    at = ids.clamp_min(0)
    dw = torch.where(chosen, dw, torch.zeros_like(dw))
    sel = torch.where(chosen, p.gather(1, at), torch.zeros_like(dw))
    if case["renorm"]:
        mean = (w * dw).sum(-1, keepdim=True)
        d = (case["scale"] * dw - mean) / sel.sum(-1, keepdim=True).clamp_min(1e-38)
    else:
        d = case["scale"] * dw
    if case["score"] == "sigmoid":
        d = d * sel * (1.0 - sel)
        return torch.zeros_like(p).scatter_add_(1, at, torch.where(chosen, d, torch.zeros_like(d))).to(s["logits"].dtype)
    mean = (d * sel).sum(-1, keepdim=True) if not case["renorm"] else torch.zeros_like(d[:, :1])
    dz = torch.zeros_like(p).scatter_add_(1, at, torch.where(chosen, d * sel, torch.zeros_like(d)))
    return (dz - p * mean).to(s["logits"].dtype)


def _plain_linear(s):
    x, sx = _quantize(s["x"].float())
    codes, scale = s["W"]
    return (x @ codes.float().t() * sx * scale).to(DTYPE[s["case"]["y"]])


def _plain_moe(s):
    case = s["case"]
    E, d, f, k = (case[n] for n in ("E", "d", "f", "k"))
    r = _plain_scores(case, s["logits"], s["bias"])
    flat = r["ids"].reshape(-1).long()
    e = torch.where(flat < 0, torch.full_like(flat, E), flat)
    counts = torch.zeros(E + 1, dtype=torch.long, device=DEV).scatter_add_(0, e, torch.ones_like(e))
    e_sorted, order = torch.sort(e, stable=True)
    first = torch.cumsum(counts, 0) - counts
    cap = max(1, int(counts[:E].max()))                      # every expert's rows, padded to the fullest expert's
    row = torch.where(e_sorted < E, e_sorted * cap + torch.arange(e.numel(), device=DEV) - first[e_sorted], torch.full_like(e_sorted, E * cap))
    place = torch.empty_like(row).scatter_(0, order, row)
    token = torch.arange(e.numel(), device=DEV) // k
    xq, sx = _quantize(s["x"].float())
    a = torch.zeros((E * cap + 1, d), device=DEV)
    sa = torch.zeros((E * cap + 1, 1), device=DEV)
    a[place], sa[place] = xq[token], sx[token]
    a, sa = a[:E * cap].view(E, cap, d), sa[:E * cap].view(E, cap, 1)

    def product(q, sq, weights, n, inner):
        codes, scale = weights
        return torch.bmm(q, codes.float().view(E, n, inner).transpose(1, 2)) * sq * scale.view(E, 1, n)

    u, g = product(a, sa, s["W1"], f, d), product(a, sa, s["W2"], f, d)
    h = (u * (g * (1.0 / (1.0 + torch.exp(-g))))).to(torch.bfloat16)       # the activation between the layers is bf16
    hq, sh = _quantize(h.float())
    o = product(hq, sh, s["W3"], d, f).view(E * cap, d)
    o = torch.cat([o, torch.zeros((1, d), device=DEV)])[place].view(-1, k, d)
    return (o * r["weights"][:, :, None]).sum(1).to(torch.bfloat16)


_run_plain = {"route": _plain_route, "route_bwd": _plain_route_bwd, "linear": _plain_linear, "moe": _plain_moe}


# ---------------------------------------------------------------- the work of one pass
def _bytes(name):
    return 2 if name == "bf16" else 4


def work(case):
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * K * _bytes(case["x"]) + N * K + 4 * N + M * N * _bytes(case["y"]), "flops": 2 * M * N * K}
    T, E, k = case["T"], case["E"], case["k"]
    logits = T * E * _bytes(case["dtype"])
    if case["op"] == "route":
        # logits and bias; ids and weights; counts and offsets; the place of every assignment and the source of every row
        return {"bytes": logits + 4 * E * case["bias"] + 8 * T * k + 8 * E + 4 * T * k + 4 * _rows(case), "flops": T * E * 4}
    if case["op"] == "route_bwd":
        # where the weights are renormalised, or scores are sigmoids, only the chosen experts' logits matter
        dense = case["score"] == "softmax" and not case["renorm"]
        return {"bytes": (logits if dense else T * k * _bytes(case["dtype"])) + 12 * T * k + logits, "flops": T * E * 4}
    d, f = case["d"], case["f"]
    active = E * (1.0 - (1.0 - k / E) ** T)                 # experts that a token chooses, on average over even choices
    return {"bytes": logits + 2 * T * d * 2 + active * (3 * d * f + 4 * (2 * f + d)), "flops": 6 * T * k * d * f}


# ---------------------------------------------------------------- from the definition, in 64 bits
def _exact_choice(case, logits, bias):
    """ids, weights, and the scores, by ranking every expert against every other."""
    E, k, G = case["E"], case["k"], case["groups"]
    z = logits[:, :E].double()
    shut = ~(z > -math.inf)
    if case["score"] == "softmax":
        s = torch.nan_to_num(torch.softmax(z.masked_fill(shut, -math.inf), -1), nan=0.0)
    else:
        s = torch.special.expit(z).masked_fill(shut, 0.0)
    key = (z if bias is None else s + bias.double()).masked_fill(shut, -math.inf)
    if case["top_groups"] < G:
        v = (key if case["group_top"] == 1 else (s if bias is None else s + bias.double()).masked_fill(shut, -math.inf)).unflatten(1, (G, E // G))
        best = v.topk(min(case["group_top"], E // G), dim=-1).values
        gk = best[..., 0] + best[..., 1:].masked_fill(torch.isneginf(best[..., 1:]), 0.0).sum(-1)
        idx = torch.arange(G, device=gk.device)
        ahead = (gk[:, None, :] > gk[:, :, None]) | ((gk[:, None, :] == gk[:, :, None]) & (idx[None, :] < idx[:, None]))
        keep = ahead.sum(-1) < case["top_groups"]
        key = key.masked_fill(~keep.repeat_interleave(E // G, 1), -math.inf)
    ids = torch.full((case["T"], k), -1, dtype=torch.long, device=key.device)
    left = key.clone()
    for j in range(k):
        top = left.amax(-1, keepdim=True)
        first = (left == top).double().argmax(-1, keepdim=True)
        ok = top[:, 0] > -math.inf
        ids[:, j] = torch.where(ok, first[:, 0], ids[:, j])
        left.scatter_(1, first, -math.inf)
    w = s.gather(1, ids.clamp_min(0)).masked_fill(ids < 0, 0.0)
    if case["renorm"]:
        w = torch.nan_to_num(w / w.sum(-1, keepdim=True), nan=0.0)
    return ids, w * case["scale"], s


def _exact_quantize(x):
    """Codes and scales of rows; x holds binary32 values."""
    x = x.double()
    top = x.abs().amax(1)
    safe = top.masked_fill(top == 0, 1.0)
    return torch.round(x * (127.0 / safe)[:, None]), top / 127.0


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "linear":
        (q, sx), (codes, scale) = _exact_quantize(s["x"]), s["W"]
        return (q @ codes.double().t()) * sx[:, None] * scale.double()
    if case["op"] == "route_bwd":
        ids, dw, z = s["ids"].long(), s["dweights"].double(), s["logits"][:, :case["E"]].double().requires_grad_(True)
        shut = torch.isneginf(z.detach())
        p = torch.softmax(z.masked_fill(shut, -1e300), -1) if case["score"] == "softmax" else torch.sigmoid(z.masked_fill(shut, -700.0))
        w = p.gather(1, ids.clamp_min(0)) * (ids >= 0)
        if case["renorm"]:
            w = w / w.sum(-1, keepdim=True).clamp_min(1e-300)
        (w * dw * case["scale"]).sum().backward()
        return z.grad.masked_fill(shut, 0.0)
    ids, w, _ = _exact_choice(case, s["logits"], s["bias"])
    T, E, k = case["T"], case["E"], case["k"]
    if case["op"] == "route":
        host = ids.reshape(-1).cpu().tolist()
        lists = [[] for _ in range(E)]
        for a, e in enumerate(host):
            if e >= 0:
                lists[e].append(a)
        offsets, place, source = [0], [-1] * (T * k), [-1] * _rows(case)
        for held in lists:
            for i, a in enumerate(held):
                place[a] = offsets[-1] + i
                source[offsets[-1] + i] = a
            offsets.append(offsets[-1] + -(-len(held) // ALIGN) * ALIGN)

        def whole(v):
            return torch.tensor(v, dtype=torch.int32)

        return {"ids": ids.int(), "weights": w, "counts": whole([len(v) for v in lists]), "offsets": whole(offsets), "place": whole(place),
                "source": whole(source)}
    d, f = case["d"], case["f"]
    y = torch.zeros((T, d), dtype=torch.float64, device=DEV)
    for e in range(E):
        tok, slot = torch.nonzero(ids == e, as_tuple=True)
        if not tok.numel():
            continue

        def part(weights, n):
            return weights[0][e * n:(e + 1) * n].double(), weights[1][e * n:(e + 1) * n].double()

        q, sq = _exact_quantize(s["x"][tok])
        (c1, t1), (c2, t2), (c3, t3) = part(s["W1"], f), part(s["W2"], f), part(s["W3"], d)
        u, g = q @ c1.t() * sq[:, None] * t1, q @ c2.t() * sq[:, None] * t2
        hq, sh = _exact_quantize((u * g * torch.sigmoid(g)).to(torch.bfloat16))
        y.index_add_(0, tok, (hq @ c3.t() * sh[:, None] * t3) * w[tok, slot][:, None])
    return y
