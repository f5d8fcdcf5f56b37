"""What the router's operators and those of the 8-bit integer layers are timed on, beside the plain form of each in elementary torch operations.

A case is a plain dict.  `op` says what a pass does:

  route     moe_route: a router's logits to each token's experts and weights, and the rows sorted by expert
  combine   moe_combine: the experts' output rows, weighted and added up for each token, with a shared expert's output
  quantize  int8_quantize: 8-bit integers with a scale for each row (weights on loading, activations)
  project   int8_rmsnorm_quantize and int8_gemm: the residual's addition, the norm, and the projection that reads it
  down      int8_quantize of silu(gate) * up and int8_gemm: the down projection of a feed-forward layer
  gemm      int8_gemm: activations times weights, both 8-bit integers, a scale for each token and each channel
  grouped   int8_grouped_gemm: the same with the rows sorted by expert, each expert with weights of its own

Codes are integers between -127 and 127 in what this file makes.  What rounds to codes behind an exponential or a root is timed together with the product
that reads it: a value next to the middle of two codes may go to either.  `own` chooses the framework's calls; otherwise run() computes the plain form.
"""
import math

import torch

own = False

TOP = 127.0                # the largest code
AMAX_LEAST = 2.0 ** -100   # a row's abs-max counts as at least this
EPS = 1e-6


def listed():
    return [
        # One decoded token's choice of experts: latency.
        {"name": "route_t1", "op": "route", "tokens": 1, "experts": 64, "top": 4, "score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "f32": False},
        # A mixed batch on many experts in groups, scores of their own and a bias that balances the experts' load.
        {"name": "route_t777_groups", "op": "route", "tokens": 777, "experts": 256, "top": 8, "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4, "f32": True},
        # The prompts of a full batch, logits as a bf16 router leaves them (many are equal).
        {"name": "route_t16384", "op": "route", "tokens": 16384, "experts": 128, "top": 8, "score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "f32": False},
        # The end of a mixture layer: a few decoded tokens, and a prompt.
        {"name": "combine_t5", "op": "combine", "tokens": 5, "top": 4, "cols": 4096, "shared": True, "f32": False},
        {"name": "combine_t4095", "op": "combine", "tokens": 4095, "top": 8, "cols": 4096, "shared": True, "f32": False},
        # Weights on loading: the gate and up projection of the 70B-shaped layer.
        {"name": "quantize_n57344", "op": "quantize", "rows": 57344, "cols": 8192},
        # A decoding batch with an odd number of tokens: the down projection behind the gated activation.
        {"name": "down_m33", "op": "down", "tokens": 33, "n": 4096, "k": 14336},
        # One token through the norm and the fused projection behind it: latency, and weights streamed from HBM.
        {"name": "project_m1", "op": "project", "tokens": 1, "n": 6144, "k": 4096, "residual": True},
        # The same for a prompt of 4095 tokens on the 70B-shaped q/k/v projection, the largest ordinary product.
        {"name": "project_m4095", "op": "project", "tokens": 4095, "n": 10240, "k": 8192, "residual": True},
        # A mixed batch, an odd number of columns, columns of activations that are no whole blocks of 128.
        {"name": "gemm_m201", "op": "gemm", "tokens": 201, "n": 5001, "k": 2896, "f32": True},
        # Sixteen decoded tokens, four experts each out of 64: the weights of the experts in use.
        {"name": "grouped_decode", "op": "grouped", "tokens": 16, "top": 4, "experts": 64, "n": 4096, "k": 4096, "gather": True},
        # A prompt of 4096 tokens, four experts each out of 64, the tokens' rows gathered by index.
        {"name": "grouped_prefill", "op": "grouped", "tokens": 4096, "top": 4, "experts": 64, "n": 4096, "k": 4096, "gather": True},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _columns(rng, most):
    """K: sixteens, half of the time whole blocks of 128."""
    return 128 * _log_int(rng, 2, most // 128) if rng.random() < 0.5 else 16 * _log_int(rng, 12, most // 16)


def draw(rng):
    op = rng.choice(["route", "route", "combine", "quantize", "down", "project", "gemm", "gemm", "grouped", "grouped"])
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log_int(rng, 4, 512 // groups)
        top_groups = rng.randint(1, groups)
        return {"op": op, "tokens": _log_int(rng, 1, 16384), "experts": experts, "top": rng.randint(1, min(8, experts // groups * top_groups)),
                "score": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5, "groups": groups, "top_groups": top_groups, "f32": rng.random() < 0.5}
    if op == "combine":
        return {"op": op, "tokens": _log_int(rng, 1, 4096), "top": rng.randint(1, 8), "cols": _log_int(rng, 100, 8192) if rng.random() < 0.3 else 64 * _log_int(rng, 4, 128),
                "shared": rng.random() < 0.6, "f32": rng.random() < 0.3}
    if op == "quantize":
        cols = _columns(rng, 14336)
        return {"op": op, "rows": min(_log_int(rng, 1, 57344), 57344 * 8192 // cols), "cols": cols}
    if op == "grouped":
        experts = _log_int(rng, 2, 64)
        n = _log_int(rng, 200, 4096)
        return {"op": op, "tokens": _log_int(rng, 1, 4096), "top": rng.randint(1, min(4, experts)), "experts": experts, "n": n // 8 * 8 if rng.random() < 0.7 else n,
                "k": _columns(rng, 4096), "gather": rng.random() < 0.6}
    n, k = _log_int(rng, 200, 28672), _columns(rng, 14336)
    n = n // 8 * 8 if rng.random() < 0.7 else n
    tokens = max(1, min(_log_int(rng, 1, 4096), 4095 * 10240 * 8192 // (n * k)))
    case = {"op": op, "tokens": tokens, "n": n, "k": k}
    if op == "project":
        case["residual"] = rng.random() < 0.7
    if op == "gemm":
        case["f32"] = rng.random() < 0.3
    return case


def _activations(g, rows, cols):
    """bf16: normal, with 0.5 % of the channels 50 times as large."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    loud = torch.randperm(cols, device="cuda", generator=g)[: max(1, round(0.005 * cols))]
    x[:, loud] *= 50.0
    return x.to(torch.bfloat16)


def _codes(g, *shape):
    """Normal, reaching the largest code now and then."""
    return torch.randn(*shape, device="cuda", generator=g).mul_(35.0).round_().clamp_(-TOP, TOP).to(torch.int8)


def _operand_a(g, rows, k):
    return _codes(g, rows, k), torch.rand(rows, device="cuda", generator=g).add_(0.5).mul_(1.0 / 35.0)


def _operand_w(g, experts, n, k):
    codes = torch.empty(experts, n, k, device="cuda", dtype=torch.int8)
    for e in range(experts):
        codes[e] = _codes(g, n, k)
    return codes, torch.rand(experts, n, device="cuda", generator=g).add_(0.5).mul_(0.02 / 35.0)


def _routes(g, case):
    """Rows in expert order, as a router leaves them: their tokens, where each expert's begin, the most that an expert has.
    Some experts are busier than others, and with enough of them one has no rows."""
    experts, top = case["experts"], case["top"]
    logits = torch.randn(case["tokens"], experts, device="cuda", generator=g) + 0.5 * torch.randn(experts, device="cuda", generator=g)
    if experts > top:
        logits[:, experts - 1] = -math.inf
    chosen = logits.topk(top, dim=1).indices.reshape(-1)
    order = torch.argsort(chosen, stable=True)
    count = torch.bincount(chosen, minlength=experts)
    offsets = torch.zeros(experts + 1, device="cuda", dtype=torch.int32)
    offsets[1:] = count.cumsum(0)
    return (order // top).to(torch.int32), offsets, int(count.max())


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    if op == "route":
        experts = case["experts"]
        # (logits of a trained router: some experts are busier than others)
        logits = torch.randn(case["tokens"], experts, device="cuda", generator=g) * 1.5 + 0.5 * torch.randn(experts, device="cuda", generator=g)
        return {"op": op, "logits": logits if case["f32"] else logits.to(torch.bfloat16), "bias": 0.1 * torch.randn(experts, device="cuda", generator=g) if case["bias"] else None,
                "top": case["top"], "sigmoid": case["score"] == "sigmoid", "groups": case["groups"], "top_groups": case["top_groups"],
                "scale": 2.5 if case["score"] == "sigmoid" else 1.0}
    if op == "combine":
        tokens, top, cols = case["tokens"], case["top"], case["cols"]
        y = torch.randn(tokens * top, cols, device="cuda", generator=g)
        weights = torch.rand(tokens, top, device="cuda", generator=g) + 0.1
        return {"op": op, "y": y if case["f32"] else y.to(torch.bfloat16), "places": torch.randperm(tokens * top, device="cuda", generator=g).view(tokens, top).to(torch.int32),
                "weights": weights / weights.sum(1, keepdim=True), "f32": case["f32"],
                "shared": torch.randn(tokens, cols, device="cuda", generator=g).to(torch.bfloat16) if case["shared"] else None}
    if op == "quantize":
        return {"op": op, "x": _activations(g, case["rows"], case["cols"])}
    if op == "grouped":
        tokens, offsets, most = _routes(g, case)
        a = _operand_a(g, case["tokens"] if case["gather"] else case["tokens"] * case["top"], case["k"])
        return {"op": op, "a": a, "w": _operand_w(g, case["experts"], case["n"], case["k"]), "offsets": offsets,
                "rows": tokens if case["gather"] else None, "most": most}
    tokens, k = case["tokens"], case["k"]
    w, ws = _operand_w(g, 1, case["n"], k)
    s = {"op": op, "w": (w[0], ws[0])}
    if op == "gemm":
        return dict(s, a=_operand_a(g, tokens, k), f32=case["f32"])
    if op == "down":
        return dict(s, x=_activations(g, tokens, 2 * k))
    return dict(s, x=torch.randn(tokens, k, device="cuda", generator=g).to(torch.bfloat16), residual=_activations(g, tokens, k) if case["residual"] else None,
                weight=(1.0 + 0.2 * torch.randn(k, device="cuda", generator=g)).to(torch.bfloat16))


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2509_23202_amd import binding as fp4
    op = s["op"]
    if op == "route":
        flags = fp4.ROUTE_RENORM | (fp4.ROUTE_SIGMOID if s["sigmoid"] else 0) | (fp4.ROUTE_GROUP_SUM2 if s["groups"] > 1 and s["bias"] is not None else 0)
        weights, experts, rows, offsets, places = fp4.moe_route(s["logits"], s["top"], bias=s["bias"], groups=s["groups"], top_groups=s["top_groups"], scale=s["scale"], flags=flags)
        return {"weights": weights, "experts": experts, "rows": rows, "offsets": offsets, "places": places}
    if op == "combine":
        return fp4.moe_combine(s["y"], s["places"], s["weights"], shared=s["shared"], flags=fp4.OUT_F32 if s["f32"] else 0)
    if op == "quantize":
        codes, scales = fp4.int8_quantize(s["x"])
        return {"codes": codes, "scales": scales}
    if op == "gemm":
        return fp4.int8_gemm(*s["a"], *s["w"], flags=fp4.OUT_F32 if s["f32"] else 0)
    if op == "grouped":
        return fp4.int8_grouped_gemm(*s["a"], *s["w"], s["offsets"], rows=s["rows"])
    if op == "down":
        return fp4.int8_gemm(*fp4.int8_quantize(s["x"], flags=fp4.SILU_MUL), *s["w"])
    codes, scales, h = fp4.int8_rmsnorm_quantize(s["x"], s["weight"], EPS, residual=s["residual"])
    return {"out": fp4.int8_gemm(codes, scales, *s["w"]), "residual": h}


def _quantized(v):
    """Codes, in 32 bits, and scales of the rows of v."""
    amax = v.abs().amax(-1).clamp(min=AMAX_LEAST)
    return (v * (TOP / amax)[:, None]).round(), amax / TOP


def _product(a, a_scales, w):
    return (a @ w[0].float().t()) * a_scales[:, None] * w[1]


def _route_plain(s):
    # (64 bits: which of two scores is the larger decides)
    logits = s["logits"].double()
    tokens, experts = logits.shape
    if s["sigmoid"]:
        scores = 1.0 / (1.0 + torch.exp(-logits))
    else:
        scores = torch.exp(logits - logits.amax(1, keepdim=True))
        scores = scores / scores.sum(1, keepdim=True)
    choice = logits if s["bias"] is None else scores + s["bias"].double()
    if s["groups"] > 1:
        inside = choice.view(tokens, s["groups"], -1)
        if s["bias"] is not None:      # a group counts as its two best
            of_group = inside.sort(dim=2, descending=True).values[:, :, :2].sum(2)
        else:
            of_group = inside.amax(2)
        kept = of_group.sort(dim=1, descending=True, stable=True).indices[:, : s["top_groups"]]
        out = torch.ones(tokens, s["groups"], device=logits.device, dtype=torch.bool).scatter_(1, kept, False)
        choice = inside.masked_fill(out[:, :, None], -math.inf).view(tokens, experts)
    chosen = choice.sort(dim=1, descending=True, stable=True).indices[:, : s["top"]]      # equal ones: the first
    weights = scores.gather(1, chosen)
    weights = weights / weights.sum(1, keepdim=True) * s["scale"]
    order = torch.argsort(chosen.reshape(-1), stable=True)
    offsets = torch.zeros(experts + 1, device=logits.device, dtype=torch.int32)
    offsets[1:] = torch.searchsorted(chosen.reshape(-1)[order], torch.arange(experts, device=logits.device), right=True)
    places = torch.empty_like(order, dtype=torch.int32)
    places[order] = torch.arange(order.numel(), device=logits.device, dtype=torch.int32)
    return {"weights": weights.float(), "experts": chosen.to(torch.int32), "rows": (order // s["top"]).to(torch.int32), "offsets": offsets, "places": places.view(tokens, -1)}


def _run_plain(s):
    op = s["op"]
    if op == "route":
        return _route_plain(s)
    if op == "combine":
        y = (s["y"][s["places"].long()].float() * s["weights"][:, :, None]).sum(1)
        if s["shared"] is not None:
            y = y + s["shared"].float()
        return y if s["f32"] else y.to(torch.bfloat16)
    if op == "quantize":
        codes, scales = _quantized(s["x"].float())
        return {"codes": codes.to(torch.int8), "scales": scales}
    if op == "gemm":
        y = _product(s["a"][0].float(), s["a"][1], s["w"])
        return y if s["f32"] else y.to(torch.bfloat16)
    if op == "down":
        gate, up = s["x"].float().chunk(2, dim=1)
        return _product(*_quantized(gate / (1.0 + torch.exp(-gate)) * up), s["w"]).to(torch.bfloat16)
    if op == "project":
        h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(torch.bfloat16)
        f = h.float()
        v = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * s["weight"].float()
        return {"out": _product(*_quantized(v), s["w"]).to(torch.bfloat16), "residual": None if s["residual"] is None else h}
    # every expert's rows in a block of their own, padded to the most that an expert has
    a = s["a"][0].float() * s["a"][1][:, None]
    if s["rows"] is not None:
        a = a[s["rows"]]
    w = s["w"][0].float() * s["w"][1][..., None]
    row = torch.arange(a.shape[0], device=a.device, dtype=torch.int32)
    expert = torch.searchsorted(s["offsets"][1:], row, right=True)
    place = row - s["offsets"][expert]
    blocks = a.new_zeros(w.shape[0], s["most"], a.shape[1])
    blocks[expert, place] = a
    return torch.bmm(blocks, w.transpose(1, 2).contiguous())[expert, place].to(torch.bfloat16)


def exact(case, seed):
    """The definitions in 64 bits; codes are whole numbers and have no value here, and what a product reads has been rounded to them."""
    s = prepare(case, seed)
    op, f64 = s["op"], torch.float64
    if op == "route":
        z = s["logits"].to(f64)
        p = torch.sigmoid(z) if s["sigmoid"] else torch.softmax(z, 1)
        c = p if s["bias"] is None else p + s["bias"].to(f64)
        c = z.clone() if s["bias"] is None else c
        size = case["experts"] // case["groups"]
        if case["groups"] > 1:
            per = c.reshape(-1, case["groups"], size)
            mark = per.topk(min(2, size), dim=2).values.sum(2) if s["bias"] is not None else per.max(2).values
            lost = torch.argsort(mark, dim=1, descending=True, stable=True)[:, case["top_groups"]:]
            for q in range(lost.shape[1]):
                at = lost[:, q, None] * size + torch.arange(size, device=z.device)
                c = c.scatter(1, at, -math.inf)
        best = torch.argsort(c, dim=1, descending=True, stable=True)[:, : case["top"]]
        v = torch.take_along_dim(p, best, 1)
        return {"weights": s["scale"] * v / v.sum(1)[:, None], "experts": None, "rows": None, "offsets": None, "places": None}
    if op == "combine":
        y = torch.zeros(case["tokens"], case["cols"], device="cuda", dtype=f64) if s["shared"] is None else s["shared"].to(f64)
        for j in range(case["top"]):
            y = y + s["weights"][:, j].to(f64)[:, None] * s["y"].index_select(0, s["places"][:, j].long()).to(f64)
        return y
    if op == "quantize":
        return {"codes": None, "scales": s["x"].abs().max(1).values.to(f64).clamp(min=AMAX_LEAST) / TOP}
    if op == "gemm":
        return s["a"][0].to(f64).matmul(s["w"][0].to(f64).t()) * torch.outer(s["a"][1].to(f64), s["w"][1].to(f64))
    if op in ("down", "project"):
        h = None
        if op == "down":
            v = s["x"].to(f64)
            k = v.shape[1] // 2
            v = v[:, :k] * torch.sigmoid(v[:, :k]) * v[:, k:]
        else:
            h = s["x"].to(f64)
            if s["residual"] is not None:
                h = (h + s["residual"].to(f64)).to(torch.bfloat16).to(f64)   # the residual stream is kept in bf16
            v = h / (h.pow(2).sum(-1, keepdim=True) / h.shape[-1] + EPS).sqrt() * s["weight"].to(f64)
        scale = v.abs().max(-1, keepdim=True).values.clamp(min=AMAX_LEAST) / TOP
        y = torch.round(v / scale).matmul(s["w"][0].to(f64).t()) * scale * s["w"][1].to(f64)
        return y if op == "down" else {"out": y, "residual": None if s["residual"] is None else h}
    begin, out = s["offsets"].tolist(), []
    for e in range(case["experts"]):
        rows = slice(begin[e], begin[e + 1])
        if begin[e] == begin[e + 1]:
            continue
        at = rows if s["rows"] is None else s["rows"][rows].long()
        out.append(s["a"][0][at].to(f64).matmul(s["w"][0][e].to(f64).t()) * torch.outer(s["a"][1][at].to(f64), s["w"][1][e].to(f64)))
    return torch.cat(out)


def work(case):
    op = case["op"]
    if op == "route":
        t, e, top = case["tokens"], case["experts"], case["top"]
        return {"bytes": t * e * (4 if case["f32"] else 2) + (4 * e if case["bias"] else 0) + 16 * t * top + 4 * (e + 1), "flops": t * e * (4 + top)}
    if op == "combine":
        n, size = case["tokens"] * case["cols"], 4 if case["f32"] else 2
        return {"bytes": n * (case["top"] * size + size + (2 if case["shared"] else 0)) + 8 * case["tokens"] * case["top"], "flops": 2 * n * case["top"]}
    if op == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": 3 * n + 4 * case["rows"], "flops": 3 * n}
    n, k = case["n"], case["k"]
    weights = n * k + 4 * n
    if op == "grouped":
        rows = case["tokens"] * case["top"]
        # the experts that some row chose, counted as if all were equally likely (a token's choices differ)
        share = 1.0 - (1.0 - case["top"] / case["experts"]) ** case["tokens"]
        read = (case["tokens"] if case["gather"] else rows) * (k + 4)
        return {"bytes": read + case["experts"] * share * weights + rows * n * 2 + 4 * (case["experts"] + 1), "flops": 2 * rows * n * k}
    m = case["tokens"]
    product = 2 * m * n * k
    if op == "gemm":
        return {"bytes": m * (k + 4) + weights + m * n * (4 if case["f32"] else 2), "flops": product}
    if op == "down":
        return {"bytes": m * k * 4 + weights + m * n * 2, "flops": product + 12 * m * k}
    return {"bytes": m * k * (6 if case["residual"] else 2) + 2 * k + weights + m * n * 2, "flops": product + 10 * m * k}
