"""What the 8-bit linear operators are timed on, beside the plain form of each in elementary torch operations.

A case is a plain dict.  `op` says what a pass does:

  norm      fp8_rmsnorm_quantize: the residual's addition, the root-mean-square norm, E4M3 codes with a scale per 128 columns
  quantize  fp8_quantize: the codes and scales of activations, or of silu(gate) * up
  weights   fp8_quantize_weights: the codes and scales of weights, a scale per 128 x 128 block of each expert
  gemm      fp8_gemm: activations times weights, both in E4M3 with their scales
  grouped   fp8_grouped_gemm: the same with the rows sorted by expert, each expert with weights of its own

`own` chooses the framework's calls; otherwise run() computes the plain form, in 32 bits and rounded once.
"""
import math

import torch

own = False

BLOCK = 128            # columns to a scale
E4M3_MAX = 448.0       # the largest E4M3 value
AMAX_LEAST = 2.0 ** -100   # a block's abs-max counts as at least this
EPS = 1e-6


def listed():
    return [
        # One decoded token entering a layer of hidden size 4096: latency.
        {"name": "norm_m1", "op": "norm", "rows": 1, "cols": 4096, "residual": True, "norm_out": False},
        # An 8192-wide layer's prompt of 4095 tokens, with the normed rows in 16 bits too, as a router reads them.
        {"name": "norm_m4095_k8192", "op": "norm", "rows": 4095, "cols": 8192, "residual": True, "norm_out": True},
        # The gated activation in front of a down projection: a decoding batch with an odd number of tokens, and a prompt.
        {"name": "silu_m33", "op": "quantize", "rows": 33, "cols": 14336, "gated": True},
        {"name": "silu_m4096", "op": "quantize", "rows": 4096, "cols": 14336, "gated": True},
        # Weights on loading: a gate and up projection of the 70B-shaped layer, and 16 experts whose rows are no whole blocks.
        {"name": "weights_n57344", "op": "weights", "experts": 1, "rows": 57344, "cols": 8192},
        {"name": "weights_e16_n1000", "op": "weights", "experts": 16, "rows": 1000, "cols": 2048},
        # One token against a square projection: latency, and weights streamed from HBM.
        {"name": "gemm_m1", "op": "gemm", "tokens": 1, "n": 4096, "k": 4096, "f32": False},
        # A mixed batch with an odd number of tokens on the 70B-shaped q/k/v projection.
        {"name": "gemm_m201", "op": "gemm", "tokens": 201, "n": 10240, "k": 8192, "f32": False},
        # The 8B-shaped gate and up projection of a prompt, the largest ordinary product.
        {"name": "gemm_m4096", "op": "gemm", "tokens": 4096, "n": 28672, "k": 4096, "f32": False},
        # Sixteen decoded tokens, four experts each out of 64: the weights of the experts in use.
        {"name": "grouped_decode", "op": "grouped", "tokens": 16, "top": 4, "experts": 64, "n": 4096, "k": 4096, "gather": True},
        # A short prompt on a few experts, whole rows already in expert order, an odd number of columns.
        {"name": "grouped_ragged", "op": "grouped", "tokens": 389, "top": 2, "experts": 9, "n": 1001, "k": 2048, "gather": False},
        # A prompt of 4096 tokens, four experts each out of 64, the tokens' rows gathered by index.
        {"name": "grouped_prefill", "op": "grouped", "tokens": 4096, "top": 4, "experts": 64, "n": 4096, "k": 4096, "gather": True},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "quantize", "weights", "gemm", "gemm", "grouped", "grouped"])
    if op == "norm":
        return {"op": op, "rows": _log_int(rng, 1, 4096), "cols": BLOCK * _log_int(rng, 4, 64), "residual": rng.random() < 0.7,
                "norm_out": rng.random() < 0.4}
    if op == "quantize":
        return {"op": op, "rows": _log_int(rng, 1, 4096), "cols": BLOCK * _log_int(rng, 4, 112), "gated": rng.random() < 0.6}
    if op == "weights":
        experts = rng.choice([1, 1, _log_int(rng, 2, 32)])
        cols = BLOCK * _log_int(rng, 4, 64)
        return {"op": op, "experts": experts, "rows": min(_log_int(rng, 100, 28672), 57344 * 8192 // (experts * cols)), "cols": cols}
    if op == "gemm":
        n, k = _log_int(rng, 200, 28672), BLOCK * _log_int(rng, 4, 112)
        n = n // 8 * 8 if rng.random() < 0.7 else n
        most = 4096 * 28672 * 4096 // (n * k)
        return {"op": op, "tokens": max(1, min(_log_int(rng, 1, 4096), most)), "n": n, "k": k, "f32": rng.random() < 0.2}
    experts = _log_int(rng, 2, 64)
    n, k = _log_int(rng, 200, 4096), BLOCK * _log_int(rng, 4, 32)
    return {"op": op, "tokens": _log_int(rng, 1, 4096), "top": rng.randint(1, min(4, experts)), "experts": experts,
            "n": n // 8 * 8 if rng.random() < 0.7 else n, "k": k, "gather": rng.random() < 0.6}


def _activations(g, rows, cols):
    """bf16: normal, with 0.5 % of the channels 50 times as large."""
    x = torch.randn(rows, cols, device="cuda", generator=g)
    loud = torch.randperm(cols, device="cuda", generator=g)[: max(1, round(0.005 * cols))]
    x[:, loud] *= 50.0
    return x.to(torch.bfloat16)


def _operand_a(g, rows, k):
    """Activations in E4M3 with a scale for each 128 columns of a row."""
    x = _activations(g, rows, k).float().view(rows, k // BLOCK, BLOCK)
    amax = x.abs().amax(-1).clamp(min=AMAX_LEAST)
    return (x * (E4M3_MAX / amax)[..., None]).to(torch.float8_e4m3fn).view(rows, k), amax / E4M3_MAX


def _operand_w(g, experts, n, k):
    """Weights in E4M3, normal and reaching the largest value now and then, with a scale for each 128 x 128 block."""
    codes = torch.empty(experts, n, k, device="cuda", dtype=torch.float8_e4m3fn)
    for e in range(experts):
        codes[e] = torch.randn(n, k, device="cuda", generator=g).mul_(110.0).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    scales = torch.rand(experts, -(-n // BLOCK), k // BLOCK, device="cuda", generator=g).add_(0.5).mul_(0.02 / 110.0)
    return codes, scales


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
    if op == "norm":
        rows, cols = case["rows"], case["cols"]
        return {"op": op, "x": torch.randn(rows, cols, device="cuda", generator=g).to(torch.bfloat16),
                "residual": _activations(g, rows, cols) if case["residual"] else None,
                "weight": (1.0 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(torch.bfloat16), "norm_out": case["norm_out"]}
    if op == "quantize":
        return {"op": op, "x": _activations(g, case["rows"], case["cols"] * (2 if case["gated"] else 1)), "gated": case["gated"]}
    if op == "weights":
        w = torch.randn(case["experts"], case["rows"], case["cols"], device="cuda", generator=g, dtype=torch.bfloat16).mul_(0.02)
        return {"op": op, "w": w}
    if op == "gemm":
        w, ws = _operand_w(g, 1, case["n"], case["k"])
        return {"op": op, "a": _operand_a(g, case["tokens"], case["k"]), "w": (w[0], ws[0]), "f32": case["f32"]}
    tokens, offsets, most = _routes(g, case)
    a = _operand_a(g, case["tokens"] if case["gather"] else case["tokens"] * case["top"], case["k"])
    return {"op": op, "a": a, "w": _operand_w(g, case["experts"], case["n"], case["k"]), "offsets": offsets,
            "rows": tokens if case["gather"] else None, "most": most}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2509_23202_amd import binding as fp4
    op = s["op"]
    if op == "norm":
        norm = torch.empty_like(s["x"]) if s["norm_out"] else None
        codes, scales, h = fp4.fp8_rmsnorm_quantize(s["x"], s["weight"], EPS, residual=s["residual"], norm_out=norm)
        return {"codes": codes, "scales": scales, "residual": h, "norm": norm}
    if op == "quantize":
        codes, scales = fp4.fp8_quantize(s["x"], flags=fp4.SILU_MUL if s["gated"] else 0)
        return {"codes": codes, "scales": scales}
    if op == "weights":
        codes, scales = fp4.fp8_quantize_weights(s["w"])
        return {"codes": codes, "scales": scales}
    if op == "gemm":
        return fp4.fp8_gemm(*s["a"], *s["w"], flags=fp4.OUT_F32 if s["f32"] else 0)
    return fp4.fp8_grouped_gemm(*s["a"], *s["w"], s["offsets"], rows=s["rows"])


def _quantized(v):
    """Codes and scales of v [rows, cols] in 32 bits."""
    rows, cols = v.shape
    v = v.view(rows, cols // BLOCK, BLOCK)
    amax = v.abs().amax(-1).clamp(min=AMAX_LEAST)
    return (v * (E4M3_MAX / amax)[..., None]).view(rows, cols).to(torch.float8_e4m3fn), amax / E4M3_MAX


def _values_a(codes, scales):
    rows, k = codes.shape
    return (codes.float().view(rows, k // BLOCK, BLOCK) * scales[..., None]).view(rows, k)


def _values_w(codes, scales):
    n, k = codes.shape[-2:]
    v = codes.float().view(*codes.shape[:-1], k // BLOCK, BLOCK)
    return (v * scales.repeat_interleave(BLOCK, -2)[..., :n, :, None]).view(codes.shape)


def _run_plain(s):
    op = s["op"]
    if op == "norm":
        h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(torch.bfloat16)
        f = h.float()
        v = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * s["weight"].float()
        codes, scales = _quantized(v)
        return {"codes": codes, "scales": scales, "residual": None if s["residual"] is None else h,
                "norm": v.to(torch.bfloat16) if s["norm_out"] else None}
    if op == "quantize":
        v = s["x"].float()
        if s["gated"]:
            gate, up = v.chunk(2, dim=1)
            v = gate / (1.0 + torch.exp(-gate)) * up
        codes, scales = _quantized(v)
        return {"codes": codes, "scales": scales}
    if op == "weights":
        experts, n, k = s["w"].shape
        tall = -(-n // BLOCK)
        v = torch.nn.functional.pad(s["w"].float(), (0, 0, 0, tall * BLOCK - n)).view(experts, tall, BLOCK, k // BLOCK, BLOCK)
        amax = v.abs().amax((2, 4)).clamp(min=AMAX_LEAST)
        v = (v * (E4M3_MAX / amax)[:, :, None, :, None]).view(experts, tall * BLOCK, k)
        return {"codes": v[:, :n].to(torch.float8_e4m3fn), "scales": amax / E4M3_MAX}
    a, w = _values_a(*s["a"]), _values_w(*s["w"])
    if op == "gemm":
        y = a @ w.t()
        return y if s["f32"] else y.to(torch.bfloat16)
    # every expert's rows in a block of their own, padded to the most that an expert has
    if s["rows"] is not None:
        a = a[s["rows"]]
    row = torch.arange(a.shape[0], device=a.device, dtype=torch.int32)
    expert = torch.searchsorted(s["offsets"][1:], row, right=True)
    place = row - s["offsets"][expert]
    blocks = a.new_zeros(w.shape[0], s["most"], a.shape[1])
    blocks[expert, place] = a
    return torch.bmm(blocks, w.transpose(1, 2))[expert, place].to(torch.bfloat16)


def exact(case, seed):
    """The definitions in 64 bits.  Codes are compared before their rounding to 8 bits, as v / scale."""
    s = prepare(case, seed)
    op, f64 = s["op"], torch.float64
    if op in ("norm", "quantize", "weights"):
        out = {}
        if op == "norm":
            h = s["x"].to(f64)
            if s["residual"] is not None:
                h = (h + s["residual"].to(f64)).to(torch.bfloat16).to(f64)   # the residual stream is kept in bf16
            v = h / (h.pow(2).sum(-1, keepdim=True) / h.shape[-1] + EPS).sqrt() * s["weight"].to(f64)
            out = {"residual": None if s["residual"] is None else h, "norm": v if s["norm_out"] else None}
        elif op == "quantize":
            v = s["x"].to(f64)
            if s["gated"]:
                v = v[:, : v.shape[1] // 2].mul(torch.sigmoid(v[:, : v.shape[1] // 2])) * v[:, v.shape[1] // 2:]
        else:
            codes, scales = [], []
            for w in s["w"]:
                sc = torch.stack([rows.abs().amax(0).view(-1, BLOCK).amax(1).to(f64).clamp(min=AMAX_LEAST) / E4M3_MAX for rows in w.split(BLOCK, 0)])
                scales.append(sc)
                # (32 bits hold a bf16 over a scale to 1e-7, where a code has four bits)
                codes.append(torch.cat([rows.float() / r.float().repeat_interleave(BLOCK) for rows, r in zip(w.split(BLOCK, 0), sc)]))
            return {"codes": torch.stack(codes), "scales": torch.stack(scales)}
        scale = v.abs().reshape(v.shape[0], -1, BLOCK).max(-1).values.clamp(min=AMAX_LEAST) / E4M3_MAX
        return dict(out, codes=v / scale.repeat_interleave(BLOCK, 1), scales=scale)
    a = s["a"][0].to(f64) * s["a"][1].to(f64).repeat_interleave(BLOCK, 1)
    if op == "gemm":
        n = case["n"]
        rows = [(s["w"][0][i: i + BLOCK].to(f64) * s["w"][1][i // BLOCK].to(f64).repeat_interleave(BLOCK)) for i in range(0, n, BLOCK)]
        return torch.cat([a.matmul(r.t()) for r in rows], 1)
    begin, out = s["offsets"].tolist(), []
    for e in range(case["experts"]):
        rows = slice(begin[e], begin[e + 1])
        if begin[e] == begin[e + 1]:
            continue
        w = s["w"][0][e].to(f64) * s["w"][1][e].to(f64).repeat_interleave(BLOCK, 0)[: case["n"]].repeat_interleave(BLOCK, 1)
        out.append((a[rows] if s["rows"] is None else a[s["rows"][rows].long()]).matmul(w.t()))
    return torch.cat(out)


def work(case):
    op = case["op"]
    if op in ("norm", "quantize"):
        e = case["rows"] * case["cols"]
        if op == "norm":
            read, extra = 4 if case["residual"] else 2, (2 if case["residual"] else 0) + (2 if case["norm_out"] else 0)
            return {"bytes": e * (read + extra + 1) + e // BLOCK * 4 + 2 * case["cols"], "flops": 8 * e}
        return {"bytes": e * (5 if case["gated"] else 3) + e // BLOCK * 4, "flops": (10 if case["gated"] else 3) * e}
    if op == "weights":
        e = case["experts"] * case["rows"] * case["cols"]
        return {"bytes": 3 * e + case["experts"] * -(-case["rows"] // BLOCK) * (case["cols"] // BLOCK) * 4, "flops": 3 * e}
    n, k = case["n"], case["k"]
    weights = n * k + -(-n // BLOCK) * (k // BLOCK) * 4
    if op == "gemm":
        m = case["tokens"]
        return {"bytes": m * (k + k // BLOCK * 4) + weights + m * n * (4 if case["f32"] else 2), "flops": 2 * m * n * k}
    rows = case["tokens"] * case["top"]
    # the experts that some row chose, counted as if all were equally likely (a token's choices differ)
    share = 1.0 - (1.0 - case["top"] / case["experts"]) ** case["tokens"]
    read = (case["tokens"] if case["gather"] else rows) * (k + k // BLOCK * 4)
    return {"bytes": read + case["experts"] * share * weights + rows * n * 2 + 4 * (case["experts"] + 1), "flops": 2 * rows * n * k}
