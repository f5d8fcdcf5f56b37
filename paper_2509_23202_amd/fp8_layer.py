"""A feed-forward layer kept at 8 bits, as a decoder runs it: the residual's addition and the norm leave quantized activations, which one
shared expert and a router's choice of experts multiply; the gated activations are quantized in front of the down projections.

    python -m paper_2509_23202_amd.fp8_layer [--hidden 4096] [--inter 2048] [--experts 32] [--top 4] [--tokens 1 64 2048]

prints for each number of tokens how long the layer takes and how far it is from the same layer in fp32 without quantization.
"""
import argparse

import torch

from . import binding as fp4


class Fp8Layer:
    """weights: norm [H]; router [E,H]; gate_up [E + 1, 2 I, H] and down [E + 1, H, I], the shared expert's last (all bf16)."""

    def __init__(self, norm, router, gate_up, down, top: int, eps: float = 1e-6):
        self.norm, self.router, self.top, self.eps = norm, router, top, eps
        self.experts = router.shape[0]
        self.gate_up, self.down = fp4.fp8_quantize_weights(gate_up), fp4.fp8_quantize_weights(down)

    def _routed(self, operand):
        return tuple(t[: self.experts] for t in operand)

    def _shared(self, operand):
        return tuple(t[self.experts] for t in operand)

    def route(self, x):
        """Rows in the experts' order: the token of each, where each expert's begin, each token's rows and weights."""
        weights, chosen = (x @ self.router.t()).float().softmax(1).topk(self.top, dim=1)
        order = torch.argsort(chosen.reshape(-1), stable=True)
        offsets = torch.zeros(self.experts + 1, dtype=torch.int32, device=x.device)
        offsets[1:] = torch.cumsum(torch.bincount(chosen.reshape(-1), minlength=self.experts), 0)
        place = torch.empty_like(order)
        place[order] = torch.arange(order.numel(), device=x.device)
        return (order // self.top).to(torch.int32), offsets, place.view(chosen.shape), weights / weights.sum(1, keepdim=True)

    def __call__(self, x, residual):
        """x, residual: bf16 [T,H].  Returns the layer's output and the new residual."""
        normed = torch.empty_like(x)
        codes, scales, residual = fp4.fp8_rmsnorm_quantize(x, self.norm, self.eps, residual=residual, norm_out=normed)
        tokens, offsets, place, weights = self.route(normed)
        y = fp4.fp8_grouped_gemm(codes, scales, *self._routed(self.gate_up), offsets, rows=tokens)
        y = fp4.fp8_grouped_gemm(*fp4.fp8_quantize(y, flags=fp4.SILU_MUL), *self._routed(self.down), offsets)
        shared = fp4.fp8_gemm(codes, scales, *self._shared(self.gate_up))
        shared = fp4.fp8_gemm(*fp4.fp8_quantize(shared, flags=fp4.SILU_MUL), *self._shared(self.down), flags=fp4.OUT_F32)
        # (every token's rows in the order of its choices: the same sum every time)
        return (shared + (y[place].float() * weights[..., None]).sum(1)).to(torch.bfloat16), residual


def make_weights(hidden: int, inter: int, experts: int, seed: int, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device=device, generator=g, dtype=torch.float32)
    return dict(norm=(1 + 0.1 * normal(hidden)).to(torch.bfloat16), router=(normal(experts, hidden) * hidden ** -0.5).to(torch.bfloat16),
                gate_up=torch.stack([(normal(2 * inter, hidden) * hidden ** -0.5).to(torch.bfloat16) for _ in range(experts + 1)]),
                down=torch.stack([(normal(hidden, inter) * inter ** -0.5).to(torch.bfloat16) for _ in range(experts + 1)]))


def plain_layer(w, x, residual, top: int, eps: float = 1e-6, dtype=torch.float32):
    """The same layer in `dtype` without quantization, token by token's experts in a loop over the experts."""
    h = (x.to(dtype) + residual.to(dtype)).to(torch.bfloat16)
    f = h.to(dtype)
    v = f * torch.rsqrt((f * f).mean(1, keepdim=True) + eps) * w["norm"].to(dtype)
    weights, chosen = (v.to(torch.bfloat16) @ w["router"].t()).float().softmax(1).topk(top, dim=1)
    weights = (weights / weights.sum(1, keepdim=True)).to(dtype)

    def expert(e, rows):
        gate, up = (rows @ w["gate_up"][e].to(dtype).t()).chunk(2, dim=1)
        return (gate / (1 + torch.exp(-gate)) * up) @ w["down"][e].to(dtype).t()

    y = expert(-1, v)
    for e in range(w["router"].shape[0]):
        token, choice = (chosen == e).nonzero(as_tuple=True)
        if token.numel():
            y[token] += expert(e, v[token]) * weights[token, choice, None]
    return y, h


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("hidden", 4096), ("inter", 2048), ("experts", 32), ("top", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--tokens", type=int, nargs="*", default=[1, 64, 2048])
    args = ap.parse_args()
    w = make_weights(args.hidden, args.inter, args.experts, 1)
    layer = Fp8Layer(w["norm"], w["router"], w["gate_up"], w["down"], args.top)
    for T in args.tokens:
        g = torch.Generator(device="cuda")
        g.manual_seed(T)
        x, residual = (torch.randn(T, args.hidden, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
        y, h = layer(x, residual)
        ref, ref_h = plain_layer(w, x, residual, args.top)
        off = float((y.float() - ref).norm() / ref.norm())
        assert torch.equal(h, ref_h)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(3):
            layer(x, residual)
        begin.record()
        for _ in range(10):
            layer(x, residual)
        end.record()
        end.synchronize()
        print(f"{T} tokens: {begin.elapsed_time(end) * 100:.0f} us a layer, {100 * off:.1f} % from fp32 without quantization", flush=True)


if __name__ == "__main__":
    main()
