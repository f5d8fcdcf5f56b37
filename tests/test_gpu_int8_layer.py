"""The router's operators and the 8-bit integer ones together, as the feed-forward layers of paper_2509_23202_amd/fp8_layer.py run them."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SIZES = [(1, 512, 256, 4, 2), (7, 512, 384, 9, 3), (200, 1024, 512, 16, 4), (600, 640, 272, 3, 1)]


def inputs(tokens, hidden):
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    return tuple(torch.randn(tokens, hidden, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))


@pytest.mark.parametrize("tokens,hidden,inter,experts,top", SIZES)
def test_integer_layer_against_the_plain_one_in_64_bits(tokens, hidden, inter, experts, top):
    """A vector's codes are off by a step over sqrt 12 each, 1/440 of its largest value: 1 % of the norm where that is 4.4 times the root mean square (normal values, up to a thousand of them),
    2.5 % where it is 11 times (products of two such).  Weights and activations of two products, the first through the product of two of its outputs: sqrt(2 (1 + 1) + 2.5^2 + 1) = 3.4 %.
    Twice that is allowed."""
    from paper_2509_23202_amd.fp8_layer import Int8Layer, make_weights, plain_layer
    print(f"[case] int8 layer {tokens} {hidden} {inter} {experts} {top}", flush=True)
    w = make_weights(hidden, inter, experts, 3)
    x, residual = inputs(tokens, hidden)
    layer = Int8Layer(w["norm"], w["router"], w["gate_up"], w["down"], top)
    y, h = layer(x, residual)
    ref, ref_h = plain_layer({k: v.cpu() for k, v in w.items()}, x.cpu(), residual.cpu(), top, dtype=torch.float64)
    assert torch.equal(h.cpu(), ref_h)
    off = (y.double().cpu() - ref).norm(dim=1) / ref.norm(dim=1)
    assert float((y.double().cpu() - ref).norm() / ref.norm()) < 0.068, off.max()
    assert torch.equal(y, layer(x, residual)[0])


@pytest.mark.parametrize("tokens,hidden,inter,experts,top", [s for s in SIZES if s[2] % 128 == 0])
def test_e4m3_layer_with_either_routing(tokens, hidden, inter, experts, top):
    """The same choices (torch's topk leaves the order of equal bf16 logits open, so places are compared without theirs), weights within 2^-20 of each other and sums in another order: two roundings to bf16, 2^-8 of
    the value each, of nearly the same number."""
    from paper_2509_23202_amd import binding as fp4
    from paper_2509_23202_amd.fp8_layer import Fp8Layer, make_weights
    w = make_weights(hidden, inter, experts, 3)
    x, residual = inputs(tokens, hidden)
    args = (w["norm"], w["router"], w["gate_up"], w["down"], top)
    one, two = Fp8Layer(*args), Fp8Layer(*args, routing={"flags": fp4.ROUTE_RENORM})
    normed = fp4.fp8_rmsnorm_quantize(x, w["norm"], 1e-6, residual=residual, norm_out=(n := torch.empty_like(x))) and n
    (t1, o1, p1, w1), (t2, o2, p2, w2) = one.route(normed), two.route(normed)
    (p1, i1), (p2, i2) = p1.to(torch.int32).sort(1), p2.sort(1)
    w1, w2 = w1.gather(1, i1), w2.gather(1, i2)
    assert torch.equal(t1, t2) and torch.equal(o1, o2) and torch.equal(p1, p2) and ((w1 - w2).abs() <= w1 * 2.0 ** -19).all()
    (y1, h1), (y2, h2) = one(x, residual), two(x, residual)
    assert torch.equal(h1, h2)
    size = y1.float().abs()
    assert ((y1.float() - y2.float()).abs() <= size * 2.0 ** -7 + size.max() * 2.0 ** -17).all()


def test_integer_layer_with_groups_and_a_bias_in_a_graph():
    """A router with sigmoid scores, a bias and groups; padding among the tokens has no logits of its own here, so every token has its experts.  Recorded and replayed on other inputs."""
    from paper_2509_23202_amd import binding as fp4
    from paper_2509_23202_amd.fp8_layer import Int8Layer, make_weights
    T, H = 30, 512
    w = make_weights(H, 256, 16, 3)
    bias = 0.1 * torch.randn(16, device="cuda")
    layer = Int8Layer(w["norm"], w["router"], w["gate_up"], w["down"], 4,
                      routing=dict(bias=bias, groups=4, top_groups=2, scale=2.5, flags=fp4.ROUTE_SIGMOID | fp4.ROUTE_RENORM | fp4.ROUTE_GROUP_SUM2))
    sets = [inputs(T + i, H) for i in range(3)]
    x, residual = sets[0][0][:T].clone(), sets[0][1][:T].clone()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        layer(x, residual)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            y, h = layer(x, residual)
    for rnd in range(2):
        for a, b in sets:
            x.copy_(a[:T])
            residual.copy_(b[:T])
            eager, _ = layer(x, residual)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, eager) and torch.isfinite(y).all() and float(y.float().abs().sum()) > 0
