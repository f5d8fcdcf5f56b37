"""The 8-bit operators together, as the feed-forward layer of paper_2509_23202_amd/fp8_layer.py runs them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,hidden,inter,experts,top", [(1, 512, 256, 4, 2), (7, 512, 384, 9, 3), (200, 1024, 512, 16, 4), (600, 640, 256, 3, 1)])
def test_layer_against_the_plain_one_in_64_bits(tokens, hidden, inter, experts, top):
    """A code is within 2^-4 of its value, 2.7 % of a vector's norm for values spread over the codes; weights and activations of two products, the
    first through the product of two of its outputs, add up to sqrt(2 (2.7^2 + 2.7^2) + 2.7^2 + 2.7^2) = 6.6 %.  Twice that is allowed."""
    from paper_2509_23202_amd.fp8_layer import Fp8Layer, make_weights, plain_layer
    print(f"[case] layer {tokens} {hidden} {inter} {experts} {top}", flush=True)
    w = make_weights(hidden, inter, experts, 3)
    g = torch.Generator(device="cuda")
    g.manual_seed(tokens)
    x, residual = (torch.randn(tokens, hidden, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    layer = Fp8Layer(w["norm"], w["router"], w["gate_up"], w["down"], top)
    y, h = layer(x, residual)
    ref, ref_h = plain_layer({k: v.cpu() for k, v in w.items()}, x.cpu(), residual.cpu(), top, dtype=torch.float64)
    assert torch.equal(h.cpu(), ref_h)
    # (a token whose choice of experts hangs on the last bit of its router's sums may differ: none of these does by more than its neighbours)
    off = (y.double().cpu() - ref).norm(dim=1) / ref.norm(dim=1)
    assert float((y.double().cpu() - ref).norm() / ref.norm()) < 0.132, off.max()
    again, _ = layer(x, residual)
    assert torch.equal(y, again)
