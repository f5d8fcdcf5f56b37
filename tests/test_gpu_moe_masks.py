"""Router calls whose biases take experts out by a finite number, or differ in size: what a score leaves in doubt is a matter of the values that are compared."""
import numpy as np
import pytest
import torch

from tests import moe_util as R
from tests.fp8_util import f64
from tests.test_gpu_moe import check, fp4, logits, say  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("low", [-100.0, -1e4, -1e9, torch.finfo(torch.bfloat16).min, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("T,E,top,groups,top_groups", [(50, 16, 3, 1, 1), (700, 128, 8, 1, 1), (300, 256, 8, 8, 3), (5000, 96, 6, 8, 4), (5000, 256, 8, 8, 4), (40, 600, 20, 6, 2)])
def test_a_finite_mask_takes_an_expert_out_as_minus_infinity_does(fp4, low, T, E, top, groups, top_groups):
    """Bit for bit, and so in the same arithmetic: the tokens whose scores are formed in binary64 have weights of their own last bits, and a mask puts none of the others among them.
    Each group keeps two experts or loses all, so that a sum of two is one of scores."""
    say(f"finite masks {low} T={T} E={E} groups={groups}")
    z = logits(T, E, T + E)
    size = E // groups
    mask = torch.zeros(E, dtype=torch.bool)
    mask[1::3] = True
    for g in range(groups):
        mask[g * size : g * size + 2] = False
    if groups > 3:
        mask[-size:] = True
    bias = 0.2 * torch.randn(E, generator=torch.Generator().manual_seed(E))
    finite, out = (torch.where(mask, torch.tensor(v), bias).cuda() for v in (low, -float("inf")))
    for flags in (0, fp4.ROUTE_SIGMOID):
        for sum2 in (0, fp4.ROUTE_GROUP_SUM2) if groups > 1 else (0,):
            got, want = (fp4.moe_route(z, top, bias=b, groups=groups, top_groups=top_groups, flags=flags | sum2) for b in (finite, out))
            assert not mask.cuda()[want[1].long()].any()
            for g, w in zip(got, want):
                assert torch.equal(g, w)


@pytest.mark.parametrize("groups", [1, 16])
@pytest.mark.parametrize("big", [3.0, 1e3, 1e5, 1e7, 1e12])
def test_biases_beside_which_scores_lose_their_bits(fp4, groups, big):
    """Biases of two sizes, equal ones within each: where fp32 loses a score beside its bias, binary64 decides.  Of a group of two, one up and one down, the sum has few bits of either."""
    say(f"biases of {big} groups={groups}")
    T, E = 400, 32
    z = logits(T, E, int(big) % 1000)
    for bias in (torch.where(torch.arange(E) % 2 == 0, big, -big), torch.where(torch.arange(E) % 3 == 0, big, 0.0), torch.where(torch.arange(E) < E // 2, big, -big),
                 big + 1e-3 * torch.arange(E)):
        for sum2 in (0, fp4.ROUTE_GROUP_SUM2):
            for top_groups in {1, groups // 2 or 1, max(groups - 1, 1)}:
                for top in {1, min(8, E // groups * top_groups)}:
                    check(fp4, z, top, bias=bias.float().cuda(), groups=groups, top_groups=top_groups, flags=fp4.ROUTE_SIGMOID | sum2 | fp4.ROUTE_RENORM)
                    check(fp4, z, top, bias=bias.float().cuda(), groups=groups, top_groups=top_groups, flags=sum2)


def test_biases_of_every_size(fp4):
    """Many tokens, each bias of a size of its own from 2^-30 to 2^40, of either sign."""
    T, E = 3000, 64
    z = logits(T, E, 9, spread=3.0)
    g = torch.Generator().manual_seed(2)
    bias = (torch.randn(E, generator=g) * 2.0 ** torch.randint(-30, 40, (E,), generator=g)).float().cuda()
    for groups, top_groups in ((1, 1), (8, 3), (32, 9)):
        for flags in (fp4.ROUTE_SIGMOID, 0, fp4.ROUTE_GROUP_SUM2, fp4.ROUTE_GROUP_SUM2 | fp4.ROUTE_SIGMOID):
            check(fp4, z, 6, bias=bias, groups=groups, top_groups=top_groups, flags=flags)


def test_infinite_biases(fp4):
    """An expert of plus infinity comes before all others, two of them in the order of their index."""
    T, E = 100, 24
    z = logits(T, E, 4)
    bias = (0.2 * torch.randn(E, generator=torch.Generator().manual_seed(1))).cuda()
    bias[7] = bias[20] = float("inf")
    bias[3] = -float("inf")
    for groups, top_groups in ((1, 1), (4, 2)):
        for flags in (0, fp4.ROUTE_SIGMOID, fp4.ROUTE_GROUP_SUM2):
            weights, experts, *_ = check(fp4, z, 5, bias=bias, groups=groups, top_groups=top_groups, flags=flags)
            assert (experts[:, 0] == 7).all() and (experts[:, 1] == 20).all()


def test_what_a_run_with_one_expert_left_counts_as(fp4):
    """The one alone, where minus infinity takes the others out; where a finite bias does, the sum with it."""
    E, groups = 12, 3
    z = torch.zeros(2, E, device="cuda")                      # scores of 1/2
    bias = torch.full((E,), -0.9, device="cuda")              # c = -0.4, sums of two -0.8
    bias[4:8] = torch.tensor([-0.9, -float("inf"), -float("inf"), -float("inf")])
    bias[8:] = -1.2                                           # -0.7, -1.4
    flags = fp4.ROUTE_SIGMOID | fp4.ROUTE_GROUP_SUM2
    assert (check(fp4, z, 1, bias=bias, groups=groups, top_groups=1, flags=flags)[1] == 4).all()
    bias[5:8] = -1e30
    assert (check(fp4, z, 1, bias=bias, groups=groups, top_groups=1, flags=flags)[1] == 0).all()
    z[1, :8] = -float("inf")
    assert check(fp4, z, 1, bias=bias, groups=groups, top_groups=1, flags=flags)[1].flatten().tolist() == [0, 8]


@pytest.mark.parametrize("biased", [False, True])
def test_the_sum_of_two_means_nothing_with_one_run(fp4, biased):
    """Saturated scores are equal, logits are not: without a bias they are compared as they are, whatever the flag."""
    z = torch.linspace(30.0, 60.0, 16, device="cuda").repeat(3, 1)
    bias = torch.zeros(16, device="cuda") if biased else None
    got = [check(fp4, z, 3, bias=bias, flags=fp4.ROUTE_SIGMOID | f) for f in (0, fp4.ROUTE_GROUP_SUM2)]
    assert all(torch.equal(a, b) for a, b in zip(*got))
    if not biased:
        assert got[0][1][0].tolist() == [15, 14, 13]
