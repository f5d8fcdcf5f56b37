"""A router's choice and the experts' outputs added up, against their definitions in 64 bits (tests/moe_util.py)."""
import itertools
import sys

import numpy as np
import pytest
import torch

from tests import moe_util as R
from tests.fp8_util import f64

pytestmark = pytest.mark.gpu


def say(msg):
    print("[case] " + msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def fp4():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2509_23202_amd import binding
    return binding


def check(fp4, logits, top, **kw):
    """Everything that moe_route leaves: whole numbers exactly, weights within 2^-20, or 2^-50 of the scale (what its documentation says)."""
    bias, flags = kw.get("bias"), kw.pop("flags", 0)
    got = fp4.moe_route(logits, top, flags=flags, **kw)
    weights, experts, rows, offsets, places = got
    want = R.choose(f64(logits), top, None if bias is None else f64(bias), kw.get("groups", 1), kw.get("top_groups", 1), kw.get("scale", 1.0), bool(flags & fp4.ROUTE_SIGMOID),
                    bool(flags & fp4.ROUTE_RENORM), bool(flags & fp4.ROUTE_GROUP_SUM2))
    np.testing.assert_array_equal(experts.cpu().numpy(), want[1])
    np.testing.assert_array_equal(offsets.cpu().numpy(), want[3])
    np.testing.assert_array_equal(places.cpu().numpy(), want[4])
    np.testing.assert_array_equal(rows.cpu().numpy()[: want[3][-1]], want[2])
    w = weights.cpu().numpy().astype(np.float64)
    np.testing.assert_array_equal(np.isnan(w), np.isnan(want[0]))
    ok = ~np.isnan(w)
    assert (np.abs(w[ok] - want[0][ok]) <= np.abs(want[0][ok]) * 2.0 ** -20 + kw.get("scale", 1.0) * 2.0 ** -50).all()
    return got


def logits(T, E, seed, dtype=torch.float32, apart=0, spread=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E + apart, generator=g) * spread).to(dtype).cuda()[:, :E]


SIZES = [(1, 1, 1), (1, 64, 4), (2, 3, 3), (5, 8, 2), (16, 64, 6), (17, 60, 4), (33, 128, 8), (64, 65, 1), (65, 200, 10), (257, 256, 8), (100, 257, 5), (300, 512, 22), (40, 1000, 64), (1111, 16, 2), (4099, 32, 4)]


@pytest.mark.parametrize("T,E,top", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_route(fp4, T, E, top, dtype):
    """bf16 logits are equal often: the lower index is taken."""
    say(f"route T={T} E={E} top={top} {dtype}")
    z = logits(T, E, T + E, dtype, apart=3 if T % 2 else 0)
    bias = (0.2 * torch.randn(E, generator=torch.Generator().manual_seed(E))).cuda()
    for sigmoid, renorm, b in itertools.product((0, fp4.ROUTE_SIGMOID), (0, fp4.ROUTE_RENORM), (None, bias)):
        check(fp4, z, top, bias=b, scale=1.0 if b is None else 2.5, flags=sigmoid | renorm)


@pytest.mark.parametrize("T,E,top,groups,top_groups", [(1, 64, 4, 8, 3), (33, 256, 8, 8, 4), (50, 160, 6, 8, 3), (20, 60, 5, 20, 7), (9, 64, 5, 64, 9), (130, 512, 8, 4, 1), (70, 1000, 30, 50, 2), (300, 96, 7, 3, 2)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_route_by_groups(fp4, T, E, top, groups, top_groups, dtype):
    say(f"route by groups T={T} E={E} top={top} {top_groups} of {groups} {dtype}")
    z = logits(T, E, T + E, dtype)
    bias = (0.2 * torch.randn(E, generator=torch.Generator().manual_seed(E))).cuda()
    for sigmoid, sum2, b in itertools.product((0, fp4.ROUTE_SIGMOID), (0, fp4.ROUTE_GROUP_SUM2), (None, bias)):
        check(fp4, z, top, bias=b, groups=groups, top_groups=top_groups, flags=sigmoid | sum2 | fp4.ROUTE_RENORM)


@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("groups", [1, 4])
def test_masks_equal_logits_and_numbers_that_are_not_finite(fp4, biased, sigmoid, groups):
    """Rows of padding, rows with fewer experts left than are chosen, whole groups masked, equal logits, zeros of both signs, saturated scores, infinities and NaN."""
    E, top = 32, 4
    inf, nan = float("inf"), float("nan")
    z = logits(20, E, 5)
    z[1] = -inf
    z[2, 3:] = -inf
    z[3, :] = -inf
    z[3, 30] = 1.0
    z[4] = 2.0
    z[5, ::2], z[5, 1::2] = 0.0, -0.0
    z[6, 7] = nan
    z[7, 9] = inf
    z[8] = -1e30
    z[9] = 200.0
    z[9, 5] = 300.0
    z[10] = -300.0
    z[11, :8] = -inf
    z[12, 8:] = -inf
    z[12, :7] = -inf
    z[13] = -120.0 + torch.arange(E, device="cuda") * 1.0
    z[14] = -inf
    z[14, 3] = nan
    bias = (0.2 * torch.randn(E, generator=torch.Generator().manual_seed(1))).cuda() if biased else None
    for renorm, sum2 in itertools.product((0, fp4.ROUTE_RENORM), (0, fp4.ROUTE_GROUP_SUM2)):
        flags = renorm | sum2 | (fp4.ROUTE_SIGMOID if sigmoid else 0)
        check(fp4, z, top, bias=bias, groups=groups, top_groups=max(1, groups // 2), flags=flags)
        if biased:
            off = bias.clone()
            off[4:9] = -inf
            check(fp4, z, top, bias=off, groups=groups, top_groups=max(1, groups // 2), flags=flags)
            off[20] = nan
            w, e, _, offsets, _ = check(fp4, z, top, bias=off, groups=groups, top_groups=max(1, groups // 2), flags=flags)
            assert torch.isnan(w).all() and (e == -1).all() and (offsets == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,top,groups", [(8, 8, 1), (70, 16, 7), (256, 20, 8)])
def test_the_largest_and_lowest_logits_and_biases(fp4, dtype, E, top, groups):
    """Masks of the type's lowest value beside its largest one, whose difference is beyond the type, and biases beside which a score counts for nothing."""
    say(f"largest and lowest E={E} {dtype}")
    z = logits(40, E, E, dtype).clone()
    end = torch.finfo(dtype)
    z[0] = end.min
    z[1] = end.max
    z[2, ::2] = end.min
    z[3, 1:] = end.min
    z[4, 1::2], z[4, ::2] = end.max, end.min
    z[5, 3] = end.max
    z[6, 3] = end.min
    z[7] = -87.0 - torch.arange(E, device="cuda") % 3
    bias = torch.zeros(E, device="cuda")
    bias[1], bias[2], bias[4], bias[5] = 3e38, -3e38, 1e30, 3e38
    rising = torch.linspace(-3e38, 3e38, E, device="cuda")
    for sigmoid, renorm, b in itertools.product((0, fp4.ROUTE_SIGMOID), (0, fp4.ROUTE_RENORM), (None, bias, rising)):
        for g in {1, groups}:
            check(fp4, z, top, bias=b, groups=g, top_groups=(g + 1) // 2 if top <= E // g * ((g + 1) // 2) else g, flags=sigmoid | renorm)


@pytest.mark.parametrize("T", [16384, 30011])
def test_many_tokens(fp4, T):
    """Plain torch in 64 bits on the device: experts in descending order of their choice, a stable sort."""
    say(f"route T={T}")
    E, top = 128, 8
    z = logits(T, E, 1, torch.bfloat16)
    bias = (0.2 * torch.randn(E, generator=torch.Generator().manual_seed(E))).cuda()
    z[T // 2] = -float("inf")
    for b in (None, bias):
        weights, experts, rows, offsets, places = fp4.moe_route(z, top, bias=b, flags=fp4.ROUTE_SIGMOID)
        s = 1 / (1 + torch.exp(-z.double()))
        c = z.double() if b is None else s + b.double()
        chosen = c.sort(dim=1, descending=True, stable=True).indices[:, :top]
        chosen[T // 2] = -1
        assert torch.equal(experts, chosen.to(torch.int32))
        flat = torch.where(chosen < 0, E, chosen).reshape(-1)
        order = torch.argsort(flat, stable=True)[: (T - 1) * top]
        assert torch.equal(rows[: (T - 1) * top], (order // top).to(torch.int32))
        assert torch.equal(offsets.long(), torch.searchsorted(flat[order], torch.arange(E + 1, device="cuda")))
        want = torch.full((T * top,), -1, device="cuda")
        want[order] = torch.arange(order.numel(), device="cuda")
        assert torch.equal(places.reshape(-1).long(), want)


@pytest.mark.parametrize("T,E,top", [(40, 24, 3), (9000, 24, 3), (200003, 24, 3), (70001, 300, 2)])
def test_every_token_in_doubt(fp4, T, E, top):
    """Few different logits and biases: whatever the arithmetic, equal scores are equal, and every token's choice is among them.  Runs of tokens from a few to more than a bit to each of sixteen words holds."""
    say(f"route in doubt T={T} E={E}")
    g = torch.Generator().manual_seed(T)
    z = (torch.randint(0, 4, (T, E), generator=g).float() * 0.5).cuda()
    bias = (torch.arange(E) % 3 * 0.125).cuda()
    for flags in (fp4.ROUTE_SIGMOID, 0):
        weights, experts, rows, offsets, places = fp4.moe_route(z, top, bias=bias, flags=flags)
        s = 1 / (1 + torch.exp(-z.double())) if flags else z.double().softmax(1)
        # (softmax: sums of the same terms in other orders differ between rows, not within one: a row's equal logits have equal scores)
        chosen = (s + bias.double()).sort(dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(experts, chosen.to(torch.int32))
        assert ((weights - s.gather(1, chosen)).abs() <= s.gather(1, chosen) * 2.0 ** -20).all()
        flat = chosen.reshape(-1)
        order = torch.argsort(flat, stable=True)
        assert torch.equal(rows, (order // top).to(torch.int32))
        assert torch.equal(offsets.long(), torch.searchsorted(flat[order], torch.arange(E + 1, device="cuda")))


def test_as_many_tokens_as_there_may_be(fp4):
    say("route T=2^24")
    T, E, top = 1 << 24, 8, 2
    z = torch.randn(T, E, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    bias = (0.1 * torch.arange(E)).cuda()
    weights, experts, rows, offsets, places = fp4.moe_route(z, top, bias=bias, flags=fp4.ROUTE_SIGMOID)
    # (of two equal scores the lower index: eight experts in descending order of their score, chosen one by one)
    c = 1 / (1 + torch.exp(-z.double())) + bias.double()
    first = c.argmax(1)
    first = (c == c.gather(1, first[:, None])).float().argmax(1)
    c.scatter_(1, first[:, None], -1.0)
    second = (c == c.max(1, keepdim=True).values).float().argmax(1)
    assert torch.equal(experts[:, 0].long(), first) and torch.equal(experts[:, 1].long(), second)
    del c
    assert torch.equal(offsets[1:].long(), torch.bincount(experts.reshape(-1).long(), minlength=E).cumsum(0))
    flat = experts.reshape(-1)
    order = torch.argsort(flat, stable=True)
    assert torch.equal(rows.long(), order // top)
    assert torch.equal(places.reshape(-1)[order], torch.arange(T * top, device="cuda", dtype=torch.int32))


def test_no_tokens(fp4):
    weights, experts, rows, offsets, places = fp4.moe_route(torch.empty(0, 37, device="cuda"), 4)
    assert weights.shape == experts.shape == places.shape == (0, 4) and rows.numel() == 0 and offsets.shape == (38,) and (offsets == 0).all()
    assert fp4.moe_combine(torch.empty(0, 64, device="cuda"), places, weights).shape == (0, 64)


def test_rows_behind_the_last_are_left_as_they_were(fp4):
    T, E, top = 40, 16, 3
    z = logits(T, E, 3)
    z[::2] = -float("inf")
    L, st = fp4.lib, torch.cuda.current_stream().cuda_stream
    w, i32 = torch.empty(T, top, device="cuda"), lambda *s: torch.full(s, -77, dtype=torch.int32, device="cuda")
    experts, rows, offsets, places = i32(T, top), i32(T * top), i32(E + 1), i32(T, top)
    ws = torch.empty(fp4.moe_workspace_bytes(T, E, top), dtype=torch.uint8, device="cuda")
    assert L.moe_route(z.data_ptr(), E, None, T, E, top, 1, 1, 1.0, w.data_ptr(), experts.data_ptr(), rows.data_ptr(), offsets.data_ptr(), places.data_ptr(), ws.data_ptr(), ws.numel(),
                       fp4.INPUT_F32, st) == 0
    assert int(offsets[-1]) == T // 2 * top and (rows[T // 2 * top:] == -77).all() and (rows[: T // 2 * top] % 2 == 1).all()


# ---------------------------------------------------------------- the experts' outputs added up
@pytest.mark.parametrize("T,top,H", [(1, 1, 1), (1, 4, 4096), (5, 4, 7), (3, 2, 129), (130, 8, 2048), (77, 3, 1000), (4, 64, 72), (2, 6, 65544)])
@pytest.mark.parametrize("y_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shared", [None, torch.bfloat16, torch.float32])
def test_combine(fp4, T, top, H, y_type, shared):
    say(f"combine T={T} top={top} H={H} {y_type} {shared}")
    g = torch.Generator().manual_seed(T + H)
    R_ = T * top + 3
    y = torch.randn(R_, H, generator=g).to(y_type).cuda()
    places = torch.randperm(R_, generator=g)[: T * top].view(T, top).to(torch.int32).cuda()
    if T > 2:
        places[1, 0], places[2, top - 1], places[0] = -1, R_, 5       # nobody's, outside, and one row again and again
    weights = torch.randn(T, top, generator=g).cuda()
    s = None if shared is None else torch.randn(T, H, generator=g).to(shared).cuda()
    p, Y = places.cpu().long(), torch.cat([y.double().cpu(), torch.zeros(1, H, dtype=torch.float64)])
    p = torch.where((p < 0) | (p >= R_), R_, p)
    terms = Y[p] * weights.double().cpu()[:, :, None]
    want, size = terms.sum(1), terms.abs().sum(1)
    if s is not None:
        want, size = want + s.double().cpu(), size + s.double().cpu().abs()
    for f32 in (False, True):
        out = fp4.moe_combine(y, places, weights, shared=s, flags=fp4.OUT_F32 if f32 else 0)
        assert out.dtype == (torch.float32 if f32 else torch.bfloat16)
        # every partial sum within 2^-24 of the sum of magnitudes, one rounding to bf16 of 2^-8 of the value (at most) behind
        bound = size * top * 2.0 ** -24 + (0 if f32 else (want.abs() + size * top * 2.0 ** -24) * 2.0 ** -8)
        assert ((out.double().cpu() - want).abs() <= bound).all()
        if s is not None and s.dtype == out.dtype:
            place = s.clone()
            assert fp4.moe_combine(y, places, weights, shared=place, flags=fp4.OUT_F32 if f32 else 0, out=place) is place and torch.equal(place, out)


def test_combine_at_any_element_and_what_is_not_finite(fp4):
    T, top, H = 6, 3, 264
    y = torch.randn(20, H, device="cuda").to(torch.bfloat16)
    places = torch.randint(0, 20, (T, top), device="cuda", dtype=torch.int32)
    weights = torch.rand(T, top, device="cuda")
    want = fp4.moe_combine(y, places, weights)
    moved = torch.cat([y.new_zeros(3), y.reshape(-1)])[3:].view(20, H)
    out = torch.zeros(T * H + 1, device="cuda", dtype=torch.bfloat16)[1:].view(T, H)
    assert torch.equal(fp4.moe_combine(moved, places, weights, out=out), want)
    weights[2, 1] = float("nan")
    places[2, 1] = -1
    y[int(places[4, 0]), 9] = float("inf")
    got = fp4.moe_combine(y, places, weights)
    assert torch.isnan(got[2]).all() and not torch.isfinite(got[4, 9])


def test_router_and_experts_together_on_a_stream_and_in_a_graph(fp4):
    """Route, product by expert, combine: with weights that multiply by two to the expert's number every token's sum is known."""
    T, E, top, H = 40, 8, 3, 128
    w, sw = torch.zeros(E, H, H, dtype=torch.int8, device="cuda"), torch.ones(E, H, device="cuda")
    for e in range(E):
        w[e] = torch.eye(H, device="cuda").to(torch.int8)
        sw[e] = 2.0 ** e
    a = torch.randint(-9, 10, (T, H), device="cuda", dtype=torch.int8)
    sa = torch.ones(T, device="cuda")
    zs = [logits(T, E, i) for i in range(3)]
    zs[1][7] = -float("inf")
    z = zs[0].clone()

    def step():
        weights, experts, rows, offsets, places = fp4.moe_route(z, top, flags=fp4.ROUTE_RENORM)
        y = fp4.int8_grouped_gemm(a, sa, w, sw, offsets, rows=rows)
        return weights, experts, fp4.moe_combine(y, places, weights, flags=fp4.OUT_F32)

    def right(weights, experts, out):
        factor = (weights.double() * torch.where(experts < 0, 0.0, 2.0 ** experts.double())).sum(1, keepdim=True)
        want = a.double() * factor
        return bool(((out.double() - want).abs() <= want.abs() * 2.0 ** -21).all())

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            got = step()
    for rnd in range(2):
        for zi in zs:
            z.copy_(zi)
            eager = step()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, eager)) and right(*got)


def test_refusals_of_the_binding(fp4):
    z = logits(4, 16, 1)
    bias = torch.zeros(16, device="cuda")
    w, e, r, o, p = fp4.moe_route(z, 2)
    y = torch.zeros(8, 32, device="cuda", dtype=torch.bfloat16)
    for call in (lambda: fp4.moe_route(z.half(), 2), lambda: fp4.moe_route(z.cpu(), 2), lambda: fp4.moe_route(z.t(), 2), lambda: fp4.moe_route(z, 17), lambda: fp4.moe_route(z, 0),
                 lambda: fp4.moe_route(z, 2, bias=bias[:8]), lambda: fp4.moe_route(z, 2, bias=bias.bfloat16()), lambda: fp4.moe_route(z, 2, workspace=torch.empty(4096, dtype=torch.uint8)),
                 lambda: fp4.moe_combine(y.half(), p, w), lambda: fp4.moe_combine(y, p.long(), w), lambda: fp4.moe_combine(y, p, w[:3]), lambda: fp4.moe_combine(y.t(), p, w),
                 lambda: fp4.moe_combine(y, p, w, shared=y), lambda: fp4.moe_combine(y, p, w, out=torch.empty(4, 32, device="cuda"))):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: fp4.moe_route(z, 2, groups=3), lambda: fp4.moe_route(z, 2, groups=0), lambda: fp4.moe_route(z, 2, groups=4, top_groups=5), lambda: fp4.moe_route(z, 5, groups=4),
                 lambda: fp4.moe_route(z, 2, flags=fp4.OUT_F32), lambda: fp4.moe_route(logits(100, 16, 1), 2, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), lambda: fp4.moe_combine(y, p, w, flags=fp4.SILU_MUL),
                 lambda: fp4.moe_route(torch.zeros(2, 1025, device="cuda"), 2), lambda: fp4.moe_route(torch.zeros(2, 128, device="cuda"), 65)):
        with pytest.raises(fp4.Fp4mrError):
            call()


def test_flags_that_name_a_type_have_to_be_the_tensors(fp4):
    """Of the compiled calls too, which hand such calls on to the binding."""
    z = logits(4, 16, 1, torch.bfloat16)
    w, e, r, o, p = fp4.moe_route(z, 2)
    y = torch.zeros(8, 32, device="cuda", dtype=torch.bfloat16)
    for call in (lambda: fp4.moe_route(z, 2, flags=fp4.INPUT_F32), lambda: fp4.moe_combine(y, p, w, flags=fp4.INPUT_F32), lambda: fp4.moe_combine(y, p, w, shared=y[:4], flags=fp4.SHARED_F32)):
        with pytest.raises(AssertionError):
            call()
    assert torch.equal(fp4.moe_route(z.float(), 2, flags=fp4.INPUT_F32)[1], e)
    assert torch.equal(fp4.moe_combine(y.float(), p, w, flags=fp4.INPUT_F32), fp4.moe_combine(y, p, w))


def test_rows_and_outputs_beyond_32_bits(fp4):
    say("combine from 4.6e9 elements, and to as many")
    R_, H = 70000, 65544
    y = torch.zeros(R_, H, dtype=torch.bfloat16, device="cuda")
    y[-3:] = torch.randn(3, H, device="cuda").to(torch.bfloat16)
    places = torch.tensor([[R_ - 1, 0], [R_ - 3, R_ - 2]], dtype=torch.int32, device="cuda")
    weights = torch.tensor([[0.5, 1.0], [2.0, 0.25]], device="cuda")
    few = y[-3:].clone()
    small = torch.tensor([[2, -1], [0, 1]], dtype=torch.int32, device="cuda")
    assert torch.equal(fp4.moe_combine(y, places, weights), fp4.moe_combine(few, small, weights))
    del y
    many = torch.randint(0, 3, (R_, 1), dtype=torch.int32, device="cuda")
    out = fp4.moe_combine(few, many, torch.ones(R_, 1, device="cuda"))
    assert all(torch.equal(out[i : i + 5000], few[many[i : i + 5000, 0].long()]) for i in range(0, R_, 5000))
    del out
    out = fp4.moe_combine(few[:, 1:8].contiguous(), many, torch.ones(R_, 1, device="cuda"))
    assert torch.equal(out, few[many[:, 0].long(), 1:8])


def test_two_streams_at_once_and_two_graphs(fp4):
    """Both launches of a route, each call with a workspace of its own, on two streams that wait for nothing of each other's; then both recorded, with a workspace each, and replayed at once."""
    T, E, top = 700, 96, 6
    zs = [logits(T, E, 60 + i) for i in range(2)]
    assert fp4.moe_workspace_bytes(T, E, top) > 0
    want = [fp4.moe_route(z, top) for z in zs]
    rows = [int(w[3][-1]) for w in want]
    same = lambda got, i: all(torch.equal(g[: rows[i]] if g.dim() == 1 and g.numel() == T * top else g, w[: rows[i]] if w.dim() == 1 and w.numel() == T * top else w) for g, w in zip(got, want[i]))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in zs], [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(fp4.moe_route(zs[i], top))
    torch.cuda.synchronize()
    assert all(same(g, i) for i in range(2) for g in got[i])
    graphs, held = [torch.cuda.CUDAGraph() for _ in zs], []
    rooms = [torch.empty(fp4.moe_workspace_bytes(T, E, top), dtype=torch.uint8, device="cuda") for _ in zs]
    for i, s in enumerate(streams):
        with torch.cuda.stream(s), torch.cuda.graph(graphs[i], stream=s):
            held.append(fp4.moe_route(zs[i], top, workspace=rooms[i]))
    for _ in range(5):
        for t in (t for h in held for t in h):
            t.zero_()
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(same(h, i) for i, h in enumerate(held))


def test_combine_of_more_tokens_than_a_launch_has(fp4):
    """Wide rows: a launch takes 2^22 tokens.  Places, weights, the shared expert's rows and the outputs of the next one begin there; the sums are those of the same tokens in calls of their own."""
    say("combine of 2^22 + 600 tokens")
    T, H, top, R_ = (1 << 22) + 600, 1032, 2, 999
    g = torch.Generator(device="cuda").manual_seed(7)
    y = torch.randn(R_, H, device="cuda", generator=g).to(torch.bfloat16)
    places = torch.randint(-1, R_, (T, top), dtype=torch.int32, device="cuda", generator=g)
    weights = torch.randn(T, top, device="cuda", generator=g)
    shared = torch.empty(T, H, dtype=torch.bfloat16, device="cuda").random_(-100, 100, generator=g)
    out = fp4.moe_combine(y, places, weights, shared=shared)
    for at in range(0, T, 100000):
        part = slice(at, min(at + 100000, T))
        assert torch.equal(out[part], fp4.moe_combine(y, places[part], weights[part], shared=shared[part])), at
    # the tokens on both sides by the definition: two products and two sums in fp32, one rounding
    for part in (slice(0, 50), slice((1 << 22) - 50, (1 << 22) + 50), slice(T - 50, T)):
        terms = torch.where((places[part] >= 0)[:, :, None], y[places[part].clamp(min=0).long()], y.new_zeros(1)).double() * weights[part].double()[:, :, None]
        want, size = terms.sum(1) + shared[part].double(), terms.abs().sum(1) + shared[part].double().abs()
        bound = size * 2 * 2.0 ** -24
        assert ((out[part].double() - want).abs() <= bound + (want.abs() + bound) * 2.0 ** -8).all()
