"""The compiled form of the calls of the 8-bit integer layers and of the router against their Python form: the same outputs for what both take, and everything else handed on."""
import pytest
import torch

from tests import int8_util as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fp4():
    from paper_2509_23202_amd import binding
    assert binding._calls is not None
    return binding


def normal(*shape, dtype=torch.bfloat16, seed=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g).to(dtype)


@pytest.mark.parametrize("M,N,K", [(1, 40, 32), (9, 136, 1168), (64, 256, 8192)])
def test_compiled_calls_equal_the_python_ones(fp4, monkeypatch, M, N, K):
    (a, sa), (w, sw) = R.operand(M, K, 1), R.operand(N, K, 2, 0.01)
    x, weight, res, norm = normal(M, K + 8)[:, :K], normal(K, seed=2), normal(M, K, seed=3), torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    gated, experts = normal(M, 2 * K, seed=4), normal(3, N, K, seed=5)
    we, se = R.operand(3 * N, K, 6, 0.01)
    offsets, rows = torch.tensor([0, 1, M, M + 2], dtype=torch.int32, device="cuda"), (torch.arange(M + 2, dtype=torch.int32) % M).cuda()
    z, bias = normal(M, 48, dtype=torch.float32), normal(48, dtype=torch.float32, seed=8)
    y, places, weights = normal(40, N, seed=9), torch.randint(-1, 41, (M, 3), device="cuda", dtype=torch.int32), normal(M, 3, dtype=torch.float32, seed=10)
    shared = normal(M, N, seed=11)
    calls = [lambda: fp4.int8_gemm(a, sa, w, sw), lambda: fp4.int8_gemm(a, sa, w, sw, flags=fp4.OUT_F32), lambda: fp4.int8_quantize(x), lambda: fp4.int8_quantize(gated, flags=fp4.SILU_MUL),
             lambda: fp4.int8_quantize(experts), lambda: fp4.int8_rmsnorm_quantize(x, weight), lambda: fp4.int8_rmsnorm_quantize(x, weight, 1e-5, residual=res, norm_out=norm) + (norm.clone(),),
             lambda: fp4.int8_grouped_gemm(a, sa, we.view(3, N, K), se.view(3, N), offsets, rows=rows), lambda: fp4.moe_combine(y, places, weights),
             lambda: fp4.moe_combine(y.float(), places, weights, shared=shared, flags=fp4.OUT_F32), lambda: fp4.moe_combine(y, places, weights, shared=shared.float())]
    route = lambda **kw: [t for i, t in enumerate(fp4.moe_route(**kw))]
    calls += [lambda: route(logits=z, top=3), lambda: route(logits=z.bfloat16(), top=4, bias=bias, groups=4, top_groups=2, scale=2.0, flags=fp4.ROUTE_SIGMOID | fp4.ROUTE_RENORM | fp4.ROUTE_GROUP_SUM2)]
    flat = lambda out: [out] if isinstance(out, torch.Tensor) else [t for t in out if t is not None]
    got = [call() for call in calls]
    monkeypatch.setattr(fp4, "_calls", None)
    for one, call in zip(got, calls):
        two = call()
        assert len(flat(one)) == len(flat(two))
        for s, t in zip(flat(one), flat(two)):
            assert type(s) is torch.Tensor and s.dtype == t.dtype and s.shape == t.shape and s.stride() == t.stride() and torch.equal(s, t)


def test_other_calls_are_handed_on(fp4):
    (a, sa), (w, sw) = R.operand(2, 256, 1), R.operand(32, 256, 2)
    want = fp4.int8_gemm(a, sa, w, sw)
    out = torch.empty_like(want)
    assert fp4.int8_gemm(a, sa, w, sw, out=out) is out and torch.equal(out, want)
    sub = fp4.int8_gemm(torch.nn.Parameter(a, requires_grad=False), sa, w, sw)
    assert type(sub) is torch.Tensor and torch.equal(sub, want)
    z = normal(4, 16, dtype=torch.float32)
    one, two = fp4.moe_route(z, 2, scale=2), fp4.moe_route(z, 2, scale=2.0)       # (a scale that is a whole number)
    assert all(torch.equal(s, t) for s, t in zip(one, two))
    with pytest.raises(AssertionError):
        fp4.int8_gemm(a.t(), sa, w, sw)
    with pytest.raises(fp4.Fp4mrError):
        fp4.moe_route(z, 2, groups=3)


def test_an_error_of_the_device_is_raised_at_once(fp4):
    """Entry points that report one without having touched the device: each is called once, and the calls raise."""
    import ctypes
    names = ["int8_rmsnorm_quantize", "int8_quantize", "int8_gemm", "int8_workspace_bytes", "int8_grouped_gemm", "moe_route", "moe_workspace_bytes", "moe_combine"]
    functions = [getattr(fp4.lib, name) for name in names]
    address = lambda f: ctypes.cast(f, ctypes.c_void_p).value
    called, device = [], 7

    def stub(name):
        f = getattr(fp4.lib, name)
        return ctypes.CFUNCTYPE(f.restype, *f.argtypes)(lambda *args: called.append(name) or device)

    stubs = {name: stub(name) for name in names if "workspace" not in name}
    (a, sa), (w, sw) = R.operand(2, 256, 1), R.operand(32, 256, 2)
    x, off = normal(2, 256), torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    route = fp4.moe_route(normal(2, 8), 1)
    fp4._calls.bind8i(*(address(stubs.get(n, f)) for n, f in zip(names, functions)))
    try:
        for call in (lambda: fp4.int8_rmsnorm_quantize(x, x[0]), lambda: fp4.int8_quantize(x), lambda: fp4.int8_gemm(a, sa, w, sw), lambda: fp4.int8_grouped_gemm(a, sa, w[None], sw[None], off),
                     lambda: fp4.moe_route(x, 2), lambda: fp4.moe_combine(x, route[4], route[0])):
            with pytest.raises(fp4.Fp4mrError):
                call()
    finally:
        fp4._calls.bind8i(*(address(f) for f in functions))
    assert called == [n for n in names if "workspace" not in n]
