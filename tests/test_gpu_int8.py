"""The 8-bit integer layers against their definition (tests/int8_util.py): products and the codes of a tensor as it is bit for bit."""
import sys

import numpy as np
import pytest
import torch

from tests import int8_util as R

pytestmark = pytest.mark.gpu
U = R.U


def say(msg):
    print("[case] " + msg, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def fp4():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2509_23202_amd import binding
    return binding


def bf16(rows, cols, seed, apart=0, loud=True):
    """Rows of normal values, some channels louder, `apart` elements more between rows than they hold."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols + apart, generator=g)
    if loud:
        x[:, ::37] *= 40.0
    return x.to(torch.bfloat16).cuda()[:, :cols]


# ---------------------------------------------------------------- quantizers
@pytest.mark.parametrize("rows,K,apart", [(1, 16, 0), (5, 48, 8), (3, 384, 8), (33, 4096, 0), (130, 656, 24), (7, 14336, 0), (1, 16528, 8), (2100, 256, 0), (2, 33000, 0), (3, 65552, 0), (2, 131056, 0)])
def test_quantize_as_it_is(fp4, rows, K, apart):
    say(f"int8 quantize {rows}x{K} apart={apart}")
    K -= K % 16
    x = bf16(rows, K, rows + K, apart)
    codes, scales = fp4.int8_quantize(x)
    c, s = R.quantized(x)
    assert codes.shape == (rows, K) and scales.shape == (rows,)
    np.testing.assert_array_equal(codes.cpu().numpy(), c)
    np.testing.assert_array_equal(scales.cpu().numpy(), s)


@pytest.mark.parametrize("rows,K,apart", [(1, 16, 0), (5, 48, 8), (33, 4096, 0), (130, 656, 24), (7, 14336, 0), (2, 32784, 0), (2, 65552, 8)])
def test_quantize_of_gated_rows(fp4, rows, K, apart):
    say(f"int8 quantize gated {rows}x{K} apart={apart}")
    x = bf16(rows, 2 * K, rows + K, apart)
    codes, scales = fp4.int8_quantize(x, flags=fp4.SILU_MUL)
    v = R.f64(x)
    g, u = v[:, :K], v[:, K:]
    with np.errstate(over="ignore"):
        v = g / (1 + np.exp(-g)) * u
    # the exponential's argument is rounded in its product with log2 e (|g| / ln 2 steps of the exponent), the instruction, the sum, the reciprocal
    # and two products each within a step
    R.check_rows(codes, scales, v, (1.5 * np.minimum(np.abs(g), 128.0) + 8) * 2 * U)


def test_quantize_of_every_bf16_below_a_largest_one(fp4):
    """All numbers of fourteen binades below each of a few largest ones, the ones with exact halves (a mantissa of 127) among them: ties go to the even code."""
    rows = []
    for top in (0x42fe, 0x437e, 0x3f80, 0x3fff, 0x7f7f, 0x4049, 0x3ffe, 0x0080):      # 127, 254, 1, 1.99, the largest, pi, 1.98, the smallest normal
        bits = np.arange(max(top - 14 * 128, 0), top + 1, dtype=np.uint16)
        for sign in (0, 0x8000):
            rows.append(np.pad(bits | sign, (0, 1808 - len(bits)), mode="edge"))
    x = torch.from_numpy(np.stack(rows).view(np.int16)).cuda().view(torch.bfloat16)
    codes, scales = fp4.int8_quantize(x)
    c, s = R.quantized(x)
    np.testing.assert_array_equal(codes.cpu().numpy(), c)
    np.testing.assert_array_equal(scales.cpu().numpy(), s)


def test_quantize_of_zeros_and_of_the_smallest_numbers(fp4):
    x = torch.zeros(4, 256, dtype=torch.bfloat16, device="cuda")
    x[1, :128] = 1e-38
    x[2, 7] = 2.0 ** -100
    x[2, 8] = -2.0 ** -102
    x[3, 130] = 2.0 ** -133      # the smallest subnormal
    codes, scales = fp4.int8_quantize(x)
    c, s = R.quantized(x)
    np.testing.assert_array_equal(codes.cpu().numpy(), c)
    np.testing.assert_array_equal(scales.cpu().numpy(), s)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("K", [384, 70000 - 70000 % 16])
def test_a_number_that_is_not_finite_stays_in_its_row(fp4, bad, K):
    x = bf16(5, K, 3)
    x[2, 200] = bad
    codes, scales = fp4.int8_quantize(x)
    assert torch.isfinite(scales.cpu())[[0, 1, 3, 4]].all() and not torch.isfinite(scales[2])
    y = x.clone()
    y[2] = 0
    codes2, scales2 = fp4.int8_quantize(y)
    keep = [0, 1, 3, 4]
    assert torch.equal(codes[keep], codes2[keep]) and torch.equal(scales[keep], scales2[keep])
    w, ws = R.operand(48, K, 4)
    out = fp4.int8_gemm(codes, scales, w, ws)
    assert not torch.isfinite(out[2]).any() and torch.isfinite(out[keep]).all()
    gated = torch.cat([x, x], 1)
    gated[2, 200] = 1.0        # (the up half alone)
    codes, scales = fp4.int8_quantize(gated, flags=fp4.SILU_MUL)
    assert torch.isfinite(scales.cpu())[keep].all() and not torch.isfinite(scales[2])


@pytest.mark.parametrize("shape", [(1, 16), (127, 256), (1, 1, 128), (3, 200, 272), (5, 129, 1024)])
def test_quantize_of_weights(fp4, shape):
    w = bf16(int(np.prod(shape[:-1])), shape[-1], 5).contiguous().view(shape)
    codes, scales = fp4.int8_quantize(w)
    c, s = R.quantized(w)
    assert codes.shape == shape and scales.shape == shape[:-1]
    np.testing.assert_array_equal(codes.cpu().numpy(), c)
    np.testing.assert_array_equal(scales.cpu().numpy(), s)


@pytest.mark.parametrize("rows,K,apart", [(1, 16, 0), (5, 528, 8), (3, 656, 0), (4, 2048, 0), (2, 2192, 16), (1, 4096, 0), (300, 4096, 0), (3, 8192, 8), (2, 8208, 0), (2, 16384, 0), (1, 16528, 0),
                                          (2, 65536, 0)])
@pytest.mark.parametrize("residual,norm", [(False, False), (True, False), (True, True)])
def test_rmsnorm_quantize(fp4, rows, K, apart, residual, norm):
    say(f"int8 rmsnorm {rows}x{K} apart={apart} residual={residual} norm={norm}")
    x, r = bf16(rows, K, 7 + K, apart, loud=False), bf16(rows, K, 8 + K) if residual else None
    w = (1.0 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(9))).to(torch.bfloat16).cuda()
    n = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda") if norm else None
    codes, scales, h = fp4.int8_rmsnorm_quantize(x, w, 1e-5, residual=r, norm_out=n)
    if residual:
        assert torch.equal(h, (x.float() + r.float()).to(torch.bfloat16))
    else:
        assert h is None
    f = R.f64(h if residual else x)
    v = f / np.sqrt((f * f).mean(1, keepdims=True) + 1e-5) * R.f64(w)
    # sum of squares: at most 64 values in a thread, then 6 + 15 additions; half of that in the root, whose own steps, two products and the division by K add eight
    delta = (0.5 * (64 + 21) + 8) * U
    R.check_rows(codes, scales, v, delta)
    if norm:
        assert (np.abs(R.f64(n) - v) <= np.abs(v) * (2.0 ** -8 + delta)).all()


def test_rmsnorm_in_place_and_of_a_row_of_zeros(fp4):
    K = 1296
    x, r = bf16(9, K, 1), bf16(9, K, 2)
    x[4] = 0
    r[4] = 0
    w = torch.full((K,), 0.5, dtype=torch.bfloat16, device="cuda")
    ref = fp4.int8_rmsnorm_quantize(x, w, 1e-6, residual=r)
    for target in ("residual", "x"):
        xx, rr = x.clone(), r.clone()
        out = fp4.int8_rmsnorm_quantize(xx, w, 1e-6, residual=rr, residual_out=rr if target == "residual" else xx)
        assert all(torch.equal(a, b) for a, b in zip(out, ref))
    assert (ref[0][4] == 0).all() and torch.isfinite(ref[1]).all()


def test_more_rows_than_a_launch_has(fp4):
    K, first = 64, 1 << 21
    rows = first + 600
    torch.manual_seed(5)
    x, r = (torch.randn(rows, K, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.randn(K, device="cuda").to(torch.bfloat16)
    norm = torch.empty_like(x)
    got = fp4.int8_rmsnorm_quantize(x, w, 1e-5, residual=r, norm_out=norm) + (norm,) + fp4.int8_quantize(x)
    for part in (slice(0, first), slice(first, rows)):
        n = torch.empty_like(x[part])
        want = fp4.int8_rmsnorm_quantize(x[part], w, 1e-5, residual=r[part], norm_out=n) + (n,) + fp4.int8_quantize(x[part])
        for g, e in zip(got, want):
            assert torch.equal(g[part], e)


# ---------------------------------------------------------------- products
SHAPES = [(1, 16, 16), (1, 4096, 4096), (2, 1, 272), (3, 129, 384), (15, 200, 656), (16, 1000, 2048), (17, 136, 1168), (33, 72, 14336), (64, 256, 512), (65, 257, 880), (100, 520, 256),
          (128, 128, 128), (129, 640, 400), (200, 1001, 1024), (256, 512, 2048), (257, 264, 624), (300, 96, 4096), (512, 768, 256), (700, 1288, 384), (1030, 200, 144), (201, 5001, 2896)]


def check_gemm(fp4, M, N, K, f32, workspace=None):
    (a, sa), (w, sw) = R.operand(M, K, M + K), R.operand(N, K, N + K, 0.01)
    ops = [R.around(t, 0x7f if t.dtype != torch.float32 else 0xff) for t in (a, sa, w, sw)]
    flags = fp4.OUT_F32 if f32 else 0
    room = torch.full((M * N * (4 if f32 else 2) + 8192,), 0x5a, dtype=torch.uint8, device="cuda")
    out = room[4096: -4096].view(torch.float32 if f32 else torch.bfloat16).view(M, N)
    fp4.int8_gemm(*ops, flags=flags, out=out, workspace=workspace)
    want = R.product(a, sa, w, sw, out.dtype)
    assert torch.equal(out.cpu(), want), f"{(out.cpu() != want).sum()} of {M * N}"
    assert (room[:4096] == 0x5a).all() and (room[-4096:] == 0x5a).all()
    return a, sa, w, sw, out


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("f32", [False, True])
def test_gemm(fp4, M, N, K, f32):
    """Every code in both operands; the bytes beside the operands, and their scales' neighbours, reach no output."""
    say(f"int8_gemm M={M} N={N} K={K} f32={f32}")
    a, sa, w, sw, out = check_gemm(fp4, M, N, K, f32)
    assert torch.equal(out, fp4.int8_gemm(a, sa, w, sw, flags=fp4.OUT_F32 if f32 else 0))


@pytest.mark.parametrize("M", [1, 20, 70, 300])
@pytest.mark.parametrize("low", [(-128, -128), (-128, 127), (127, 127)])
def test_the_largest_sums_have_32_bits(fp4, M, low):
    """K at its most, every code the largest: 2^14 (2^17 - 16) is below 2^31."""
    K, N = 131056, 40
    a, w = torch.full((M, K), low[0], dtype=torch.int8, device="cuda"), torch.full((N, K), low[1], dtype=torch.int8, device="cuda")
    one = lambda n: torch.ones(n, device="cuda")
    out = fp4.int8_gemm(a, one(M), w, one(N), flags=fp4.OUT_F32)
    assert (out == float(np.float32(low[0] * low[1] * K))).all()


KERNELS = list(range(1, 10))
PARTS = [9 * p + k for p in (1, 2, 3) for k in (5, 6, 7)]        # 2, 4 and 8 parts of three of them


@pytest.fixture
def forced(fp4):
    """Forces a kernel of the products for one test."""
    yield lambda kernel: fp4.set_option(fp4.OPT_INT8_VARIANT, kernel)
    fp4.set_option(fp4.OPT_INT8_VARIANT, 0)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("M,N,K", [(1, 16, 16), (5, 130, 144), (70, 300, 1168), (300, 520, 2064), (33, 1100, 640)])
def test_every_kernel(fp4, forced, kernel, M, N, K):
    say(f"int8 kernel {kernel} M={M} N={N} K={K}")
    forced(kernel)
    for f32 in (False, True):
        check_gemm(fp4, M, N, K, f32)


@pytest.mark.parametrize("kernel", PARTS)
@pytest.mark.parametrize("M,N,K", [(70, 300, 3856), (1, 130, 4112), (300, 257, 8192)])
def test_in_parts_of_k(fp4, forced, kernel, M, N, K):
    say(f"int8 kernel {kernel} M={M} N={N} K={K}")
    forced(kernel)
    for f32 in (False, True):
        check_gemm(fp4, M, N, K, f32, workspace=torch.full((8 * M * N * 4,), 0xff, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("kernel", KERNELS)
def test_a_walk_over_tiles_on_every_kernel(fp4, forced, kernel):
    """More tiles than workgroups, of a K of one step and of a few: the next tile's loads and scales beside this one's output."""
    forced(kernel)
    for M, N, K in ((3000, 5000, 48), (2100, 9000, 400)):
        say(f"int8 kernel {kernel} M={M} N={N} K={K}")
        check_gemm(fp4, M, N, K, kernel % 2 == 0)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("gather", [None, 50])
def test_grouped_on_every_kernel(fp4, forced, kernel, gather):
    say(f"int8 grouped kernel {kernel} gather={gather}")
    forced(kernel)
    grouped(fp4, [70, 0, 3, 129, 0, 300, 64, 257, 1, 40], 1100, 656, kernel, gather)
    grouped(fp4, [i % 5 for i in range(200)], 72, 512, kernel, gather, f32=True)


def grouped(fp4, counts, N, K, seed, gather=None, f32=False):
    E, T = len(counts), sum(counts)
    rows = gather or T
    (a, sa), (w, sw) = R.operand(rows, K, seed), R.operand(E * N, K, seed + 1, 0.01)
    w, sw = w.view(E, N, K), sw.view(E, N)
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    offsets[1:] = torch.tensor(counts, dtype=torch.int32).cumsum(0)
    index = torch.randint(0, rows, (T,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda() if gather else None
    ops = [R.around(t, 0x7f if t.dtype != torch.float32 else 0xff) for t in (a, sa, w, sw)]
    flags = fp4.OUT_F32 if f32 else 0
    out = fp4.int8_grouped_gemm(*ops, offsets.cuda(), rows=index, flags=flags)
    at = torch.arange(T) if index is None else index.cpu().long()
    b = offsets.tolist()
    want = torch.cat([R.product(a.cpu()[at[b[e]: b[e + 1]]], sa.cpu()[at[b[e]: b[e + 1]]], w[e], sw[e], out.dtype) for e in range(E)])
    assert torch.equal(out.cpu(), want), f"{(out.cpu() != want).sum()} of {out.numel()}"


COUNTS = [([5], 48, 272, None), ([3, 0, 7, 1], 130, 400, None), ([16, 17, 0, 0, 31, 64, 65], 264, 640, 40), ([200, 0, 300], 1001, 256, 77), ([1] * 70, 72, 512, 9), ([0, 0, 40], 64, 4112, None),
          ([130, 128, 257, 0, 5], 520, 384, 300)]


@pytest.mark.parametrize("counts,N,K,gather", COUNTS)
def test_grouped_gemm(fp4, counts, N, K, gather):
    say(f"int8 grouped {len(counts)} experts, {sum(counts)} rows, N={N} K={K} gather={gather}")
    grouped(fp4, counts, N, K, len(counts) + N, gather, f32=N % 16 == 0)


@pytest.mark.parametrize("T,counts", [(50, [20, 0, 10]), (300, [130, 60]), (9, [0, 0])])
def test_grouped_rows_of_no_expert_and_indexes_outside(fp4, T, counts):
    K, N = 656, 136
    (a, sa), (w, sw) = R.operand(12, K, 1), R.operand(len(counts) * N, K, 2, 0.01)
    w, sw = w.view(-1, N, K), sw.view(-1, N)
    sw[0, 3] = float("inf")
    index = torch.randint(0, 12, (T,), dtype=torch.int32, generator=torch.Generator().manual_seed(3))
    outside = [0, 4, T - 1]
    index[outside] = torch.tensor([-1, 12, 2 ** 31 - 1], dtype=torch.int32)
    offsets = torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(torch.int32)
    out = torch.full((T, N), -7.0, device="cuda")
    fp4.int8_grouped_gemm(a, sa, w, sw, offsets.cuda(), rows=index.cuda(), flags=fp4.OUT_F32, out=out)
    out, have = out.cpu(), int(offsets[-1])
    assert (out[have:] == -7.0).all()
    for e, n in enumerate(counts):
        for t in range(int(offsets[e]), int(offsets[e + 1])):
            if t in outside:
                bad = torch.isnan(out[t])
                assert bool(bad[3]) == (e == 0) and bad.sum() == (e == 0) and (out[t][~bad] == 0).all()
            else:
                i = int(index[t])
                want = R.product(a[i: i + 1], sa[i: i + 1], w[e], sw[e], torch.float32)[0]
                assert torch.equal(out[t].nan_to_num(9.0, 9.0, 9.0), want.nan_to_num(9.0, 9.0, 9.0))


@pytest.mark.parametrize("offsets", [[-5, 20, 30, 1000], [0, 30, 10, 50], [50, 0, 0, 0], [2 ** 31 - 1, -2 ** 31, 7, 7]])
def test_grouped_offsets_stay_within_the_rows(fp4, offsets):
    """A number outside the rows counts as the nearest within; decreasing ones leave it open which products the rows hold, and reach nothing else."""
    T, K, N = 50, 272, 72
    (a, sa), (w, sw) = R.operand(T, K, 1), R.operand(3 * N, K, 2, 0.01)
    room = torch.full((T * N + 4096,), 3.0, dtype=torch.bfloat16, device="cuda")
    out = room[2048: -2048].view(T, N)
    fp4.int8_grouped_gemm(a, sa, w.view(3, N, K), sw.view(3, N), torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=out)
    assert (room[:2048] == 3.0).all() and (room[-2048:] == 3.0).all()
    if offsets[0] == -5:
        assert torch.equal(out, fp4.int8_grouped_gemm(a, sa, w.view(3, N, K), sw.view(3, N), torch.tensor([0, 20, 30, 50], dtype=torch.int32, device="cuda")))


def test_outputs_and_scales_at_any_element(fp4):
    M, N, K = 35, 77, 272
    (a, sa), (w, sw) = R.operand(M, K, 1), R.operand(N, K, 2, 0.01)
    shifted = lambda t, by: torch.cat([torch.zeros(by, device="cuda", dtype=t.dtype), t.reshape(-1)])[by:].view(t.shape)
    for f32 in (False, True):
        want = fp4.int8_gemm(a, sa, w, sw, flags=fp4.OUT_F32 if f32 else 0)
        out = torch.zeros(M * N + 3, device="cuda", dtype=want.dtype)[3:].view(M, N)
        fp4.int8_gemm(a, shifted(sa, 1), w, shifted(sw, 3), flags=fp4.OUT_F32 if f32 else 0, out=out)
        assert torch.equal(out, want)


def test_no_rows(fp4):
    w, sw = R.operand(32, 256, 1)
    a, sa = torch.empty(0, 256, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda")
    x = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    assert fp4.int8_gemm(a, sa, w, sw).shape == (0, 32)
    assert fp4.int8_grouped_gemm(a, sa, w[None], sw[None], torch.zeros(2, dtype=torch.int32, device="cuda")).shape == (0, 32)
    assert fp4.int8_quantize(x)[0].shape == (0, 256)
    assert fp4.int8_rmsnorm_quantize(x, torch.ones(256, dtype=torch.bfloat16, device="cuda"), residual=x)[2].shape == (0, 256)


def test_weights_of_more_than_4_gb(fp4):
    """The last expert's weights begin beyond 2^32 bytes, and a single matrix's rows too."""
    K, N, E = 16384, 16384, 18
    say("int8 grouped with 4.8 GB of weights")
    w = torch.zeros(E, N, K, dtype=torch.int8, device="cuda")
    (last, s_last), (a, sa) = R.operand(N, K, 3, 0.01), R.operand(20, K, 4)
    w[E - 1] = last
    sw = torch.zeros(E, N, device="cuda")
    sw[E - 1] = s_last
    pick = torch.tensor([0, 1, 8191, 16383], device="cuda")
    want = R.product(a, sa, last[pick], s_last[pick], torch.bfloat16)
    out = fp4.int8_grouped_gemm(a, sa, w, sw, torch.tensor([0] * E + [20], dtype=torch.int32, device="cuda"))
    assert torch.equal(out[:, pick].cpu(), want)
    flat = fp4.int8_gemm(a, sa, w.view(E * N, K), sw.view(-1))
    assert torch.equal(flat[:, pick + (E - 1) * N].cpu(), want) and (flat[:, :-N] == 0).all()


def test_streams_and_graphs(fp4):
    """The path on a stream of its own, then recorded and replayed on other inputs, eager work between the replays."""
    K, N, E, T = 528, 544, 4, 24
    w, sw = fp4.int8_quantize(bf16(E * N, K, 1).contiguous().view(E, N, K))
    w2, sw2 = fp4.int8_quantize(bf16(48, 272, 2).contiguous())
    ones = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0, 7, 7, 20, T], dtype=torch.int32, device="cuda")
    index = (torch.arange(T, dtype=torch.int32) * 5 % 12).cuda()
    xs = [bf16(12, K, 20 + i) for i in range(3)]
    x, res = xs[0].clone(), bf16(12, K, 30)

    def step():
        c, s, h = fp4.int8_rmsnorm_quantize(x, ones, residual=res)
        y = fp4.int8_grouped_gemm(c, s, w, sw, offsets, rows=index)
        return h, y, fp4.int8_gemm(*fp4.int8_quantize(y, flags=fp4.SILU_MUL), w2, sw2)

    ref = []
    for xi in xs:
        x.copy_(xi)
        ref.append([t.clone() for t in step()])
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        x.copy_(xs[0])
        got = step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref[0]))
        with torch.cuda.graph(graph, stream=side):
            got = step()
    for rnd in range(2):
        for i, xi in enumerate(xs):
            x.copy_(xi)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, ref[i])), (rnd, i)
            assert float(got[1].float().abs().sum()) > 0


def test_refusals_of_the_binding(fp4):
    (a, sa), (w, sw) = R.operand(4, 256, 1), R.operand(32, 256, 2)
    x = bf16(4, 256, 3)
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    for call in (lambda: fp4.int8_gemm(a, sa[:3], w, sw), lambda: fp4.int8_gemm(a.view(torch.uint8), sa, w, sw), lambda: fp4.int8_gemm(a.cpu(), sa, w, sw),
                 lambda: fp4.int8_gemm(a[:, :128].contiguous(), sa, w, sw), lambda: fp4.int8_gemm(a, sa, w, sw[:, None]), lambda: fp4.int8_gemm(a, sa.double(), w, sw),
                 lambda: fp4.int8_gemm(a, sa, w, sw, out=torch.empty(4, 32, device="cuda")), lambda: fp4.int8_quantize(x.float()), lambda: fp4.int8_quantize(x.t()),
                 lambda: fp4.int8_rmsnorm_quantize(x, x[0, :128]), lambda: fp4.int8_rmsnorm_quantize(x, x[0].contiguous(), residual=x[:3]),
                 lambda: fp4.int8_quantize(x.view(2, 2, 256).transpose(0, 1)), lambda: fp4.int8_grouped_gemm(a, sa, w, sw, off), lambda: fp4.int8_grouped_gemm(a, sa, w[None], sw[None], off.long()),
                 lambda: fp4.int8_grouped_gemm(a, sa, w[None], sw[None], off[:1].contiguous())):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: fp4.int8_quantize(x[:, :200]), lambda: fp4.int8_rmsnorm_quantize(x, x[0].contiguous(), -1.0), lambda: fp4.int8_quantize(x, flags=fp4.LAYOUT_GEMM),
                 lambda: fp4.int8_gemm(a, sa, w, sw, flags=1), lambda: fp4.int8_quantize(torch.empty(4, 260, dtype=torch.bfloat16, device="cuda")[:, 4:]),
                 lambda: fp4.int8_rmsnorm_quantize(x, x[0].contiguous(), residual_out=torch.empty_like(x))):
        with pytest.raises(fp4.Fp4mrError):
            call()


@pytest.mark.parametrize("K", [80, 528, 4112, 8208, 16400, 40000])
def test_rmsnorm_into_what_it_adds_with_rows_that_leave_threads_idle(fp4, K):
    """The sum may take the place of the residual or of x: with rows that are a little longer than a number of threads, idle ones read what others store."""
    rows = 2048
    x, r = bf16(rows, K, 1), bf16(rows, K, 2)
    w = bf16(1, K, 3)[0].contiguous()
    want = fp4.int8_rmsnorm_quantize(x, w, residual=r)
    for place in ("residual", "x"):
        xi, ri = x.clone(), r.clone()
        got = fp4.int8_rmsnorm_quantize(xi, w, residual=ri, residual_out=ri if place == "residual" else xi)
        assert all(torch.equal(g, t) for g, t in zip(got, want)), place


def test_rows_and_outputs_beyond_32_bits(fp4):
    """Elements of an output and of a quantizer's input past 2^32 and 2^31."""
    M, N, K = 70000, 65552, 128
    say("int8 gemm of 4.6e9 outputs")
    (a, sa), (w, sw) = R.operand(M, K, 1), R.operand(N, K, 2)
    out = fp4.int8_gemm(a, sa, w, sw)
    m, n = torch.tensor([0, 32767, 65535, 65536, M - 1], device="cuda"), torch.tensor([0, 255, 65535, N - 1], device="cuda")
    assert torch.equal(out[m][:, n].cpu(), R.product(a[m], sa[m], w[n], sw[n], torch.bfloat16))
    del out
    say("int8 quantize of 2.5e9 elements")
    x = torch.zeros(150000, 16400, dtype=torch.bfloat16, device="cuda")
    x[-2:] = bf16(2, 16400, 3)
    codes, scales = fp4.int8_quantize(x)
    c, s = fp4.int8_quantize(x[-2:].clone())
    assert torch.equal(codes[-2:], c) and torch.equal(scales[-2:], s) and (codes[:-2] == 0).all() and (scales[:-2] == float(np.float32(2.0 ** -100) / np.float32(127))).all()


@pytest.mark.parametrize("M,N,parts", [(64, 512, False), (160, 4096, True)])
def test_two_streams_at_once(fp4, M, N, parts):
    """Products, also in parts of K, each call with a workspace of its own, and quantizers, on two streams that wait for nothing of each other's."""
    sets = [(bf16(M, 14336, 40 + i).contiguous(), *R.operand(N, 14336, 50 + i, 0.01)) for i in range(2)]
    assert (fp4.int8_workspace_bytes(M, N, 14336) > 0) == parts
    want = [fp4.int8_gemm(*fp4.int8_quantize(x), w, sw) for x, w, sw in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                x, w, sw = sets[i]
                got[i].append(fp4.int8_gemm(*fp4.int8_quantize(x), w, sw))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i]) for i in range(2) for g in got[i])


def test_parts_of_k_in_a_graph(fp4):
    """The parts and the launch that joins them, recorded with a workspace of their own and replayed on other inputs, with eager work in the same form of room between the replays."""
    M, N, K = 160, 4096, 14336
    need = fp4.int8_workspace_bytes(M, N, K)
    assert need > 0
    xs = [bf16(M, K, 70 + i).contiguous() for i in range(3)]
    w, sw = R.operand(N, K, 80, 0.01)
    x, room = xs[0].clone(), torch.full((need,), 0x7f, dtype=torch.uint8, device="cuda")
    want = []
    for xi in xs:
        (c, s), pick = fp4.int8_quantize(xi), torch.tensor([0, 77, 159], device="cuda")
        want.append(fp4.int8_gemm(c, s, w, sw))
        assert torch.equal(want[-1][pick].cpu(), R.product(c[pick], s[pick], w, sw, torch.bfloat16))
    out = torch.zeros_like(want[0])
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            fp4.int8_gemm(*fp4.int8_quantize(x), w, sw, out=out, workspace=room)
    for rnd in range(3):
        for i, xi in enumerate(xs):
            x.copy_(xi)
            out.zero_()
            room.fill_(0x55 + i)
            assert torch.equal(fp4.int8_gemm(*fp4.int8_quantize(xi), w, sw), want[i])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[i]), (rnd, i)


def test_norm_of_a_prompt_repeats_itself_and_differs_from_64_bits_in_ties_alone(fp4):
    """The residual's addition and the norm of 4095 x 8192, with loud channels: the same bits every time, and the code of the 64-bit quotient but where that is the middle of two within the roundings' reach."""
    M, K = 4095, 8192
    x, r = bf16(M, K, 90, loud=False), bf16(M, K, 91)
    w = (1.0 + 0.2 * torch.randn(K, generator=torch.Generator().manual_seed(92))).to(torch.bfloat16).cuda()
    first = fp4.int8_rmsnorm_quantize(x, w, 1e-6, residual=r)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(fp4.int8_rmsnorm_quantize(x, w, 1e-6, residual=r), first))
    h = first[2].double()
    assert torch.equal(first[2], (x.float() + r.float()).to(torch.bfloat16))
    v = h / ((h * h).mean(1, keepdim=True) + 1e-6).sqrt() * w.double()
    t = v * (127.0 / v.abs().amax(1, keepdim=True))
    # The factor of the whole row is the same in v and in its largest: what is left are the two products of each, the reciprocal and the two products that make the code, seven roundings.
    assert ((first[0].double() - t).abs() <= 0.5 + t.abs() * 7 * U).all()
