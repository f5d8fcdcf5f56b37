"""The 8-bit linear layers against their definition in 64 bits (tests/fp8_util.py)."""
import sys

import numpy as np
import pytest
import torch

from tests import fp8_util as R

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
@pytest.mark.parametrize("rows,K,apart", [(1, 128, 0), (3, 384, 8), (33, 4096, 0), (130, 640, 24), (7, 14336, 0), (1, 16512, 8), (2100, 256, 0)])
@pytest.mark.parametrize("silu", [False, True])
def test_quantize(fp4, rows, K, apart, silu):
    say(f"quantize {rows}x{K} apart={apart} silu={silu}")
    x = bf16(rows, 2 * K if silu else K, rows + K, apart)
    codes, scales = fp4.fp8_quantize(x, flags=fp4.SILU_MUL if silu else 0)
    v, delta = R.f64(x), 0.0
    if silu:
        g, u = v[:, :K], v[:, K:]
        with np.errstate(over="ignore"):
            v = g / (1 + np.exp(-g)) * u
        # the exponential's argument is rounded in its product with log2 e (|g| / ln 2 steps of the exponent), the instruction, the sum, the reciprocal
        # and two products each within a step
        delta = (1.5 * np.minimum(np.abs(g), 128.0) + 8) * 2 * U
    R.check_operand(codes, scales, v, delta)


def test_quantize_rounds_every_bf16_to_the_nearest_code(fp4):
    """Blocks whose abs-max is 448: the reciprocal is 1, and every value's code is the nearest E4M3 value exactly."""
    bits = np.arange(0, 0x43e0 + 1, dtype=np.uint16)      # 0 .. 448
    v = np.concatenate([bits, bits | 0x8000])
    v = np.pad(v, (0, -len(v) % 127))
    rows = np.concatenate([v.reshape(-1, 127), np.full((len(v) // 127, 1), 0x43e0, np.uint16)], 1)
    x = torch.from_numpy(rows.view(np.int16)).cuda().view(torch.bfloat16)
    codes, scales = fp4.fp8_quantize(x)
    assert (scales == 1.0).all()
    np.testing.assert_array_equal(R.f64(codes), R.e4m3(R.f64(x)))
    negative_zero = (x.view(torch.int16) < 0).cpu() & (x.cpu() == 0)
    assert (codes.view(torch.uint8).cpu()[negative_zero] == 0x80).all()


def test_quantize_of_zeros_and_of_the_smallest_and_largest_numbers(fp4):
    x = torch.zeros(6, 256, dtype=torch.bfloat16, device="cuda")
    x[1, :128] = 1e-38
    x[2, 5] = -3.3e38
    x[2, 6] = 1e38
    x[3, 7] = 2.0 ** -100
    x[3, 8] = -2.0 ** -102
    x[4, 130] = 2.0 ** -133      # the smallest subnormal
    x[5] = 7.0
    codes, scales = fp4.fp8_quantize(x)
    R.check_operand(codes, scales, R.f64(x), 0.0)
    assert (codes.view(torch.uint8)[0] == 0).all() and (scales[0] == 2.0 ** -100 / 448).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_number_that_is_not_finite_stays_in_its_block(fp4, bad):
    x = bf16(5, 384, 3)
    x[2, 200] = bad
    codes, scales = fp4.fp8_quantize(x)
    good = torch.ones(5, 3, dtype=torch.bool)
    good[2, 1] = False
    assert torch.isfinite(scales.cpu())[good].all() and not torch.isfinite(scales[2, 1])
    assert not torch.isfinite(R_values(codes, scales)[2, 128:256]).any()
    y = x.clone()
    y[2, 128:256] = 0
    codes2, scales2 = fp4.fp8_quantize(y)
    keep = good.repeat_interleave(128, 1).cuda()
    assert torch.equal(codes.view(torch.uint8)[keep], codes2.view(torch.uint8)[keep])
    w, ws = R.operand(48, 384, 4, 128)
    out = fp4.fp8_gemm(codes, scales, w, ws)
    assert not torch.isfinite(out[2]).any() and torch.isfinite(out[[0, 1, 3, 4]]).all()


def R_values(codes, scales):
    return codes.float() * scales.repeat_interleave(128, 1)


@pytest.mark.parametrize("rows,K,apart", [(1, 128, 0), (5, 512, 8), (3, 640, 0), (4, 2048, 0), (2, 2176, 16), (1, 4096, 0), (300, 4096, 0), (3, 8192, 8), (2, 8320, 0), (2, 16384, 0),
                                          (1, 16512, 0), (2, 65536, 0)])
@pytest.mark.parametrize("residual,norm", [(False, False), (True, False), (True, True)])
def test_rmsnorm_quantize(fp4, rows, K, apart, residual, norm):
    say(f"rmsnorm {rows}x{K} apart={apart} residual={residual} norm={norm}")
    x, r = bf16(rows, K, 7 + K, apart, loud=False), bf16(rows, K, 8 + K) if residual else None
    w = (1.0 + 0.3 * torch.randn(K, generator=torch.Generator().manual_seed(9))).to(torch.bfloat16).cuda()
    n = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda") if norm else None
    codes, scales, h = fp4.fp8_rmsnorm_quantize(x, w, 1e-5, residual=r, norm_out=n)
    if residual:
        assert torch.equal(h, (x.float() + r.float()).to(torch.bfloat16))
    else:
        assert h is None
    f = R.f64(h if residual else x)
    v = f / np.sqrt((f * f).mean(1, keepdims=True) + 1e-5) * R.f64(w)
    # sum of squares: at most 64 values in a thread, then 6 + 15 additions; half of that in the root, whose own steps, two products and the division by K add eight
    delta = (0.5 * (64 + 21) + 8) * U
    R.check_operand(codes, scales, v, delta)
    if norm:
        assert (np.abs(R.f64(n) - v) <= np.abs(v) * (2.0 ** -8 + delta)).all()


def test_rmsnorm_in_place_and_of_a_row_of_zeros(fp4):
    K = 1280
    x, r = bf16(9, K, 1), bf16(9, K, 2)
    x[4] = 0
    r[4] = 0
    w = torch.full((K,), 0.5, dtype=torch.bfloat16, device="cuda")
    ref = fp4.fp8_rmsnorm_quantize(x, w, 1e-6, residual=r)
    for target in ("residual", "x"):
        xx, rr = x.clone(), r.clone()
        out = fp4.fp8_rmsnorm_quantize(xx, w, 1e-6, residual=rr, residual_out=rr if target == "residual" else xx)
        assert torch.equal(out[0].view(torch.uint8), ref[0].view(torch.uint8)) and torch.equal(out[1], ref[1]) and torch.equal(out[2], ref[2])
    assert (ref[0].view(torch.uint8)[4] == 0).all() and torch.isfinite(ref[1]).all()


def test_rmsnorm_of_more_rows_than_a_launch_has(fp4):
    K, first = 128, 1 << 21
    rows = first + 600
    torch.manual_seed(5)
    x, r = (torch.randn(rows, K, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.randn(K, device="cuda").to(torch.bfloat16)
    norm = torch.empty_like(x)
    got = fp4.fp8_rmsnorm_quantize(x, w, 1e-5, residual=r, norm_out=norm) + (norm,)
    for part in (slice(0, first), slice(first, rows)):       # (the same kernel: the same bits)
        n = torch.empty_like(x[part])
        want = fp4.fp8_rmsnorm_quantize(x[part], w, 1e-5, residual=r[part], norm_out=n) + (n,)
        for g, e in zip(got, want):
            assert torch.equal(g[part].view(torch.uint8), e.view(torch.uint8))


@pytest.mark.parametrize("shape", [(1, 128), (127, 256), (128, 128), (129, 384), (300, 1152), (1, 1, 128), (3, 200, 256), (5, 129, 128)])
def test_quantize_weights(fp4, shape):
    say(f"weights {shape}")
    K = shape[-1]
    w = bf16(int(np.prod(shape[:-1])), K, 5 + K).contiguous().view(shape)
    codes, scales = fp4.fp8_quantize_weights(w)
    for e in range(shape[0] if len(shape) == 3 else 1):
        at = (lambda t: t[e]) if len(shape) == 3 else (lambda t: t)
        R.check_operand(at(codes), at(scales), R.f64(at(w)), 0.0, per_rows=128)


# ---------------------------------------------------------------- products
SHAPES = [(1, 16, 128), (1, 4096, 4096), (2, 1, 256), (3, 129, 384), (15, 200, 640), (16, 1000, 2048), (17, 136, 1152), (33, 72, 14336), (64, 256, 512), (65, 257, 896), (100, 520, 256),
          (128, 128, 128), (129, 640, 384), (200, 1001, 1024), (256, 512, 2048), (257, 264, 640), (300, 96, 4096), (512, 768, 256), (700, 1288, 384), (1030, 200, 128)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("f32", [False, True])
def test_gemm(fp4, M, N, K, f32):
    """Codes of every finite pattern; bytes beside the operands, and their scales' neighbours, are NaN and reach no output."""
    say(f"fp8_gemm M={M} N={N} K={K} f32={f32}")
    (a, sa), (w, sw) = R.operand(M, K, M + K), R.operand(N, K, N + K, 128, 0.01)
    ops = [R.around(t, 0x7f if t.dtype != torch.float32 else 0xff) for t in (a, sa, w, sw)]
    flags = fp4.OUT_F32 if f32 else 0
    room = torch.full((M * N * (4 if f32 else 2) + 8192,), 0x5a, dtype=torch.uint8, device="cuda")
    out = room[4096: -4096].view(torch.float32 if f32 else torch.bfloat16).view(M, N)
    fp4.fp8_gemm(*ops, flags=flags, out=out)
    R.check_product(out, R.values(a, sa), R.values(w, sw, 128), K)
    assert (room[:4096] == 0x5a).all() and (room[-4096:] == 0x5a).all()
    assert torch.equal(out, fp4.fp8_gemm(a, sa, w, sw, flags=flags))      # the same bits every time


@pytest.mark.parametrize("M,N,K", [(1, 48, 256), (5, 256, 1024), (48, 130, 640), (100, 300, 384), (260, 520, 512)])
def test_gemm_of_integers_is_exact(fp4, M, N, K):
    """Small integers and scales that are powers of two: every sum is exact, whatever its order."""
    g = torch.Generator().manual_seed(M)
    a = torch.randint(-8, 9, (M, K), generator=g).float()
    w = torch.randint(-4, 5, (N, K), generator=g).float()
    sa = 2.0 ** torch.randint(-3, 3, (M, K // 128), generator=g)
    sw = 2.0 ** torch.randint(-2, 2, (-(-N // 128), K // 128), generator=g)
    out = fp4.fp8_gemm(a.to(torch.float8_e4m3fn).cuda(), sa.cuda(), w.to(torch.float8_e4m3fn).cuda(), sw.cuda(), flags=fp4.OUT_F32)
    A = a.double() * sa.double().repeat_interleave(128, 1)
    W = w.double() * sw.double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)
    assert torch.equal(out.cpu().double(), A @ W.T)


def grouped(fp4, counts, N, K, seed, gather=None, f32=False):
    """Rows of the given numbers per expert; gather: rows of A to draw from.  Checked expert by expert."""
    E, T = len(counts), sum(counts)
    a_rows = gather or T
    a, sa = R.operand(max(a_rows, 1), K, seed)
    a, sa = a[:a_rows], sa[:a_rows]
    pairs = [R.operand(N, K, seed + 1 + e, 128, 0.01) for e in range(E)]
    w, sw = torch.stack([p[0].view(torch.uint8) for p in pairs]).view(torch.float8_e4m3fn), torch.stack([p[1] for p in pairs])
    begin = np.concatenate([[0], np.cumsum(counts)])
    offsets = torch.tensor(begin, dtype=torch.int32, device="cuda")
    index = torch.randint(0, a_rows, (T,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda() if gather else None
    ops = [R.around(t, 0x7f if t.dtype != torch.float32 else 0xff) for t in (a, sa, w, sw)]
    out = fp4.fp8_grouped_gemm(*ops, offsets, rows=index, flags=fp4.OUT_F32 if f32 else 0)
    assert tuple(out.shape) == (T, N)
    A = R.values(a, sa)
    if gather:
        A = A[index.cpu().numpy()]
    for e in range(E):
        if counts[e]:
            R.check_product(out[begin[e]: begin[e + 1]], A[begin[e]: begin[e + 1]], R.values(*pairs[e], 128), K)
    assert torch.equal(out, fp4.fp8_grouped_gemm(a, sa, w, sw, offsets, rows=index, flags=fp4.OUT_F32 if f32 else 0))


@pytest.mark.parametrize("counts,N,K", [([1], 16, 128), ([5, 0, 1], 48, 256), ([0, 0, 7], 129, 384), ([3, 0, 0], 200, 128), ([1] * 40, 72, 640), ([16, 17, 0, 15, 33], 264, 512),
                                        ([0] * 70 + [2] + [0] * 60 + [9], 40, 256), ([64, 0, 65, 63], 136, 1152), ([200, 1, 0, 90], 300, 384), ([300, 257, 0, 128], 520, 256),
                                        ([129] * 9, 1001, 256), ([700, 0, 3], 256, 128)])
@pytest.mark.parametrize("gather", [None, 23])
def test_grouped_gemm(fp4, counts, N, K, gather):
    say(f"grouped {len(counts)} experts, {sum(counts)} rows, N={N} K={K} gather={gather}")
    grouped(fp4, counts, N, K, len(counts) + N, gather, f32=N % 16 == 0)


@pytest.mark.parametrize("T,counts", [(40, [3, 0, 9]), (300, [100, 130, 20])])
def test_grouped_rows_of_no_expert_and_indexes_outside(fp4, T, counts):
    """Rows behind the last offset keep what they held; an index outside A is a row of zeros, whatever A's rows hold."""
    K, N, E = 384, 200, 3
    a, sa = R.operand(10, K, 1)
    a.view(torch.uint8)[0] = 0x7f
    a.view(torch.uint8)[9] = 0x7f
    w, sw = R.operand(E * 256, K, 2, 128, 0.01)
    w, sw = w.view(torch.uint8).view(E, 256, K)[:, :N].contiguous().view(torch.float8_e4m3fn), sw.view(E, 2, K // 128)
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")
    index = (torch.arange(T, dtype=torch.int32) % 8 + 1).cuda()
    outside = {1: -1, 4: 10, 10: 2 ** 31 - 1, 11: -2 ** 31}
    for t, i in outside.items():
        index[t] = i
    out = torch.full((T, N), 7.0, dtype=torch.bfloat16, device="cuda")
    fp4.fp8_grouped_gemm(a, sa, w, sw, offsets, rows=index, out=out)
    used = sum(counts)
    assert (out[used:] == 7.0).all()
    assert (out[list(outside)] == 0).all()
    A, begin = R.values(a, sa), offsets.tolist()
    for e in range(E):
        rows = [t for t in range(begin[e], begin[e + 1]) if t not in outside]
        if rows:
            R.check_product(out[rows], A[index[rows].cpu().numpy()], R.values(w[e], sw[e], 128), K)


KERNELS = list(range(1, 8))      # few rows (1 to 4), tiles of 64, 128 and 256 rows


@pytest.fixture
def forced(fp4):
    """Every product on one kernel, whatever the library would choose."""
    yield lambda kernel: fp4.set_option(fp4.OPT_FP8_VARIANT, kernel)
    fp4.set_option(fp4.OPT_FP8_VARIANT, 0)


@pytest.mark.parametrize("kernel", KERNELS + list(range(8, 14)))
@pytest.mark.parametrize("M,N,K", [(1, 16, 128), (5, 129, 512), (33, 136, 640), (70, 300, 1152), (260, 520, 2176), (2100, 1100, 640)])
def test_gemm_on_every_kernel(fp4, forced, kernel, M, N, K):
    """Each kernel on sizes that it would not be chosen for too; 8 to 13: two, four and eight parts of K."""
    say(f"kernel {kernel} M={M} N={N} K={K}")
    forced(kernel)
    (a, sa), (w, sw) = R.operand(M, K, M), R.operand(N, K, N, 128, 0.01)
    ops = [R.around(t, 0x7f if t.dtype != torch.float32 else 0xff) for t in (a, sa, w, sw)]
    room = torch.full((16 * M * N * 4,), 0xff, dtype=torch.uint8, device="cuda")
    out = fp4.fp8_gemm(*ops, workspace=room)
    R.check_product(out, R.values(a, sa), R.values(w, sw, 128), K)
    assert torch.equal(out, fp4.fp8_gemm(a, sa, w, sw, workspace=room))


@pytest.mark.parametrize("kernel", KERNELS + [9, 12])
@pytest.mark.parametrize("f32", [False, True])
def test_scales_and_outputs_at_any_element(fp4, forced, kernel, f32):
    """A part of a tensor of scales, or of an output with an odd number of columns, begins where it begins."""
    forced(kernel)
    M, N, K = 40, 131, 640
    (a, sa), (w, sw) = R.operand(M, K, 1), R.operand(N, K, 2, 128, 0.01)
    shifted = lambda t, by: torch.cat([torch.full((by,), float("nan"), device="cuda"), t.reshape(-1)])[by:].view(t.shape)
    whole = torch.full((M + 2, N), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    flags, room = fp4.OUT_F32 if f32 else 0, torch.empty(8 * M * N * 4, dtype=torch.uint8, device="cuda")
    fp4.fp8_gemm(a, shifted(sa, 1), w, shifted(sw, 3), flags=flags, out=whole[1: M + 1], workspace=room)
    R.check_product(whole[1: M + 1], R.values(a, sa), R.values(w, sw, 128), K)
    assert (whole[[0, M + 1]] == 7.0).all()
    whole.fill_(7.0)
    fp4.fp8_grouped_gemm(a, shifted(sa, 2), w[None], shifted(sw, 1)[None], torch.tensor([9, 0, M], dtype=torch.int32, device="cuda")[1:], flags=flags, out=whole[1: M + 1])
    R.check_product(whole[1: M + 1], R.values(a, sa), R.values(w, sw, 128), K)
    assert (whole[[0, M + 1]] == 7.0).all()


@pytest.mark.parametrize("kernel", [6, 7])
def test_a_workgroup_walks_several_tiles(fp4, forced, kernel):
    """More tiles than compute units, of whole and partial rows and columns, and a K that is not a multiple of four blocks."""
    forced(kernel)
    M, N, K = 4200, 4440, 896
    (a, sa), (w, sw) = R.operand(M, K, 1), R.operand(N, K, 2, 128, 0.01)
    out = fp4.fp8_gemm(a, sa, w, sw)
    rows = np.r_[0:70, 250:260, 2040:2100, 4090:4200]
    R.check_product(out[rows], R.values(a, sa)[rows], R.values(w, sw, 128), K)
    cols = np.r_[0:20, 250:260, 4090:4110, 4430:4440]
    R.check_product(out[:, cols].contiguous(), R.values(a, sa), R.values(w, sw, 128)[cols], K)


@pytest.mark.parametrize("kernel", KERNELS)
def test_grouped_on_every_kernel(fp4, forced, kernel):
    """Experts of many sizes, empty ones among them, more tiles than compute units for the smaller tiles; rows in order, and gathered."""
    forced(kernel)
    counts = [700, 0, 3, 129, 0, 1100, 64, 257, 1, 400]
    for gather in (None, 333):
        say(f"grouped kernel {kernel} gather={gather}")
        grouped(fp4, counts, 1100, 640, kernel, gather)


@pytest.mark.parametrize("kernel", KERNELS)
def test_grouped_of_many_experts_on_every_kernel(fp4, forced, kernel):
    """Tiles that are found behind the first 64 experts, and behind the first 128."""
    forced(kernel)
    counts = [0] * 30 + [3, 70] + [0] * 31 + [5] + [0] * 10 + [1, 0, 40] + [0] * 60 + [2, 0, 33, 0]
    grouped(fp4, counts, 72, 512, kernel)


@pytest.mark.parametrize("f32", [False, True])
def test_a_k_that_only_the_few_row_kernels_take(fp4, f32):
    M, N, K = 200, 40, 262144
    (a, sa), (w, sw) = R.operand(M, K, 5), R.operand(N, K, 6, 128, 0.01)
    out = fp4.fp8_gemm(a, sa, w, sw, flags=fp4.OUT_F32 if f32 else 0)
    R.check_product(out, R.values(a, sa), R.values(w, sw, 128), K)


def test_grouped_offsets_are_kept_within_the_rows(fp4):
    """Offsets below 0 and beyond the rows count as 0 and as the number of rows."""
    K, N, T = 256, 80, 50
    a, sa = R.operand(T, K, 5)
    pairs = [R.operand(N, K, 6 + e, 128) for e in range(3)]
    w, sw = torch.stack([p[0].view(torch.uint8) for p in pairs]).view(torch.float8_e4m3fn), torch.stack([p[1] for p in pairs])
    out = fp4.fp8_grouped_gemm(a, sa, w, sw, torch.tensor([-5, 20, 30, 1000], dtype=torch.int32, device="cuda"))
    ref = fp4.fp8_grouped_gemm(a, sa, w, sw, torch.tensor([0, 20, 30, 50], dtype=torch.int32, device="cuda"))
    assert torch.equal(out, ref)


@pytest.mark.parametrize("offsets", [[30, 10, 40, 5], [0, 50, 50, 20], [0, 0, 0, 0], [-2 ** 31, 2 ** 31 - 1, 0, 50]])
def test_grouped_offsets_that_decrease_stay_within_the_rows(fp4, offsets):
    """Not what the call is for, but nothing beside the output's rows is written, and rows that one expert alone has are its products."""
    K, N, T = 640, 200, 50
    a, sa = R.operand(T, K, 5)
    w, sw = R.operand(3 * 256, K, 2, 128, 0.01)
    w, sw = w.view(torch.uint8).view(3, 256, K)[:, :N].contiguous().view(torch.float8_e4m3fn), sw.view(3, 2, K // 128)
    room = torch.full((T * N * 2 + 65536,), 0x5a, dtype=torch.uint8, device="cuda")
    out = room[32768: -32768].view(torch.bfloat16).view(T, N)
    fp4.fp8_grouped_gemm(a, sa, w, sw, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=out)
    torch.cuda.synchronize()
    assert (room[:32768] == 0x5a).all() and (room[-32768:] == 0x5a).all()


def test_no_rows(fp4):
    w, sw = R.operand(32, 256, 1, 128)
    a, sa = torch.empty(0, 256, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(0, 2, device="cuda")
    x = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    assert fp4.fp8_gemm(a, sa, w, sw).shape == (0, 32)
    assert fp4.fp8_grouped_gemm(a, sa, w[None], sw[None], torch.zeros(2, dtype=torch.int32, device="cuda")).shape == (0, 32)
    assert fp4.fp8_quantize(x)[0].shape == (0, 256)
    assert fp4.fp8_rmsnorm_quantize(x, torch.ones(256, dtype=torch.bfloat16, device="cuda"), residual=x)[2].shape == (0, 256)


def test_weights_of_more_than_4_gb(fp4, forced):
    """The last expert's weights begin beyond 2^32 bytes, and a single expert's rows too.  On one kernel the same bits with that expert alone (left to itself the library may
    take another for one expert than for eighteen, with its sums in another order)."""
    K, N, E = 16384, 16384, 18
    say("grouped with 4.8 GB of weights")
    w = torch.zeros(E, N, K, dtype=torch.uint8, device="cuda")
    (last, s_last), (a, sa) = R.operand(N, K, 3, 128, 0.01), R.operand(20, K, 4)
    w[E - 1] = last.view(torch.uint8)
    sw = torch.zeros(E, N // 128, K // 128, device="cuda")
    sw[E - 1] = s_last
    offsets = torch.tensor([0] * E + [20], dtype=torch.int32, device="cuda")
    for kernel in KERNELS:
        forced(kernel)
        out = fp4.fp8_grouped_gemm(a, sa, w.view(torch.float8_e4m3fn), sw, offsets)
        assert torch.equal(out, fp4.fp8_grouped_gemm(a, sa, last[None], s_last[None], offsets[-2:].contiguous()))
    forced(0)
    out = fp4.fp8_grouped_gemm(a, sa, w.view(torch.float8_e4m3fn), sw, offsets)
    pick = torch.tensor([0, 1, 8191, 16383], device="cuda")
    R.check_product(out[:, pick], R.values(a, sa), R.values(last.view(torch.uint8)[pick].view(torch.float8_e4m3fn), s_last.repeat_interleave(128, 0)[pick], 1), K)
    flat = fp4.fp8_gemm(a, sa, w.view(torch.float8_e4m3fn).view(E * N, K), sw.view(-1, K // 128))
    R.check_product(flat[:, pick + (E - 1) * N], R.values(a, sa), R.values(last.view(torch.uint8)[pick].view(torch.float8_e4m3fn), s_last.repeat_interleave(128, 0)[pick], 1), K)
    assert (flat[:, :-N] == 0).all()


def test_streams_and_graphs(fp4):
    """The path on a stream of its own, then recorded and replayed on other inputs, eager work between the replays."""
    K, N, E, T = 512, 384, 4, 24
    w, sw = fp4.fp8_quantize_weights(bf16(E * N, K, 1).contiguous().view(E, N, K))
    ones = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    offsets = torch.tensor([0, 7, 7, 20, T], dtype=torch.int32, device="cuda")
    index = (torch.arange(T, dtype=torch.int32) * 5 % 12).cuda()
    xs = [bf16(12, K, 20 + i) for i in range(3)]
    x, res = xs[0].clone(), bf16(12, K, 30)

    def step():
        c, s, h = fp4.fp8_rmsnorm_quantize(x, ones, residual=res)
        y = fp4.fp8_grouped_gemm(c, s, w, sw, offsets, rows=index)
        c2, s2 = fp4.fp8_quantize(y[:, :256], flags=fp4.SILU_MUL)
        return h, y, fp4.fp8_gemm(c2, s2, w[0, :, :128].contiguous(), sw[0, :, :1].contiguous())

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


def test_modes_see_the_outputs_made_and_new_memory_is_filled_where_asked_for(fp4):
    from torch.utils._python_dispatch import TorchDispatchMode

    class Seen(TorchDispatchMode):
        def __init__(self):
            super().__init__()
            self.empties = 0

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            self.empties += "empty" in str(func)
            return func(*args, **(kwargs or {}))

    x, w = bf16(3, 256, 21, loud=False), bf16(130, 256, 22, loud=False)
    plain = fp4.fp8_quantize(x) + fp4.fp8_quantize_weights(w)
    with Seen() as seen:
        watched = fp4.fp8_quantize(x) + fp4.fp8_quantize_weights(w)
    assert seen.empties >= 4
    for a, b in zip(plain, watched):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))

    was = torch.are_deterministic_algorithms_enabled()
    torch.use_deterministic_algorithms(True)
    try:      # (row 2 is nobody's)
        y = fp4.fp8_grouped_gemm(*plain[:2], plain[2][None], plain[3][None], torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    finally:
        torch.use_deterministic_algorithms(was)
    assert torch.isnan(y[2]).all() and torch.isfinite(y[:2]).all()


def test_refusals_of_the_binding(fp4):
    (a, sa), (w, sw) = R.operand(4, 256, 1), R.operand(32, 256, 2, 128)
    x = bf16(4, 256, 3)
    off = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    for call in (lambda: fp4.fp8_gemm(a, sa[:, :1].contiguous(), w, sw), lambda: fp4.fp8_gemm(a.view(torch.uint8), sa, w, sw), lambda: fp4.fp8_gemm(a.cpu(), sa, w, sw),
                 lambda: fp4.fp8_gemm(a[:, :128].contiguous(), sa[:, :1].contiguous(), w, sw), lambda: fp4.fp8_gemm(a, sa, w, sw.t()),
                 lambda: fp4.fp8_gemm(a, sa, w, sw, out=torch.empty(4, 32, device="cuda")), lambda: fp4.fp8_quantize(x.float()), lambda: fp4.fp8_quantize(x.t()),
                 lambda: fp4.fp8_rmsnorm_quantize(x, x[0, :128]), lambda: fp4.fp8_rmsnorm_quantize(x, x[0].contiguous(), residual=x[:3]),
                 lambda: fp4.fp8_quantize_weights(x.t()), lambda: fp4.fp8_grouped_gemm(a, sa, w, sw, off), lambda: fp4.fp8_grouped_gemm(a, sa, w[None], sw[None], off.long()),
                 lambda: fp4.fp8_grouped_gemm(a, sa, w[None], sw[None], off[:1].contiguous())):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: fp4.fp8_quantize(x[:, :192]), lambda: fp4.fp8_rmsnorm_quantize(x, x[0].contiguous(), -1.0), lambda: fp4.fp8_quantize(x, flags=fp4.LAYOUT_GEMM),
                 lambda: fp4.fp8_gemm(a, sa, w, sw, flags=1), lambda: fp4.fp8_quantize(torch.empty(4, 260, dtype=torch.bfloat16, device="cuda")[:, 4:]),
                 lambda: fp4.fp8_rmsnorm_quantize(x, x[0].contiguous(), residual_out=torch.empty_like(x))):
        with pytest.raises((fp4.Fp4mrError, AssertionError)):
            call()


def ternary(M, N, K, seed):
    """Operands of -1, 0 and 1 with scales of 1 and 2, whose products' sums are whole numbers below 2^24 in any order (K < 2^22), and that product."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for rows, per in ((M, 1), (N, 128)):
        v = torch.randint(-1, 2, (rows, K), generator=g, device="cuda", dtype=torch.int8)
        s = 1.0 + torch.randint(0, 2, (-(-rows // per), K // 128), generator=g, device="cuda").float()
        out += [v.to(torch.float8_e4m3fn), s, v.double() * s.repeat_interleave(per, 0)[:rows].repeat_interleave(128, 1).double()]
    a, sa, A, w, sw, W = out
    return (a, sa, w, sw), A @ W.t()


@pytest.mark.parametrize("kernel,parts,blocks,f32", [(7, 1, 224, False), (7, 1, 225, False), (6, 1, 1984, False), (6, 1, 1985, False), (5, 1, 6592, False), (5, 1, 6593, False), (5, 1, 5568, True),
                                                     (5, 1, 5569, True), (11, 2, 960, False), (11, 2, 964, False), (13, 8, 960, False), (13, 8, 964, False), (8, 2, 5568, False), (8, 2, 5572, False),
                                                     (8, 2, 5568, True), (8, 2, 5572, True)])
def test_products_at_the_room_for_scales(fp4, forced, kernel, parts, blocks, f32):
    """The longest K, and the longest part of K, whose weights' scales fit beside a tile's stages, and the next one, which runs on another kernel: exact."""
    M, N, K = 17, 136, 128 * (blocks if parts == 1 else parts * blocks - 3)
    say(f"kernel {kernel} K={K} in {parts} parts of {blocks} blocks, f32={f32}")
    forced(kernel)
    ops, y = ternary(M, N, K, blocks)
    room = torch.full((16 * M * N * 4,), 0xff, dtype=torch.uint8, device="cuda") if parts > 1 else None
    out = fp4.fp8_gemm(*ops, flags=fp4.OUT_F32 if f32 else 0, workspace=room)
    assert torch.equal(out, y.to(out.dtype))


@pytest.mark.parametrize("f32", [False, True])
def test_a_k_that_no_tile_takes_without_a_workspace(fp4, f32):
    M, N, K = 40, 72, 128 * 6600
    ops, y = ternary(M, N, K, 1)
    out = torch.empty(M, N, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    status = fp4.lib.fp8_gemm(*(t.data_ptr() for t in ops), M, N, K, out.data_ptr(), None, 0, fp4.OUT_F32 if f32 else 0, torch.cuda.current_stream().cuda_stream)
    assert status == 0 and torch.equal(out, y.to(out.dtype))


def test_a_long_k_in_the_parts_that_the_library_asks_for(fp4):
    """1024 x 2048 x 262144 with the workspace of fp8_workspace_bytes: parts of 1024 blocks would leave the scales no room on tiles of 128 rows."""
    M, N, K = 1024, 2048, 262144
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    rnd = lambda rows: torch.randint(-1, 2, (rows, K), generator=g, device="cuda", dtype=torch.int8).to(torch.float8_e4m3fn)
    a, w = rnd(M), rnd(N)
    sa, sw = torch.ones(M, K // 128, device="cuda"), torch.ones(N // 128, K // 128, device="cuda")
    sa[:, 1::3] = 2.0
    out = fp4.fp8_gemm(a, sa, w, sw)
    rows, cols = torch.arange(3, M, 31, device="cuda"), torch.arange(5, N, 61, device="cuda")
    u8 = lambda t, i: t.view(torch.uint8)[i].view(torch.float8_e4m3fn).double()
    y = (u8(a, rows) * sa[rows].repeat_interleave(128, 1).double()) @ u8(w, cols).t()
    assert torch.equal(out[rows][:, cols], y.to(torch.bfloat16))


def experts_that_are_not_finite(E, N, K):
    """Weights of E >= 2 experts: of the first a code in row 5 is NaN, of the second the scale of its rows 128 to 255 and one block of K is infinite."""
    w, sw = R.operand(E * -(-N // 128) * 128, K, 2, 128, 0.01)
    w, sw = w.view(torch.uint8).view(E, -1, K)[:, :N].contiguous(), sw.view(E, -1, K // 128).clone()
    w[0, 5, 200] = 0x7f
    sw[1, 1, 3] = float("inf")
    return w.view(torch.float8_e4m3fn), sw


@pytest.mark.parametrize("kernel,f32", [(k, False) for k in KERNELS] + [(k, True) for k in KERNELS[:5]])     # (tiles of 128 and 256 rows have no fp32 output)
def test_an_index_outside_is_a_row_of_zeros_on_every_kernel(fp4, forced, kernel, f32):
    """Zero codes with a scale of zero: 0, and NaN beside weights that hold a NaN or an infinite scale, whatever the rows of A hold."""
    forced(kernel)
    K, N, counts = 640, 300, [90, 150]
    T = sum(counts)
    a, sa = R.operand(10, K, 1)
    sa[0] = float("nan")
    a.view(torch.uint8)[9] = 0x7f
    w, sw = experts_that_are_not_finite(2, N, K)
    index = torch.full((T,), 4, dtype=torch.int32)
    outside = [0, 1, 17, 63, 64, 89, 90, 91, 130, 200, 239]
    index[outside] = torch.tensor([-1, 10, 2 ** 31 - 1, -2 ** 31, 11, -7, 10, -1, 4096, -1, 10], dtype=torch.int32)
    out = fp4.fp8_grouped_gemm(a, sa, w, sw, torch.tensor([0, 90, T], dtype=torch.int32, device="cuda"), rows=index.cuda(), flags=fp4.OUT_F32 if f32 else 0).float().cpu()
    row = torch.zeros(2, N)
    row[0, 5] = float("nan")
    row[1, 128:256] = float("nan")
    for t in outside:
        assert torch.equal(out[t].nan_to_num(7.0), row[int(t >= 90)].nan_to_num(7.0)), t
    inside = [t for t in range(T) if t not in outside]
    for t in inside:
        assert torch.equal(torch.isfinite(out[t]), torch.isfinite(row[int(t >= 90)]))


@pytest.mark.parametrize("kernel", KERNELS + list(range(8, 14)))
@pytest.mark.parametrize("f32", [False, True])
def test_numbers_that_are_not_finite_stay_in_their_rows_and_columns(fp4, forced, kernel, f32):
    """On every kernel and in every number of parts, of a K that is not a multiple of four blocks, the last of which are multiplied again with scales of zero: a code that is NaN, a scale that
    is NaN or infinite, of either operand, in the first, the last and other blocks.  (Those kernels that have no fp32 output leave it to another.)"""
    forced(kernel)
    M, N, K = 70, 300, 128 * 30
    (a, sa), (w, sw) = R.operand(M, K, 1), R.operand(N, K, 2, 128, 0.01)
    A, W = R.values(a, sa), R.values(w, sw, 128)
    a.view(torch.uint8)[3, K - 100] = 0x7f
    a.view(torch.uint8)[64, 0] = 0xff
    sa[40, 2], sa[41, 29] = float("inf"), float("nan")
    w.view(torch.uint8)[7, 5] = 0xff
    w.view(torch.uint8)[100, K - 1] = 0x7f
    sw[1, 28], sw[2, 0] = float("inf"), float("nan")
    out = fp4.fp8_gemm(a, sa, w, sw, flags=fp4.OUT_F32 if f32 else 0, workspace=torch.full((8 * M * N * 4,), 0xff, dtype=torch.uint8, device="cuda"))
    rows, cols = [m for m in range(M) if m not in (3, 40, 41, 64)], [n for n in range(128) if n not in (7, 100)]
    good = torch.zeros(M, N, dtype=torch.bool)
    good[np.ix_(rows, cols)] = True
    assert torch.equal(torch.isfinite(out).cpu(), good)
    R.check_product(out[rows][:, cols], A[rows], W[cols], K)


@pytest.mark.parametrize("kernel", KERNELS)
def test_numbers_that_are_not_finite_stay_with_their_expert(fp4, forced, kernel):
    forced(kernel)
    K, N, counts = 128 * 6, 300, [90, 150, 40]
    T, begin = sum(counts), np.concatenate([[0], np.cumsum(counts)])
    a, sa = R.operand(T, K, 3)
    w, sw = experts_that_are_not_finite(3, N, K)
    A = R.values(a, sa)
    sa[89, 5] = float("inf")            # (the last row of the first expert)
    a.view(torch.uint8)[240, 0] = 0x7f  # (the first one of the third)
    out = fp4.fp8_grouped_gemm(a, sa, w, sw, torch.tensor(begin, dtype=torch.int32, device="cuda"))
    good = torch.ones(T, N, dtype=torch.bool)
    good[[89, 240]] = False
    good[:90, 5] = False
    good[90:240, 128:256] = False
    assert torch.equal(torch.isfinite(out).cpu(), good)
    for e in range(3):
        rows = [t for t in range(begin[e], begin[e + 1]) if t not in (89, 240)]
        cols = [n for n in range(N) if not (e == 0 and n == 5 or e == 1 and 128 <= n < 256)]
        R.check_product(out[rows][:, cols], A[rows], R.values(w[e], torch.nan_to_num(sw[e], posinf=0.0), 128)[cols], K)


def test_a_workgroup_walks_several_tiles_of_an_fp32_output(fp4, forced):
    """More tiles of 64 x 128 than compute units, of whole and partial rows and columns, seven blocks of K; and as many by expert."""
    forced(5)
    M, N, K = 4200, 4440, 896
    (a, sa), (w, sw) = R.operand(M, K, 1), R.operand(N, K, 2, 128, 0.01)
    out = fp4.fp8_gemm(a, sa, w, sw, flags=fp4.OUT_F32)
    rows = np.r_[0:70, 250:260, 2040:2100, 4090:4200]
    R.check_product(out[rows], R.values(a, sa)[rows], R.values(w, sw, 128), K)
    cols = np.r_[0:20, 120:132, 250:260, 4090:4110, 4430:4440]
    R.check_product(out[:, cols].contiguous(), R.values(a, sa), R.values(w, sw, 128)[cols], K)
    for gather in (None, 333):
        grouped(fp4, [700, 0, 3, 129, 0, 1100, 64, 257, 1, 400], 1100, 640, 5, gather, f32=True)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("offsets,expert,first,end", [([30, 10, 40, 5], 1, 10, 40), ([0, 50, 50, 20], 0, 0, 50), ([0, 0, 0, 0], 0, 0, 0)])
def test_rows_of_one_expert_where_offsets_decrease(fp4, forced, kernel, offsets, expert, first, end):
    """An expert whose offsets decrease has no rows; with the others' apart and no more tiles than the rows have, theirs are their products and the rest stays as it was."""
    forced(kernel)
    K, N, T = 640, 200, 50
    a, sa = R.operand(T, K, 5)
    w, sw = R.operand(3 * 256, K, 2, 128, 0.01)
    w, sw = w.view(torch.uint8).view(3, 256, K)[:, :N].contiguous().view(torch.float8_e4m3fn), sw.view(3, 2, K // 128)
    room = torch.full((T * N * 2 + 65536,), 0x5a, dtype=torch.uint8, device="cuda")
    out = room[32768: -32768].view(torch.bfloat16).view(T, N)
    fp4.fp8_grouped_gemm(a, sa, w, sw, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=out)
    if end > first:
        R.check_product(out[first:end], R.values(a, sa)[first:end], R.values(w[expert], sw[expert], 128), K)
        out[first:end].view(torch.uint8).fill_(0x5a)
    assert (room == 0x5a).all()


def test_gates_far_below_zero(fp4):
    """silu(g) as far down as binary32 has e^-g and its reciprocal, in the products that a large `up` makes of it; 0 beyond; the type's lowest value too."""
    g = torch.cat([-torch.linspace(60, 87, 128), -torch.linspace(89, 200, 126), torch.tensor([-3.3e38, -1e4])]).to(torch.bfloat16)
    g = torch.where(g < -88.5, g, g.clamp(min=-87.0))
    x = torch.cat([g, torch.full((256,), 1e30).to(torch.bfloat16)])[None].cuda()
    codes, scales = fp4.fp8_quantize(x, flags=fp4.SILU_MUL)
    v = R.f64(x[:, :256])
    v, delta = v / (1 + np.exp(-np.maximum(v, -600.0))) * R.f64(x[:, 256:]), (1.5 * np.minimum(np.abs(v), 128.0) + 8) * 2 * U
    R.check_operand(codes[:, :128], scales[:, :1], v[:, :128], delta[:, :128])
    assert (codes.float()[:, 128:] == 0).all() and (scales[:, 1] == 2.0 ** -100 / 448).all()
    x[0, 3] = -float("inf")
    assert torch.isnan(fp4.fp8_quantize(x, flags=fp4.SILU_MUL)[1][0, 0])
