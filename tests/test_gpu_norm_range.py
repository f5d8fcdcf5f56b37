"""The norms in front of the 8-bit layers on rows whose squares are beyond binary32, at either end: the row's own numbers are finite, and so is its norm."""
import numpy as np
import pytest
import torch

from tests import fp8_util, int8_util
from tests.test_gpu_int8 import bf16, fp4, say  # noqa: F401

pytestmark = pytest.mark.gpu
U = int8_util.U

# (every kernel: 64 to 1024 threads with up to eight pieces of eight columns, rows that end inside a piece of a thread)
COLUMNS = [16, 528, 1280, 2560, 4096, 8192, 8208, 16384, 32768, 40000, 65536]


def rows_of_all_sizes(K, seed):
    """Rows of normal values times powers of two from bf16's largest numbers to its subnormal ones, rows of one number at either end, and one with a single large number."""
    x = bf16(12, K, seed, loud=False).cpu().double().clamp(-3.9, 3.9)
    for i, e in enumerate((125, 100, 66, 62, 0, -49, -52, -63, -75, -100, -130)):
        x[i] *= 2.0 ** e
    x[11, 1:] *= 2.0 ** -20
    x[11, 0] = 2.0 ** 90
    ends = torch.empty(4, K, dtype=torch.float64)
    ends[0], ends[1], ends[2], ends[3] = torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).min, 2.0 ** -133, 2.0 ** -126
    ends[0, 1::2] = 0.0
    return torch.cat([x, ends]).to(torch.bfloat16).cuda()


def definition(h, w, eps):
    """float64: the squares have their room there (2^256 K)."""
    f = int8_util.f64(h)
    return f / np.sqrt((f * f).mean(1, keepdims=True) + float(np.float32(eps))) * int8_util.f64(w)


@pytest.mark.parametrize("K", COLUMNS)
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-30, 1e-6, 1e30])
def test_int8_rmsnorm_of_rows_whose_squares_are_beyond_binary32(fp4, K, eps):
    say(f"int8 rmsnorm K={K} eps={eps}")
    x = rows_of_all_sizes(K, K)
    w = (1.0 + 0.2 * torch.randn(K, generator=torch.Generator().manual_seed(9)).clamp(-3, 3)).to(torch.bfloat16).cuda()
    # As where the squares have room: at most 64 in a thread, 6 + 15 additions, half of that in the root, whose own steps, two products and the division add eight; half a step in eps.
    # A number times its row's power of two loses what is below 2^-149 of the row's largest number, and nothing else.
    delta = (0.5 * (64 + 21) + 9) * U
    for residual in (None, torch.zeros_like(x)):
        n = torch.empty_like(x)
        codes, scales, h = fp4.int8_rmsnorm_quantize(x, w, eps, residual=residual, norm_out=n)
        v = definition(x, w, eps)
        assert residual is None or torch.equal(h, x)
        int8_util.check_rows(codes, scales, v, delta)
        # (bf16's own subnormal numbers are 2^-133 apart)
        assert (np.abs(int8_util.f64(n) - v) <= np.abs(v) * (2.0 ** -8 + delta) + 2.0 ** -134).all()


def test_int8_rmsnorm_of_rows_that_are_not_finite_or_have_no_norm(fp4):
    """An infinity or NaN among large or small numbers, and a row of zeros with an eps of zero (0 / 0): scales that are not finite, and no other row's affair."""
    K = 1296
    x = rows_of_all_sizes(K, 3)
    w = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    good = fp4.int8_rmsnorm_quantize(x, w, 0.0)
    x[0, 5], x[9, 1290], x[4, 700], x[12] = float("inf"), float("nan"), -float("inf"), 0.0
    codes, scales, _ = fp4.int8_rmsnorm_quantize(x, w, 0.0)
    bad = torch.zeros(len(x), dtype=torch.bool, device="cuda")
    bad[[0, 9, 4, 12]] = True
    assert not torch.isfinite(scales[bad]).any()
    assert torch.equal(codes[~bad], good[0][~bad]) and torch.equal(scales[~bad], good[1][~bad])


@pytest.mark.parametrize("K", [128, 640, 1280, 2560, 4096, 8192, 8320, 16384, 32768, 40064, 65536])
@pytest.mark.parametrize("eps", [0.0, 1e-38, 1e-30, 1e-6, 1e30])
def test_fp8_rmsnorm_of_rows_whose_squares_are_beyond_binary32(fp4, K, eps):
    say(f"fp8 rmsnorm K={K} eps={eps}")
    x = rows_of_all_sizes(K, K)
    w = (1.0 + 0.2 * torch.randn(K, generator=torch.Generator().manual_seed(9)).clamp(-3, 3)).to(torch.bfloat16).cuda()
    delta = (0.5 * (64 + 21) + 9) * U        # as above
    for residual, rows in ((None, 1), (torch.zeros_like(x), 1), (None, 20)):       # (rows of 8192 columns have other threads in calls of many rows)
        h, n = x.repeat(rows, 1), torch.empty(rows * len(x), K, dtype=torch.bfloat16, device="cuda")
        codes, scales, out = fp4.fp8_rmsnorm_quantize(h, w, eps, residual=residual, norm_out=n)
        assert residual is None or torch.equal(out, x)
        v = definition(x, w, eps)
        fp8_util.check_operand(codes[-len(x):], scales[-len(x):], v, delta)
        assert (np.abs(fp8_util.f64(n[-len(x):]) - v) <= np.abs(v) * (2.0 ** -8 + delta) + 2.0 ** -134).all()


def test_fp8_rmsnorm_of_rows_that_are_not_finite_or_have_no_norm(fp4):
    K = 1280
    x = rows_of_all_sizes(K, 3)
    w = torch.ones(K, dtype=torch.bfloat16, device="cuda")
    good = fp4.fp8_rmsnorm_quantize(x, w, 0.0)
    x[0, 5], x[9, 1270], x[4, 700], x[12] = float("inf"), float("nan"), -float("inf"), 0.0
    codes, scales, _ = fp4.fp8_rmsnorm_quantize(x, w, 0.0)
    bad = torch.zeros(len(x), dtype=torch.bool, device="cuda")
    bad[[0, 9, 4, 12]] = True
    assert not torch.isfinite(scales[bad]).all(1).any()
    assert torch.equal(codes.view(torch.uint8)[~bad], good[0].view(torch.uint8)[~bad]) and torch.equal(scales[~bad], good[1][~bad])
