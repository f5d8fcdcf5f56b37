"""The 8-bit integer operands and their products by their definition: whole numbers in 64 bits, which are exact, and binary32 steps where the definition has them."""
import numpy as np
import torch

from tests.fp8_util import U, around, f64  # noqa: F401

TOP, LEAST = 127.0, 2.0 ** -100


def check_rows(codes, scales, v, delta):
    """codes [rows, K], scales: those of v (float64 [rows, K]), whose values the library may know with the relative error `delta` (a number, or an array like v): the scale within
    that and a division's rounding, each code the nearest to some number within delta of its own value and delta of its row's abs-max, a reciprocal's rounding and two products'."""
    amax = np.maximum(np.abs(v).max(1), LEAST)
    delta = np.broadcast_to(np.asarray(delta, dtype=np.float64), v.shape)
    of_row = delta.max(1)
    s, got = f64(scales), codes.cpu().numpy().astype(np.float64)
    np.testing.assert_array_less(np.abs(s - amax / TOP), (of_row + 2 * U) * amax / TOP + 1e-300)
    t = v * (TOP / amax)[:, None]
    off = np.abs(t) * (delta + of_row[:, None] + 3 * U)
    assert ((np.rint(t - off) <= got) & (got <= np.rint(t + off))).all(), f"{((np.rint(t - off) > got) | (got > np.rint(t + off))).sum()} of {got.size} codes"
    assert np.abs(got).max() <= TOP


def quantized(x):
    """Codes and scales of bf16 rows as they are, every operation in binary32; and that the codes are those of the exact quotient, but where it is the middle of two."""
    v = f64(x)
    amax = np.maximum(np.abs(v).max(-1), LEAST).astype(np.float32)
    codes = np.rint(v.astype(np.float32) * (np.float32(TOP) * (np.float32(1.0) / amax))[..., None])
    exact = v * TOP / amax.astype(np.float64)[..., None]      # (fifteen bits over eight: binary64 rounds it off a middle by 2^-45 at most, and it is off one by 2^-18 or not at all)
    assert ((codes == np.rint(exact)) | (np.abs(exact) % 1.0 == 0.5)).all()
    return codes.astype(np.int8), np.float32(amax) / np.float32(TOP)


def operand(rows, K, seed, scale=1.0):
    """Codes (every one occurs, -128 too) and scales on the GPU."""
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-128, 128, (rows, K), generator=g, dtype=torch.int8).cuda(), ((torch.rand(rows, generator=g) + 0.25) * scale).cuda()


def product(a, sa, w, sw, dtype):
    """The product bit for bit: whole sums (binary64 holds them: K 2^14 < 2^53), rounded to binary32, times the one scale, times the other, in binary32, and to `dtype`."""
    sums = a.double().cpu() @ w.double().cpu().t()
    return (sums.float() * sa.cpu()[:, None] * sw.cpu()).to(dtype)
