"""The 8-bit operands by their definition in 64 bits, apart from the library's code: E4M3 values by searching the list of them, sums in
double precision on the host."""
import numpy as np
import torch

BLOCK, TOP, LEAST = 128, 448.0, 2.0 ** -100
U = 2.0 ** -24          # half a binary32 step, relative


def _values():
    v = [m * 2.0 ** -9 for m in range(8)]
    v += [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
    return np.array(v[:127])    # the 128th pattern is NaN


VALUES = _values()
MIDDLE = (VALUES[1:] + VALUES[:-1]) / 2


def e4m3(t):
    """The nearest E4M3 value of each number of t (float64 array), ties to the even code."""
    a = np.minimum(np.abs(t), TOP)
    i = np.searchsorted(MIDDLE, a, side="left")             # a tie is counted down
    tie = (i < len(MIDDLE)) & (a == MIDDLE[np.minimum(i, len(MIDDLE) - 1)])
    return np.sign(t) * VALUES[i + (tie & (i % 2 == 1))]


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64) if t.dtype != torch.float32 else t.detach().cpu().numpy().astype(np.float64)


def check_operand(codes, scales, v, delta, per_rows=1):
    """codes [rows, K], scales: those of v (float64 [rows, K]), whose values the library may know with the relative error `delta` (a number, or an array like v):
    the scale within that and a division's rounding, each code the nearest to some number within delta of its own value and delta of its
    block's scale, and two roundings (of the reciprocal and of the product)."""
    rows, K = v.shape
    delta = np.broadcast_to(np.asarray(delta, dtype=np.float64), v.shape)
    tall = -(-rows // per_rows)
    pad = ((0, tall * per_rows - rows), (0, 0))
    blocks = lambda a: np.pad(a, pad).reshape(tall, per_rows, K // BLOCK, BLOCK)
    amax = np.maximum(np.abs(blocks(v)).max((1, 3)), LEAST)
    d_block = blocks(delta).max((1, 3))
    s = f64(scales)
    assert s.shape == amax.shape
    np.testing.assert_array_less(np.abs(s - amax / TOP), (d_block + 2 * U) * amax / TOP + 1e-300)
    wide = lambda a: np.repeat(np.repeat(a, per_rows, 0)[:rows], BLOCK, 1)
    t = v * (TOP / wide(amax))
    off = np.abs(t) * (delta + wide(d_block) + 3 * U)
    got = f64(codes)
    lo, hi = e4m3(t - off), e4m3(t + off)
    assert np.isfinite(got).all()
    assert ((lo <= got) & (got <= hi)).all(), f"{((lo > got) | (got > hi)).sum()} of {got.size} codes"


def values(codes, scales, per_rows=1):
    """What an operand stands for, float64 [rows, K]."""
    c, s = f64(codes), f64(scales)
    return c * np.repeat(np.repeat(s, per_rows, 0)[: c.shape[0]], BLOCK, 1)


def check_product(out, a, w, K):
    """out [M,N] against a [M,K] times w [N,K] in float64.  A block's 128 products are exact and summed in at least binary32 (127 additions, each within U of
    the sum of magnitudes), scaled (2 roundings) and added to the others' (K / 128 fmas).  bf16 adds half a step, 2^-8 of the value at most, and its sums come from
    the 8-bit matrix instruction, which drops in every eight products what lies below 2^-13 of the largest one's power of two: 7 2^-13 of the sum of magnitudes."""
    y, size = a @ w.T, np.abs(a) @ np.abs(w).T
    got = f64(out)
    bound = size * U * (127 + 2 + K // BLOCK)
    if out.dtype == torch.bfloat16:
        bound += size * 7 * 2.0 ** -13 + 2.0 ** -8 * np.abs(y) * 1.01
    bad = ~(np.abs(got - y) <= bound + 1e-38)
    assert not bad.any(), f"{bad.sum()} of {bad.size} outputs, at most {np.nanmax(np.abs(got - y) / np.maximum(size, 1e-300)) / U:.1f} U of the sum of magnitudes"


def operand(rows, K, seed, per_rows=1, scale=1.0):
    """Codes (all finite patterns occur) and scales on the GPU; per_rows = 128: weights."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 127, (rows, K), generator=g, dtype=torch.uint8) | (torch.randint(0, 2, (rows, K), generator=g, dtype=torch.uint8) << 7)
    scales = (torch.rand(-(-rows // per_rows), K // BLOCK, generator=g) + 0.25) * scale
    return codes.view(torch.float8_e4m3fn).cuda(), scales.cuda()


def around(t, fill):
    """A copy of t with 4 KB of `fill` bytes in front of it and behind it."""
    n = t.numel() * t.element_size()
    room = torch.full((n + 8192,), fill, dtype=torch.uint8, device=t.device)
    room[4096: 4096 + n] = t.reshape(-1).view(torch.uint8)
    return room[4096: 4096 + n].view(t.dtype).view(t.shape)
