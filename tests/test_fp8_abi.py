"""The 8-bit entry points are declared, exported and bound, and refuse bad arguments before anything is launched (no GPU needed)."""
import re
from pathlib import Path

import pytest

HEADER = Path(__file__).resolve().parent.parent / "include" / "fp4mr.h"
NAMES = ("fp8_rmsnorm_quantize", "fp8_quantize", "fp8_quantize_weights", "fp8_gemm", "fp8_workspace_bytes", "fp8_grouped_gemm")


@pytest.fixture(scope="module")
def b():
    from paper_2509_23202_amd import binding
    return binding


def test_declared_exported_and_bound(b):
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    assert set(NAMES) == set(re.findall(r"\b(fp8_[a-z0-9_]+)\s*\(", text))
    for n in NAMES:
        assert hasattr(b.lib, n) and callable(getattr(b, n))
    assert b.SILU_MUL == 1 << int(re.search(r"FP4MR_SILU_MUL\s*=\s*1u\s*<<\s*(\d+)", HEADER.read_text()).group(1))


def test_arguments_are_checked_before_any_launch(b):
    L, fake = b.lib, 0x10000        # non-NULL, 16-byte aligned, never dereferenced: every call fails validation, or has nothing to do
    NULL, SHAPE, FMT, ALIGN = 1, 2, 4, 5

    def call(fn, names, base):
        def f(**kw):
            v = dict(base, **kw)
            assert set(v) == set(names)
            return fn(*(v[n] for n in names))
        return f

    norm = call(L.fp8_rmsnorm_quantize, ("x", "stride", "res", "w", "M", "K", "eps", "codes", "scales", "res_out", "norm", "flags", "st"),
                dict(x=fake, stride=256, res=None, w=fake, M=4, K=256, eps=1e-6, codes=fake, scales=fake, res_out=None, norm=None, flags=0, st=None))
    assert norm(x=None) == NULL and norm(w=None) == NULL and norm(codes=None) == NULL and norm(scales=None) == NULL
    assert norm(res=fake) == NULL and norm(res_out=fake) == NULL            # one without the other
    assert norm(K=192) == SHAPE and norm(K=0) == SHAPE and norm(M=-1) == SHAPE and norm(stride=248) == SHAPE and norm(stride=260) == SHAPE
    assert norm(K=65536 + 128, stride=1 << 20) == SHAPE and norm(M=(1 << 24) + 1) == SHAPE
    assert norm(eps=-1e-6) == SHAPE and norm(eps=float("nan")) == SHAPE
    assert norm(flags=1) == FMT and norm(flags=b.SILU_MUL) == FMT
    for n in ("x", "w", "codes", "norm"):
        assert norm(**{n: fake + 8}) == ALIGN, n
    assert norm(scales=fake + 2) == ALIGN
    assert norm(res=fake + 4, res_out=fake) == ALIGN and norm(res=fake, res_out=fake + 4) == ALIGN
    assert norm(M=0, x=None) == 0

    quant = call(L.fp8_quantize, ("x", "stride", "M", "K", "codes", "scales", "flags", "st"), dict(x=fake, stride=512, M=4, K=256, codes=fake, scales=fake, flags=0, st=None))
    assert quant(x=None) == NULL and quant(codes=None) == NULL and quant(scales=None) == NULL
    assert quant(K=64) == SHAPE and quant(stride=128) == SHAPE and quant(stride=504, flags=b.SILU_MUL) == SHAPE and quant(stride=516) == SHAPE and quant(M=-2) == SHAPE
    assert quant(flags=b.LAYOUT_GEMM) == FMT and quant(x=fake + 2) == ALIGN and quant(scales=fake + 1) == ALIGN and quant(M=0, codes=None) == 0

    weights = call(L.fp8_quantize_weights, ("w", "E", "N", "K", "codes", "scales", "flags", "st"), dict(w=fake, E=2, N=100, K=256, codes=fake, scales=fake, flags=0, st=None))
    assert weights(w=None) == NULL and weights(codes=None) == NULL and weights(E=0) == SHAPE and weights(N=0) == SHAPE and weights(K=130) == SHAPE
    assert weights(E=1 << 16, N=1 << 24, K=1 << 14) == SHAPE and weights(flags=1) == FMT and weights(codes=fake + 1) == ALIGN

    gemm = call(L.fp8_gemm, ("a", "sa", "w", "sw", "M", "N", "K", "out", "ws", "wsz", "flags", "st"),
                dict(a=fake, sa=fake, w=fake, sw=fake, M=4, N=16, K=128, out=fake, ws=None, wsz=0, flags=0, st=None))
    for n in ("a", "sa", "w", "sw", "out"):
        assert gemm(**{n: None}) == NULL and gemm(**{n: fake + (1 if n == "out" else 2)}) == ALIGN, n
    assert gemm(a=fake + 8) == ALIGN and gemm(w=fake + 4) == ALIGN and gemm(out=fake + 2, flags=b.OUT_F32) == ALIGN
    assert gemm(K=64) == SHAPE and gemm(N=0) == SHAPE and gemm(M=-1) == SHAPE and gemm(N=(1 << 24) + 1) == SHAPE
    assert gemm(K=(1 << 22) + 128) == SHAPE and gemm(M=1 << 24, N=(1 << 14) + 1) == SHAPE and gemm(ws=fake + 4, wsz=64) == ALIGN
    assert gemm(flags=b.A_LAYOUT_GEMM) == FMT and gemm(flags=1 << 20) == FMT and gemm(M=0) == 0

    grouped = call(L.fp8_grouped_gemm, ("a", "sa", "a_rows", "w", "sw", "off", "idx", "rows", "E", "N", "K", "out", "flags", "st"),
                   dict(a=fake, sa=fake, a_rows=4, w=fake, sw=fake, off=fake, idx=fake, rows=8, E=2, N=16, K=128, out=fake, flags=0, st=None))
    for n in ("a", "sa", "w", "sw", "out"):
        assert grouped(**{n: None}) == NULL and grouped(**{n: fake + (1 if n == "out" else 2)}) == ALIGN, n
    assert grouped(a=fake + 8) == ALIGN and grouped(w=fake + 4) == ALIGN
    assert grouped(off=None) == NULL and grouped(off=fake + 2) == ALIGN and grouped(idx=fake + 1) == ALIGN
    assert grouped(idx=None) == SHAPE                                       # without an index every row of A is a row of the output
    assert grouped(a_rows=0) == SHAPE and grouped(E=0) == SHAPE and grouped(E=(1 << 16) + 1) == SHAPE and grouped(rows=-1) == SHAPE and grouped(K=100) == SHAPE
    assert grouped(a_rows=1 << 20, K=4096) == SHAPE and grouped(E=1 << 16, N=1 << 16) == SHAPE      # gathered rows' offsets have 32 bits; weights beyond any memory
    assert grouped(flags=b.W_LAYOUT_GEMM) == FMT and grouped(rows=0, out=None) == 0


def test_workspace(b):
    """Whole fp32 copies of the output, where few tiles meet a long K; nothing for what is refused, has many tiles or few rows."""
    n = b.fp8_workspace_bytes(200, 4096, 14336)
    assert n > 0 and n % (200 * 4096 * 4) == 0 and 2 <= n // (200 * 4096 * 4) <= 16
    assert b.fp8_workspace_bytes(4096, 4096, 4096) == 0 and b.fp8_workspace_bytes(1, 4096, 4096) == 0 and b.fp8_workspace_bytes(0, 4096, 4096) == 0
    assert b.fp8_workspace_bytes(200, 4096, 100) == 0
    assert b.lib.fp4_set_option(b.OPT_FP8_VARIANT, 14) == 4 and b.lib.fp4_set_option(b.OPT_FP8_VARIANT, -1) == 4


def test_a_workspace_is_device_memory_of_its_own_size(b, monkeypatch):
    """A workspace in host memory, or of fewer bytes than its shape counts, is refused in front of the library, which would have the device write to it."""
    import torch

    class OnDevice(torch.Tensor):       # (host memory that says it is the device's: nothing is launched)
        is_cuda = True

    calls = []
    monkeypatch.setattr(b, "_stream", lambda: 0)
    monkeypatch.setattr(b.lib, "fp8_gemm", lambda *a: calls.append(a) or 0)
    M, N, K = 64, 256, 4096
    on = lambda *shape, dtype: torch.empty(shape, dtype=dtype).as_subclass(OnDevice)
    a, w = on(M, K, dtype=torch.float8_e4m3fn), on(N, K, dtype=torch.float8_e4m3fn)
    sa, sw, out = (on(*s, dtype=torch.float32) for s in ((M, K // 128), (N // 128, K // 128), (M, N)))
    room = lambda n: torch.empty(n, dtype=torch.uint8)
    for bad in (room(1 << 20), room(1).expand(1 << 20).as_subclass(OnDevice), room(1 << 20).as_subclass(OnDevice)[::2]):
        with pytest.raises(AssertionError):
            b.fp8_gemm(a, sa, w, sw, flags=b.OUT_F32, out=out, workspace=bad)
    assert not calls
    b.fp8_gemm(a, sa, w, sw, flags=b.OUT_F32, out=out, workspace=room(1 << 20).as_subclass(OnDevice))
    assert len(calls) == 1 and calls[0][9] == 1 << 20
