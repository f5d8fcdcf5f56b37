"""The entry points of the 8-bit integer layers and of the router are declared, exported and bound, and refuse bad arguments before anything is launched (no GPU needed)."""
import re
from pathlib import Path

import pytest

HEADER = Path(__file__).resolve().parent.parent / "include" / "fp4mr.h"
NAMES = ("int8_rmsnorm_quantize", "int8_quantize", "int8_gemm", "int8_workspace_bytes", "int8_grouped_gemm", "moe_route", "moe_workspace_bytes", "moe_combine")
NULL, SHAPE, FMT, ALIGN, WORKSPACE = 1, 2, 4, 5, 6
fake = 0x10000        # non-NULL, 16-byte aligned, never dereferenced: every call fails validation, or has nothing to do


@pytest.fixture(scope="module")
def b():
    from paper_2509_23202_amd import binding
    return binding


def call(fn, names, base):
    def f(**kw):
        v = dict(base, **kw)
        assert set(v) == set(names)
        return fn(*(v[n] for n in names))
    return f


def test_declared_exported_and_bound(b):
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    assert set(NAMES) == set(re.findall(r"\b((?:int8|moe)_[a-z0-9_]+)\s*\(", text))
    for n in NAMES:
        assert hasattr(b.lib, n) and callable(getattr(b, n))
    for n in ("ROUTE_SIGMOID", "ROUTE_RENORM", "ROUTE_GROUP_SUM2", "SHARED_F32"):
        assert getattr(b, n) == 1 << int(re.search(rf"FP4MR_{n}\s*=\s*1u\s*<<\s*(\d+)", HEADER.read_text()).group(1))
    assert b.INT8_MAX_K == int(re.search(r"#define FP4MR_INT8_MAX_K (\d+)", text).group(1)) and b.INT8_MAX_K << 14 < 1 << 31


def test_quantizers(b):
    norm = call(b.lib.int8_rmsnorm_quantize, ("x", "stride", "res", "w", "M", "K", "eps", "codes", "scales", "res_out", "norm", "flags", "st"),
                dict(x=fake, stride=256, res=None, w=fake, M=4, K=256, eps=1e-6, codes=fake, scales=fake, res_out=None, norm=None, flags=0, st=None))
    assert norm(x=None) == NULL and norm(w=None) == NULL and norm(codes=None) == NULL and norm(scales=None) == NULL
    assert norm(res=fake) == NULL and norm(res_out=fake) == NULL            # one without the other
    assert norm(K=200) == SHAPE and norm(K=0) == SHAPE and norm(K=-16) == SHAPE and norm(M=-1) == SHAPE and norm(stride=248) == SHAPE and norm(stride=260) == SHAPE
    assert norm(K=65536 + 16, stride=1 << 20) == SHAPE and norm(M=(1 << 24) + 1) == SHAPE
    assert norm(eps=-1e-6) == SHAPE and norm(eps=float("nan")) == SHAPE and norm(flags=b.SILU_MUL) == FMT
    for n in ("x", "w", "codes", "norm"):
        assert norm(**{n: fake + 8}) == ALIGN, n
    assert norm(scales=fake + 2) == ALIGN and norm(res=fake + 4, res_out=fake) == ALIGN and norm(res=fake, res_out=fake + 4) == ALIGN
    assert norm(M=0, x=None) == 0

    quant = call(b.lib.int8_quantize, ("x", "stride", "M", "K", "codes", "scales", "flags", "st"), dict(x=fake, stride=512, M=4, K=256, codes=fake, scales=fake, flags=0, st=None))
    assert quant(x=None) == NULL and quant(codes=None) == NULL and quant(scales=None) == NULL
    assert quant(K=72) == SHAPE and quant(stride=128) == SHAPE and quant(stride=504, flags=b.SILU_MUL) == SHAPE and quant(stride=516) == SHAPE and quant(M=-2) == SHAPE
    assert quant(K=b.INT8_MAX_K + 16, stride=1 << 20) == SHAPE and quant(M=(1 << 31) + 1) == SHAPE
    assert quant(flags=b.LAYOUT_GEMM) == FMT and quant(x=fake + 2) == ALIGN and quant(scales=fake + 1) == ALIGN and quant(M=0, codes=None) == 0


def test_products(b):
    gemm = call(b.lib.int8_gemm, ("a", "sa", "w", "sw", "M", "N", "K", "out", "ws", "wsz", "flags", "st"),
                dict(a=fake, sa=fake, w=fake, sw=fake, M=4, N=16, K=128, out=fake, ws=None, wsz=0, flags=0, st=None))
    for n in ("a", "sa", "w", "sw", "out"):
        assert gemm(**{n: None}) == NULL and gemm(**{n: fake + (1 if n == "out" else 2)}) == ALIGN, n
    assert gemm(a=fake + 8) == ALIGN and gemm(w=fake + 4) == ALIGN and gemm(out=fake + 2, flags=b.OUT_F32) == ALIGN and gemm(ws=fake + 4, wsz=64) == ALIGN
    assert gemm(K=72) == SHAPE and gemm(N=0) == SHAPE and gemm(M=-1) == SHAPE and gemm(N=(1 << 24) + 1) == SHAPE
    assert gemm(K=b.INT8_MAX_K + 16) == SHAPE and gemm(M=1 << 24, N=(1 << 14) + 1) == SHAPE
    assert gemm(flags=b.A_LAYOUT_GEMM) == FMT and gemm(flags=1 << 20) == FMT and gemm(M=0) == 0

    grouped = call(b.lib.int8_grouped_gemm, ("a", "sa", "a_rows", "w", "sw", "off", "idx", "rows", "E", "N", "K", "out", "flags", "st"),
                   dict(a=fake, sa=fake, a_rows=4, w=fake, sw=fake, off=fake, idx=fake, rows=8, E=2, N=16, K=128, out=fake, flags=0, st=None))
    for n in ("a", "sa", "w", "sw", "out"):
        assert grouped(**{n: None}) == NULL and grouped(**{n: fake + (1 if n == "out" else 2)}) == ALIGN, n
    assert grouped(a=fake + 8) == ALIGN and grouped(w=fake + 4) == ALIGN and grouped(off=None) == NULL and grouped(off=fake + 2) == ALIGN and grouped(idx=fake + 1) == ALIGN
    assert grouped(idx=None) == SHAPE                                       # without an index every row of A is a row of the output
    assert grouped(a_rows=0) == SHAPE and grouped(E=0) == SHAPE and grouped(E=(1 << 16) + 1) == SHAPE and grouped(rows=-1) == SHAPE and grouped(K=100) == SHAPE
    assert grouped(a_rows=1 << 20, K=4096) == SHAPE and grouped(E=1 << 16, N=1 << 16) == SHAPE      # gathered rows' offsets have 32 bits; weights beyond any memory
    assert grouped(flags=b.W_LAYOUT_GEMM) == FMT and grouped(rows=0, out=None) == 0


def test_router(b):
    route = call(b.lib.moe_route, ("z", "stride", "bias", "T", "E", "top", "groups", "top_groups", "scale", "w", "e", "rows", "off", "places", "ws", "wsz", "flags", "st"),
                 dict(z=fake, stride=64, bias=fake, T=4, E=64, top=4, groups=8, top_groups=2, scale=1.0, w=fake, e=fake, rows=fake, off=fake, places=fake, ws=fake, wsz=1 << 20, flags=0, st=None))
    for n in ("z", "w", "e", "rows", "off", "places"):
        assert route(**{n: None}) == NULL and route(**{n: fake + 1}) == ALIGN, n
    assert route(bias=fake + 2) == ALIGN and route(z=fake + 2, flags=b.INPUT_F32) == ALIGN and route(ws=fake + 4) == ALIGN
    assert route(T=100, ws=None) == WORKSPACE and route(T=100, wsz=b.moe_workspace_bytes(100, 64, 4) - 1) == WORKSPACE
    assert route(stride=63) == SHAPE and route(T=-1) == SHAPE and route(T=(1 << 24) + 1) == SHAPE and route(E=0) == SHAPE and route(E=1040, stride=2000) == SHAPE
    assert route(top=0) == SHAPE and route(top=17) == SHAPE and route(top=65, groups=1, top_groups=1) == SHAPE and route(groups=0) == SHAPE and route(groups=7) == SHAPE
    assert route(E=1000, stride=1000, groups=125) == SHAPE and route(top_groups=9) == SHAPE and route(top_groups=0) == SHAPE and route(T=1 << 24, top=65) == SHAPE
    assert route(flags=b.OUT_F32) == FMT and route(flags=1 << 20) == FMT and route(T=0, off=None) == NULL
    assert b.moe_workspace_bytes(0, 64, 4) == 0 and b.moe_workspace_bytes(100, 64, 4) > 0 and b.moe_workspace_bytes(100, 0, 4) == 0 and b.moe_workspace_bytes(-1, 64, 4) == 0

    combine = call(b.lib.moe_combine, ("y", "rows", "places", "w", "shared", "T", "top", "H", "out", "flags", "st"),
                   dict(y=fake, rows=8, places=fake, w=fake, shared=fake, T=4, top=2, H=64, out=fake, flags=0, st=None))
    for n in ("y", "places", "w", "out"):
        assert combine(**{n: None}) == NULL and combine(**{n: fake + 1}) == ALIGN, n
    assert combine(shared=fake + 1) == ALIGN and combine(shared=fake + 2, flags=b.SHARED_F32) == ALIGN and combine(y=fake + 2, flags=b.INPUT_F32) == ALIGN and combine(out=fake + 2, flags=b.OUT_F32) == ALIGN
    assert combine(H=0) == SHAPE and combine(H=(1 << 24) + 1) == SHAPE and combine(rows=-1) == SHAPE and combine(T=-1) == SHAPE and combine(top=0) == SHAPE and combine(top=65) == SHAPE
    assert combine(flags=b.SHARED_F32, shared=None) == FMT and combine(flags=b.SILU_MUL) == FMT and combine(T=0, out=None) == 0


def test_workspaces_are_device_memory_of_their_own_size(b, monkeypatch):
    """A workspace in host memory, or of fewer bytes than its shape counts, is refused in front of the library, which would have the device write to it."""
    import torch

    class OnDevice(torch.Tensor):       # (host memory that says it is the device's: nothing is launched)
        is_cuda = True
        device = torch.device("cuda", 0)

    calls = []
    monkeypatch.setattr(b, "_stream", lambda: 0)
    monkeypatch.setattr(b, "_current_device", lambda: 0)
    monkeypatch.setattr(b, "_calls", None)
    monkeypatch.setattr(b, "_new", lambda like, shape, dtype: torch.empty(shape, dtype=dtype).as_subclass(OnDevice))
    on = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype).as_subclass(OnDevice)
    room = lambda n: torch.empty(n, dtype=torch.uint8)
    bad = (room(1 << 20), room(1).expand(1 << 20).as_subclass(OnDevice), room(1 << 20).as_subclass(OnDevice)[::2])
    for name, run in (("int8_gemm", lambda w: b.int8_gemm(on(64, 4096, dtype=torch.int8), on(64), on(256, 4096, dtype=torch.int8), on(256), workspace=w)),
                      ("moe_route", lambda w: b.moe_route(on(100, 32), 2, workspace=w))):
        monkeypatch.setattr(b.lib, name, lambda *a: calls.append(a) or 0)
        for w in bad:
            with pytest.raises(AssertionError):
                run(w)
        assert not calls
        run(room(1 << 20).as_subclass(OnDevice))
        assert len(calls) == 1 and 1 << 20 in calls.pop()


def test_flags_that_name_a_type_have_to_be_the_tensors(b, monkeypatch):
    """A flag that says that bf16 tensors are fp32 would have the device read twice what they hold: refused in front of the library, also by the compiled calls, which hand such calls on."""
    import torch

    class OnDevice(torch.Tensor):       # (host memory that says it is the device's: nothing is launched)
        is_cuda = True
        device = torch.device("cuda", 0)

    calls = []
    monkeypatch.setattr(b, "_stream", lambda: 0)
    monkeypatch.setattr(b, "_current_device", lambda: 0)
    monkeypatch.setattr(b, "_calls", None)
    monkeypatch.setattr(b, "_new", lambda like, shape, dtype: torch.empty(shape, dtype=dtype).as_subclass(OnDevice))
    on = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype).as_subclass(OnDevice)
    for name in ("moe_route", "moe_combine"):
        monkeypatch.setattr(b.lib, name, lambda *a: calls.append(a) or 0)
    half, places = torch.bfloat16, on(4, 2, dtype=torch.int32)
    for run in (lambda: b.moe_route(on(4, 32, dtype=half), 2, flags=b.INPUT_F32), lambda: b.moe_combine(on(8, 32, dtype=half), places, on(4, 2), flags=b.INPUT_F32),
                lambda: b.moe_combine(on(8, 32, dtype=half), places, on(4, 2), shared=on(4, 32, dtype=half), flags=b.SHARED_F32),
                lambda: b.moe_combine(on(8, 32, dtype=half), places, on(4, 2), flags=b.SHARED_F32)):
        with pytest.raises(AssertionError):
            run()
    assert not calls
    b.moe_route(on(4, 32), 2, flags=b.INPUT_F32)
    b.moe_combine(on(8, 32), places, on(4, 2), shared=on(4, 32), flags=b.INPUT_F32 | b.SHARED_F32)
    assert len(calls) == 2


def test_tensors_of_another_device_are_refused(b, monkeypatch):
    """Kernels run on the current device: tensors of another one are refused in front of the library."""
    import torch

    class OnDevice(torch.Tensor):       # (host memory that says it is a device's: nothing is launched)
        is_cuda = True
        device = torch.device("cuda", 1)

    calls = []
    monkeypatch.setattr(b, "_stream", lambda: 0)
    monkeypatch.setattr(b, "_current_device", lambda: 0)
    monkeypatch.setattr(b, "_calls", None)
    monkeypatch.setattr(b, "_new", lambda like, shape, dtype: torch.empty(shape, dtype=dtype).as_subclass(OnDevice))
    on = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype).as_subclass(OnDevice)
    i8, i32, half = torch.int8, torch.int32, torch.bfloat16
    runs = {"int8_quantize": lambda: b.int8_quantize(on(4, 32, dtype=half)), "int8_rmsnorm_quantize": lambda: b.int8_rmsnorm_quantize(on(4, 32, dtype=half), on(32, dtype=half)),
            "int8_gemm": lambda: b.int8_gemm(on(4, 32, dtype=i8), on(4), on(8, 32, dtype=i8), on(8)),
            "int8_grouped_gemm": lambda: b.int8_grouped_gemm(on(4, 32, dtype=i8), on(4), on(2, 8, 32, dtype=i8), on(2, 8), on(3, dtype=i32)),
            "moe_route": lambda: b.moe_route(on(4, 32), 2), "moe_combine": lambda: b.moe_combine(on(8, 32), on(4, 2, dtype=i32), on(4, 2))}
    for name, run in runs.items():
        monkeypatch.setattr(b.lib, name, lambda *a: calls.append(a) or 0)
        with pytest.raises(AssertionError):
            run()
        assert not calls, name
    OnDevice.device = torch.device("cuda", 0)
    for run in runs.values():
        run()
    assert len(calls) == 6
