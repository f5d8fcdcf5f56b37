"""Which kernels the 8-bit integer products launch, with how much LDS and into which bytes of their workspace, as the library's host code decides it
(the stand-in for HIP of test_dispatch; no GPU runs)."""
import json
import random
import shutil
import subprocess
import sys

import pytest

from tests.test_dispatch import HIP, LIB

LDS = 163840                     # bytes that a workgroup has
BF16, F32 = 0, 1 << 5

HOST = r"""
import ctypes, json, sys
hip = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
hip.fake_launches.restype = ctypes.c_char_p
P, I, Z, U = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_uint32
lib.int8_workspace_bytes.restype = Z
lib.int8_workspace_bytes.argtypes = [I, I, I]
lib.int8_gemm.argtypes = [P] * 4 + [I] * 3 + [P, P, Z, U, P]
lib.int8_grouped_gemm.argtypes = [P, P, I] + [P] * 4 + [I] * 4 + [P, U, P]
BUF, WS = 1 << 40, 1 << 41       # addresses that nothing reads
hip.fake_device(0, 256)
def launches(status):
    lines = hip.fake_launches().decode().split("\n")[:-1]
    return {"status": status, "launches": [{"kernel": f[0], "grid": int(f[1]), "lds": int(f[3]), "partial": int(f[4]), "parts": int(f[5])} for f in (l.split(" ") for l in lines)]}
for what, *a in json.load(sys.stdin):
    if what == "kernel": r = lib.fp4_set_option(4, a[0])
    elif what == "gemm":         # M, N, K, flags, bytes of workspace, or None: int8_workspace_bytes'
        M, N, K, flags, room = a
        if room is None: room = lib.int8_workspace_bytes(M, N, K)
        r = dict(launches(lib.int8_gemm(BUF, BUF, BUF, BUF, M, N, K, BUF, WS if room else None, room, flags, None)), room=room)
    else:                        # rows, experts, N, K, flags
        rows, E, N, K, flags = a
        r = launches(lib.int8_grouped_gemm(BUF, BUF, rows, BUF, BUF, BUF, None, rows, E, N, K, BUF, flags, None))
    print(json.dumps(r))
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    if not LIB.exists():
        from paper_2509_23202_amd import build
        build.build(verbose=False)
    d = tmp_path_factory.mktemp("int8_dispatch")
    # (the kernel that adds the parts: its second and third arguments)
    (d / "hip.c").write_text(HIP.replace('if (strstr(name, "splitk_reduce_kernel")) {', 'if (strstr(name, "int8_join_kernel")) { v[0] = *(long long*)args[1]; v[1] = *(int*)args[2]; } else if (strstr(name, "splitk_reduce_kernel")) {'))
    subprocess.run([cc, "-shared", "-fPIC", "-w", "-o", str(d / "hip.so"), str(d / "hip.c")], check=True)

    def ask(*requests):
        r = subprocess.run([sys.executable, "-c", HOST, str(d / "hip.so"), str(LIB)], input=json.dumps(requests), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        return [json.loads(l) for l in r.stdout.splitlines()]

    return ask


def held(run):
    """The call launched, and within the LDS that there is."""
    assert run["status"] == 0 and run["launches"]
    assert all(l["lds"] <= LDS and 0 < l["grid"] < 1 << 31 for l in run["launches"]), run
    return run["launches"]


def test_every_plan_is_held_by_lds_and_by_its_workspace(host):
    rng = random.Random(8)
    log = lambda low, high: int(round(low * (high / low) ** rng.random()))
    asks = []
    for _ in range(900):
        M, N, K = log(1, 1 << 14), log(1, 30000), 16 * log(1, 8191)
        asks.append((rng.choice([0, 0, 0] + list(range(1, 37))), M, N, K, rng.choice([BF16, F32]), rng.choice([None, 0, 1 << 44, log(16, 1 << 32) // 16 * 16])))
    runs = host(*(r for kernel, *a in asks for r in (["kernel", kernel], ["gemm", *a])))[1::2]
    split = 0
    for (kernel, M, N, K, flags, given), run in zip(asks, runs):
        first, *rest = held(run)
        if rest:                 # in parts: their tiles, and their sum
            (join,) = rest
            split += 1
            assert "int8_tile_kernel" in first["kernel"] and "int8_join_kernel" in join["kernel"] and join["parts"] >= 2
            assert join["partial"] == 1 << 41 and join["parts"] * M * N * 4 <= run["room"]
    assert split > 50


def test_every_plan_by_expert_is_held_by_lds(host):
    rng = random.Random(9)
    log = lambda low, high: int(round(low * (high / low) ** rng.random()))
    asks = [(rng.choice([0, 0] + list(range(1, 37))), log(1, 1 << 14), log(1, 256), log(1, 8192), 16 * log(1, 8191), rng.choice([BF16, F32])) for _ in range(300)]
    for run in host(*(r for kernel, *a in asks for r in (["kernel", kernel], ["grouped", *a])))[1::2]:
        assert len(held(run)) == 1


def test_the_largest_products_fit_a_launch(host):
    big = 1 << 24
    for M, N, K in ((big, 1, 16), (1, big, 16), (big, 1 << 14, 16), (1 << 14, big, 16), (big, 1 << 14, 131056)):
        for kernel in range(10):
            held(host(["kernel", kernel], ["gemm", M, N, K, BF16, 0])[1])


def test_the_room_that_the_library_asks_for_is_used(host):
    """A few tiles and a long K: parts; many tiles, few rows, or what is refused: no workspace."""
    run = host(["gemm", 160, 4096, 14336, BF16, None])[0]
    assert len(held(run)) == 2 and run["room"] == run["launches"][1]["parts"] * 160 * 4096 * 4
    for M, N, K in ((1, 4096, 4096), (4096, 4096, 4096), (4096, 28672, 4096)):
        run = host(["gemm", M, N, K, BF16, None])[0]
        assert run["room"] == 0 and len(held(run)) == 1
    assert len(held(host(["gemm", 160, 4096, 14336, BF16, 0])[0])) == 1
