"""Which kernels the 8-bit products launch, with how much LDS and into which bytes of their workspace, as the library's host code decides it
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
TILE64, TILE128, TILE256 = "4TileILi2E", "4TileILi4E", "4TileILi8E"

HOST = r"""
import ctypes, json, sys
hip = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
hip.fake_launches.restype = ctypes.c_char_p
P, I, Z, U = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_uint32
lib.fp8_workspace_bytes.restype = Z
lib.fp8_workspace_bytes.argtypes = [I, I, I, U]
lib.fp8_gemm.argtypes = [P] * 4 + [I] * 3 + [P, P, Z, U, P]
lib.fp8_grouped_gemm.argtypes = [P, P, I] + [P] * 4 + [I] * 4 + [P, U, P]
BUF, WS = 1 << 40, 1 << 41       # addresses that nothing reads
hip.fake_device(0, 256)
def launches(status):
    lines = hip.fake_launches().decode().split("\n")[:-1]
    out = []
    for f in (l.split(" ") for l in lines):
        partial, parts, elements = (int(v) for v in f[4:7])      # of the kernel that adds the parts
        out.append({"kernel": f[0], "grid": int(f[1]), "lds": int(f[3]), "parts": parts, "sums": [partial - WS, parts * elements * 4]})
    return {"status": status, "launches": out}
for what, *a in json.load(sys.stdin):
    if what == "kernel": r = lib.fp4_set_option(3, a[0])
    elif what == "bytes": r = lib.fp8_workspace_bytes(*a)
    elif what == "gemm":         # M, N, K, flags, bytes of workspace, or None: fp8_workspace_bytes'
        M, N, K, flags, room = a
        if room is None: room = lib.fp8_workspace_bytes(M, N, K, flags)
        r = dict(launches(lib.fp8_gemm(BUF, BUF, BUF, BUF, M, N, K, BUF, WS if room else None, room, flags, None)), room=room)
    else:                        # rows, experts, N, K, flags
        rows, E, N, K, flags = a
        r = launches(lib.fp8_grouped_gemm(BUF, BUF, rows, BUF, BUF, BUF, None, rows, E, N, K, BUF, flags, None))
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
    d = tmp_path_factory.mktemp("fp8_dispatch")
    (d / "hip.c").write_text(HIP.replace('if (strstr(name, "splitk_reduce_kernel"))', 'if (strstr(name, "splitk_reduce_kernel") || strstr(name, "fp8_join_kernel"))'))
    subprocess.run([cc, "-shared", "-fPIC", "-w", "-o", str(d / "hip.so"), str(d / "hip.c")], check=True)

    def ask(*requests):
        r = subprocess.run([sys.executable, "-c", HOST, str(d / "hip.so"), str(LIB)], input=json.dumps(requests), capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        return [json.loads(l) for l in r.stdout.splitlines()]

    return ask


def held(run):
    """The call launched, and within the LDS that there is."""
    assert run["status"] == 0 and run["launches"]
    assert all(l["lds"] <= LDS for l in run["launches"]), run
    return run["launches"]


@pytest.mark.parametrize("M,N,K", [(1024, 2048, 262144), (91, 9600, 246784), (1024, 1024, 729088)])
@pytest.mark.parametrize("flags", [BF16, F32])
def test_long_k_in_parts_is_held_by_lds(host, M, N, K, flags):
    """A part's sums leave as fp32 whatever the product's output is, and leave its weights' scales the less room."""
    for run in host(["gemm", M, N, K, flags, None], ["gemm", M, N, K, flags, 1 << 40], ["gemm", M, N, K, flags, 0]):
        held(run)


def test_every_plan_is_held_by_lds_and_by_its_workspace(host):
    rng = random.Random(8)
    log = lambda low, high: int(round(low * (high / low) ** rng.random()))
    asks = []
    for _ in range(600):
        M, N, K = log(1, 4096), log(1, 20000), 128 * log(1, 1 << 15)
        asks.append((rng.choice([0, 0, 0] + list(range(1, 14))), M, N, K, rng.choice([BF16, F32]), rng.choice([None, 0, 1 << 44, log(16, 1 << 32) // 16 * 16])))
    runs = host(*(r for kernel, *a in asks for r in (["kernel", kernel], ["gemm", *a])))[1::2]
    for a, run in zip(asks, runs):
        first, *rest = held(run)
        if rest:                 # in parts: their tiles, and their sum
            (join,) = rest
            assert "fp8_tile_kernel" in first["kernel"] and "fp8_join_kernel" in join["kernel"] and join["parts"] >= 2
            assert join["sums"][0] == 0 and join["sums"][1] <= run["room"], a


def test_every_plan_by_expert_is_held_by_lds(host):
    rng = random.Random(9)
    log = lambda low, high: int(round(low * (high / low) ** rng.random()))
    asks = [(rng.choice(range(14)), log(1, 4096), log(1, 256), log(1, 8192), 128 * log(1, 1 << 15), rng.choice([BF16, F32])) for _ in range(300)]
    for run in host(*(r for kernel, *a in asks for r in (["kernel", kernel], ["grouped", *a])))[1::2]:
        assert len(held(run)) == 1


@pytest.mark.parametrize("kernel,tile,flags,most", [(5, TILE64, BF16, 6592), (5, TILE64, F32, 5568), (6, TILE128, BF16, 1984), (7, TILE256, BF16, 224)])
def test_a_tile_takes_k_up_to_the_room_for_scales(host, kernel, tile, flags, most):
    at, over = host(["kernel", kernel], *(["gemm", 33, 136, 128 * blocks, flags, 0] for blocks in (most, most + 1)))[1:]
    (at,), (over,) = held(at), held(over)
    assert tile in at["kernel"] and "fp8_stream" in over["kernel"]


@pytest.mark.parametrize("kernel,parts,tile,flags,most", [(8, 2, TILE64, BF16, 5568), (9, 4, TILE64, F32, 5568), (11, 2, TILE128, BF16, 960), (13, 8, TILE128, BF16, 960)])
def test_parts_take_k_up_to_the_room_for_scales(host, kernel, parts, tile, flags, most):
    """The last part is shorter than the others."""
    at, over = host(["kernel", kernel], *(["gemm", 33, 136, 128 * (parts * blocks - 3), flags, 1 << 40] for blocks in (most, most + 4)))[1:]
    at, over = held(at), held(over)
    assert tile in at[0]["kernel"] and "fp8_join" in at[1]["kernel"] and at[1]["parts"] == parts
    assert len(over) == 1 and "fp8_stream" in over[0]["kernel"]


@pytest.mark.parametrize("flags", [BF16, F32])
def test_forced_parts_are_the_ones_that_tests_on_the_device_name(host, flags):
    for kernel in range(8, 14):
        run = held(host(["kernel", kernel], ["gemm", 70, 300, 3840, flags, 8 * 70 * 300 * 4])[1])
        if flags == F32 and kernel > 10:       # (tiles of 128 rows have no fp32 output)
            assert len(run) == 1 and "fp8_stream" in run[0]["kernel"]
        else:
            assert (TILE64 if kernel <= 10 else TILE128) in run[0]["kernel"] and run[1]["parts"] == 2 << (kernel - 8) % 3
