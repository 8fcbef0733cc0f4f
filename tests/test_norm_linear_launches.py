"""The launches of the layers in front of the LM head, on the CPU (norm_linear_trace.cpp): what the entry points accept can be launched, and every kernel that the library
holds is launched by some call."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2603_16435_amd import binding
from test_gpu_f8_tiles import TILES

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "norm_linear_trace.cpp")
pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH) or not shutil.which("g++"), reason="library not built, or no g++")
OK, SHAPE = 0, 2


@pytest.fixture(scope="module")
def trace(tmp_path_factory):
    """Calls to [(status, workspace bytes, [(workgroups, threads of each, kernel)])]."""
    exe = str(tmp_path_factory.mktemp("trace") / "norm_linear_trace")
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-o", exe, SOURCE, "-ldl"], check=True)

    def run(calls):
        r = subprocess.run([exe, binding.LIB_PATH, *(str(x) for c in calls for x in c)], capture_output=True, text=True, timeout=100)
        assert r.returncode == 0, r.stdout + r.stderr
        out, launches = [], []
        for line in r.stdout.splitlines():
            w = line.split()
            if w[0] == "status":
                out.append((int(w[1]), int(w[3]), launches))
                launches = []
            else:
                n = [int(v) for v in w[:6]]
                launches.append(((n[0], n[1], n[2]), (n[3], n[4], n[5]), w[6]))
        assert len(out) == sum(c[0] not in ("formats", "kernels") for c in calls)
        return out
    run.kernels = {line.split()[1] for line in subprocess.run([exe, binding.LIB_PATH, "kernels"], capture_output=True, text=True, timeout=100).stdout.splitlines()}
    return run


def _many():
    """Calls with as many rows, or columns, as the entry points may be asked for."""
    for M in (1 << 24, 1 << 27, (1 << 29) - 77, 1 << 29, (1 << 29) + 1, (1 << 30) - 300, (1 << 30) - 64, 1 << 30, (1 << 31) - (1 << 17)):
        for N in (1, 16, 30, 32, 33, 64, 100, 128, 256, 300, 5000, 1 << 22):
            for K in (1, 128, 700, 1700, 5000, 60_000, 1 << 22):
                for dtype in (0, 1):
                    yield "matmul", M, N, K, dtype
                    yield "forward", M, N, K, dtype, 1
    for M in (1, 20_000, 32_768, 100_000):
        for N in (1, 64, 5000, 1 << 22):
            for K in (1, 128, 60_000, 4_170_000, 1 << 22):
                for dtype in (0, 1):
                    yield "backward", M, N, K, dtype, 1, 1


def test_what_is_accepted_can_be_launched(trace):
    # a grid has less than 2^32 threads along each axis
    calls = list(_many())
    bad = [(c, l) for i in range(0, len(calls), 500) for c, (st, _, launches) in zip(calls[i:i + 500], trace(calls[i:i + 500])) for l in launches
           if any(g * b >= 1 << 32 for g, b in zip(l[0], l[1]))]
    assert not bad, (len(bad), bad[:5])


def test_what_fits_the_card_is_accepted(trace):
    # (288 GB of codes, scales, y and workspace)
    calls = [("matmul", 400_000_000, 32, 512, 1), ("matmul", 1_000_000_000, 1, 128, 1), ("forward", 200_000_000, 64, 256, 1, 1), ("forward", 16_000_000, 3584, 3584, 1, 1),
             ("backward", 16_000_000, 1024, 3584, 1, 1, 1), ("backward", 200_000, 100_000, 100_000, 1, 1, 1), ("forward", 1, 1 << 22, 1 << 14, 1, 0)]
    for c, (st, _, launches) in zip(calls, trace(calls)):
        assert st == OK and launches, c


def test_every_kernel_is_launched_by_some_call(trace):
    own = {k for k in trace.kernels if re.search(r"rlk\d+(ln|f8)_\w+kernel", k)}
    assert len(own) > 100
    sizes = [(M, N, K) for M in (1, 8, 16, 17, 64, 200, 700, 2000, 4096, 9000) for N in (16, 264, 1157, 4096) for K in (100, 600, 1163, 4096)]
    calls = []
    for fx in (0, 1):
        for fw in (0, 1):
            calls.append(("formats", fx, fw))
            for dtype in (0, 1):
                for M, N, K in sizes:
                    calls += [("matmul", M, N, K, dtype), ("forward", M, N, K, dtype, 1), ("backward", M, N, K, dtype, 1, 1)]
                calls += [("norm", R, H, dtype, kept) for R in (3, 600, 1500) for H in (64, 600, 1300, 2000, 3000, 6000, 9000) for kept in (0, 1)]
                calls += [("rows", 9, 300, dtype), ("weight", 300, 200, dtype), ("backward", 0, 40, 40, dtype, 1, 1)]
    launched = set()
    for i in range(0, len(calls), 300):                            # (the formats hold for a run of the program)
        f = [c for c in calls[:i + 1] if c[0] == "formats"][-1:]
        launched |= {l[2] for _, _, ls in trace(f + calls[i:i + 300]) for l in ls}
    assert own <= launched, sorted(own - launched)


def test_the_tests_of_the_tiles_reach_them(trace):
    got = trace([("matmul", M, N, K, 1 if dtype == "bf16" else 0) for _, _, dtype, M, N, K in TILES])
    for (tile, pieces, dtype, *size), (_, _, launches) in zip(TILES, got):
        kind = re.search(r"f8_gemm_kernelILi0ELi0E(f|DF16b)Li(\d+)ELi(\d+)", launches[0][2])
        assert kind and (kind[2] + "x" + kind[3], "cut" if len(launches) > 1 else "whole", "f32" if kind[1] == "f" else "bf16") == (tile, pieces, dtype), (tile, size)
    assert len({c[:3] for c in TILES}) == 15
