"""The launches of scoring with alternatives and of distillation, on the CPU (distill_trace.cpp): what the entry points accept can be launched, every kernel that the library holds for them is
launched by some call, and few rows take few launches."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2603_16435_amd import binding

SOURCE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "distill_trace.cpp")
pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH) or not shutil.which("g++"), reason="library not built, or no g++")


@pytest.fixture(scope="module")
def trace(tmp_path_factory):
    """Calls to [(status, workspace bytes, [(grid, block, kernel)])]."""
    exe = str(tmp_path_factory.mktemp("trace") / "distill_trace")
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-o", exe, SOURCE, "-ldl"], check=True)

    def run(calls):
        r = subprocess.run([exe, binding.LIB_PATH, *(str(x) for c in calls for x in c)], capture_output=True, text=True, timeout=200)
        assert r.returncode == 0, r.stdout[-2000:] + r.stderr
        out, launches = [], []
        for line in r.stdout.splitlines():
            w = line.split()
            if w[0] == "status":
                out.append((int(w[1]), int(w[3]), launches))
                launches = []
            else:
                n = [int(v) for v in w[:6]]
                launches.append((n[:3], n[3:], w[6]))
        assert len(out) == len(calls)
        return out
    run.kernels = {line.split()[1] for line in subprocess.run([exe, binding.LIB_PATH, "kernels"], capture_output=True, text=True, timeout=100).stdout.splitlines()}
    return run


def score(R, H, V, B=1, dtype=1, K=5, chunk=0, off=0):
    return "score", R, H, V, B, dtype, K, chunk, off


def distill(R, H, V, B=1, dtype=1, K=5, chunk=0, off=0, bwd=1, dw=0):
    return "distill", R, H, V, B, dtype, K, chunk, off, bwd, dw


def test_what_is_accepted_can_be_launched(trace):
    """A grid has less than 2^32 threads along each axis, whatever the rows, the chunk and the vocabulary are (of workspaces that a GPU could hold)."""
    calls = []
    for R in (1, 64, 4097, 1 << 20, (1 << 26) + 5, 1 << 28, (1 << 31) - (1 << 17)):
        for H, V in ((8, 8), (8, 524288), (5120, 256), (4096, 152064)):
            for dtype in (0, 1):
                for chunk in (0, 1 << 20) if R > 1 << 24 or V < 1000 else (0, 256):
                    if -(-R // (chunk or 16384)) > 20000:                    # (a chunk is a handful of launches)
                        continue
                    calls += [score(R, H, V, 3, dtype, min(V, 128), chunk), distill(R, H, V, 3, dtype, 128, chunk, dw=dtype)]
    checked = 0
    for i in range(0, len(calls), 20):
        for c, (st, ws, launches) in zip(calls[i:i + 20], trace(calls[i:i + 20])):
            assert st == 0, (c, st)
            if ws > 300 << 30:
                continue
            checked += 1
            for grid, block, name in launches:
                assert all(0 < g and g * b < 1 << 32 for g, b in zip(grid, block)), (c, grid, block, name)
    assert checked > 60


def test_every_kernel_is_launched(trace):
    calls = []
    for dtype in (0, 1):
        for off in (0, 4):
            for R in (1, 17, 33, 70, 300, 5000, 70000):
                for H in (64, 136, 200, 300, 600, 5120):
                    for V in (64, 3000, 20000, 50000, 140000, 400000):
                        calls.append(score(R, H, V, dtype=dtype, off=off))
                        for dw in {0, dtype}:
                            calls.append(distill(R, H, V, dtype=dtype, off=off, dw=dw))
    calls += [score(70, 2048, 90000), distill(100000, 2816, 152064, chunk=40000, dw=1), score(9, 5200, 16000, dtype=0), score(20, 5200, 16000, dtype=0)]
    calls += [distill(800000, 3584, 1000), score(800000, 3584, 1000), score(800000, 3592, 1000), distill(100000, 1344, 152064, chunk=40000), distill(100000, 1344, 152064, chunk=40000, dw=1),
              distill(50, 64, 300, bwd=0), distill(60, 64, 300, dtype=0), distill(128, 64, 300, dtype=0)]
    calls += [score(R, H, V, B=B, dtype=dtype) for R in (1, 17, 33, 70) for H in (64, 300, 5200) for V in (3000, 16000, 20000, 40000, 98000, 140000) for B in (1, 100) for dtype in (0, 1)]
    met = {name for i in range(0, len(calls), 200) for _, _, launches in trace(calls[i:i + 200]) for _, _, name in launches}
    mine = {k for k in trace.kernels if re.search("EpiScore|top_kernel|distill|few_grads|few_ds|few_dx|few_patch|EpiDWRounded", k)}
    assert len(mine) > 40 and mine <= met, sorted(mine - met)


def test_few_launches_for_few_rows(trace):
    (_, _, s), (_, _, d), (_, _, e), (_, _, n) = trace([score(1, 512, 3000), distill(30, 512, 3000, dw=1), distill(30, 512, 3000, bwd=0), distill(300, 512, 3000, dw=1)])
    assert [len(x) for x in (s, d, e, n)] == [2, 5, 3, 7]
    assert not any("transpose" in name for _, _, name in d + n)
