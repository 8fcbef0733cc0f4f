"""Every tile of the 8-bit product with every pair of formats and both output types, whole and cut along K, against the float64 product of the restored operands.

f32 outputs: whole numbers, whose sums are exact in any order.  bf16 outputs: single products, of seven significant bits at most.  Both: ordinary values within the tolerance of
test_gpu_norm_linear.py."""
import numpy as np
import pytest
import torch

import test_gpu_norm_linear as base
from paper_2603_16435_amd import binding

# tile, pieces along K, output type, M, N, K   (test_norm_linear_launches.py looks that the sizes reach them)
TILES = [("32x32", "whole", "f32", 70, 300, 517), ("32x32", "whole", "bf16", 70, 300, 517), ("32x32", "cut", "f32", 48, 40, 4600), ("32x32", "cut", "bf16", 48, 40, 4600),
         ("64x64", "whole", "f32", 321, 1500, 130), ("64x64", "whole", "bf16", 321, 1500, 130), ("64x64", "cut", "f32", 200, 257, 4600), ("64x64", "cut", "bf16", 900, 257, 4600),
         ("64x128", "whole", "f32", 1901, 1157, 1163), ("64x128", "whole", "bf16", 1500, 1500, 259), ("64x128", "whole", "f32", 3001, 700, 515), ("64x128", "cut", "f32", 513, 1157, 4600),
         ("128x128", "whole", "f32", 2000, 2050, 259), ("128x128", "whole", "bf16", 3001, 1500, 130), ("128x128", "cut", "f32", 1500, 1500, 4600), ("128x128", "cut", "bf16", 1500, 1500, 4600)]
FORMATS = [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")]


def _pack(a, fmt):
    p = binding.rl_f8_pack(base.rows(a, torch.float32), fmt)
    return p, base.f64(binding.rl_f8_unpack(p, torch.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("fa, fb", FORMATS)
@pytest.mark.parametrize("tile, pieces, dtype, M, N, K", TILES)
def test_tile(tile, pieces, dtype, M, N, K, fa, fb):
    rng = np.random.default_rng(M + N + K)
    t = base.DT[dtype]
    if dtype == "f32":                                               # of two bits, other scales in other rows
        a, va = _pack(rng.integers(-3, 4, size=(M, K)) * 2.0 ** rng.integers(0, 3, size=(M, 1)), fa)
        b, vb = _pack(rng.integers(-3, 4, size=(N, K)).astype(float), fb)
        want = va @ vb.T
        assert (np.abs(va) @ np.abs(vb).T).max() < 2 ** 24
    else:
        a, va = _pack(rng.normal(size=(M, K)) * 2.0 ** rng.integers(-9, 9, size=(M, 1)), fa)
        at, by = rng.integers(0, K, size=N), rng.choice([-1.0, 2.0, 0.5, 8.0], size=N)
        w = np.zeros((N, K))
        w[np.arange(N), at] = by
        b, _ = _pack(w, fb)
        want = va[:, at] * by
    y = binding.rl_f8_matmul(a, b, t)
    assert np.array_equal(base.f64(y), want)
    a, va = _pack(base.state(rng, M, K), fa)
    b, vb = _pack(rng.normal(size=(N, K)) / K ** 0.5, fb)
    y = binding.rl_f8_matmul(a, b, t)
    want = va @ vb.T
    tol = (2 * (K + 32) * base.U + base.CUT[dtype]) * (np.abs(va) @ np.abs(vb).T) + base.half_step(t, want)
    assert np.all(np.abs(base.f64(y) - want) <= tol), np.max(np.abs(base.f64(y) - want) / tol)
    assert np.linalg.norm(base.f64(y) - want) <= 2.0 ** -8 * np.linalg.norm(want)
    assert torch.equal(y, binding.rl_f8_matmul(a, b, t))


@pytest.mark.gpu
@pytest.mark.parametrize("M, N, K", [(1, 40, 300), (5, 100, 1157), (3, 16, 5000), (16, 33, 513)])
@pytest.mark.parametrize("fa, fb", FORMATS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_few_rows_packed_where_they_are_multiplied(M, N, K, fa, fb, dtype):
    rng = np.random.default_rng(M + N)
    t = base.DT[dtype]
    x = base.rows(base.state(rng, M, K), t)
    w = binding.rl_f8_pack_weight(base.rows(rng.normal(size=(N, K)) / K ** 0.5, torch.float32), fb, transposed=False)
    y, kept = binding.rl_f8_linear_forward(x, w, fa)
    packed = binding.rl_f8_pack(x, fa)
    assert torch.equal(kept.codes, packed.codes) and torch.equal(kept.scales, packed.scales)
    va, vb = base.f64(binding.rl_f8_unpack(packed, torch.float32)), base.f64(binding.rl_f8_unpack(w.rows, torch.float32))
    want = va @ vb.T
    tol = (2 * (K + 32) * base.U + base.CUT[dtype]) * (np.abs(va) @ np.abs(vb).T) + base.half_step(t, want)
    for got in (y, binding.rl_f8_matmul(packed, w.rows, t)):
        assert np.all(np.abs(base.f64(got) - want) <= tol)
