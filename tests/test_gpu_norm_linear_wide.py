"""Wide rows, many tokens and whole lines of the layers in front of the LM head: the kernels and paths that only such sizes reach.

Weight gradients are checked on whole numbers: every product and every partial sum is one of f32, so that the result is exact in whatever order it is added."""
import numpy as np
import pytest
import torch

import test_gpu_norm_linear as base
from paper_2603_16435_amd import binding

pytestmark = pytest.mark.gpu
DT = base.DT


# ------------------------------------------------------------------ layer norm
# Eight wavefronts a row (4097 to 8192 columns) and sixteen (beyond), more rows than one launch takes in the backward (512).  1300 rows: a workgroup walks a second row in the
# forward (1280 workgroups), 600 and 1300 of more than 8192 columns also in the backward (10 sqrt(rows), at most 256).
@pytest.mark.parametrize("R, H", [(520, 5120), (515, 8200), (600, 12000), (1300, 8200)])
@pytest.mark.parametrize("dtype, params, kept, pad", [("bf16", "f32", None, 0), ("bf16", "bf16", "e4m3", 5), ("f32", "f32", "e5m2", 0), ("f32", "bf16", None, 3)])
def test_layer_norm_of_wide_rows(R, H, dtype, params, kept, pad):
    base.test_layer_norm(R, H, dtype, params, kept, pad)


# Four wavefronts of one piece a row: 1537 to 2048 columns, and 1025 to 1536 up to 1024 rows.
@pytest.mark.parametrize("R, H", [(513, 1157), (1024, 1300), (700, 2048), (1500, 2001)])
@pytest.mark.parametrize("dtype, params, kept, pad", [("bf16", "f32", None, 0), ("bf16", "bf16", "e4m3", 5), ("f32", "f32", "e5m2", 0), ("f32", "bf16", None, 3)])
def test_layer_norm_of_four_wavefronts_a_row(R, H, dtype, params, kept, pad):
    base.test_layer_norm(R, H, dtype, params, kept, pad)


# ------------------------------------------------------------------ weight gradient
def _gradient(dy, kept, w, into=None, ld=None):
    """dW alone, through the C entry: overwritten in rows of `ld` floats, or added to `into`."""
    M, N = dy.shape
    K = kept.cols
    ld = ld or K
    out = torch.full((N, ld), 7.0, device="cuda")
    if into is not None:
        out[:, :K] = into
    pdy, lddy, dt = binding._rows(dy, "dy")
    cx, sx, fx = kept._pointers("kept")
    ws, pws, nws = binding._f8_workspace("rl_f8_linear_backward_workspace_bytes", dy.device, M, N, K, dt)
    binding._check(binding.lib().rl_f8_linear_backward(pdy, lddy, dt, M, N, K, 1, cx, sx, fx, None, None, 0, None, K, out.data_ptr(), ld, int(into is not None), pws, nws,
                                                       binding._stream_handle()))
    assert torch.all(out[:, K:] == 7)
    return out[:, :K]


def _whole(rng, M, N, K, most, some):
    """x, dy of whole numbers, dy below `most`, x other than zero with probability `some`; sums of magnitudes below 2^24."""
    x = rng.integers(-2, 3, size=(M, K)) * (rng.random((M, K)) < some)
    dy = rng.integers(-most, most + 1, size=(M, N))
    x, dy = x.astype(np.float64), dy.astype(np.float64)
    assert (np.abs(dy).T @ np.abs(x)).max() < 2 ** 24
    return x, dy


# Tokens are restored a chunk at a time: 10880 in f32, 32768 in bf16; the second chunk's share is added to the first's.  f32: values of 20 bits, whose three bf16 terms
# are all there.  bf16 rows on 16 bytes are read where they are, others (odd N or stride) are copied.
@pytest.mark.parametrize("M, N, K, dtype, pad, most, some", [
    (10881, 40, 136, "f32", 0, 1 << 19, 0.0005), (22000, 72, 130, "f32", 3, 1 << 19, 0.0003), (32641, 24, 260, "f32", 0, 1 << 19, 0.0002),
    (32769, 40, 136, "bf16", 0, 100, 0.5), (33000, 37, 130, "bf16", 0, 100, 0.5), (33000, 40, 130, "bf16", 3, 100, 0.5), (66000, 264, 264, "bf16", 8, 100, 0.2)])
def test_weight_gradient_over_several_chunks_of_tokens(M, N, K, dtype, pad, most, some):
    rng = np.random.default_rng(M + N)
    x, dy = _whole(rng, M, N, K, most, some)
    want = dy.T @ x
    t = base.rows(dy, DT[dtype], pad)
    kept = binding.rl_f8_pack(base.rows(x, DT[dtype]))
    w = binding.rl_f8_pack_weight(torch.zeros(N, K, device="cuda"))
    assert np.array_equal(base.f64(_gradient(t, kept, w)), want)
    start = rng.integers(-1000, 1000, size=(N, K)).astype(np.float64)
    into = torch.from_numpy(start).float().cuda()
    assert np.array_equal(base.f64(_gradient(t, kept, w, into)), want + start)
    assert np.array_equal(base.f64(binding.rl_f8_linear_backward(t, kept, w, want_dx=False, dw=into)[1]), want + start)


# Few tokens and many tiles: tiles are not cut along the tokens, and whole ones leave in lines of 128 bytes where dW has its rows on them.
@pytest.mark.parametrize("M, N, K, some", [(700, 520, 640, 0.5), (500, 1100, 1280, 0.5), (130, 256, 256, 0.5), (1, 640, 512, 1.0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weight_gradient_in_whole_lines(M, N, K, some, dtype):
    rng = np.random.default_rng(M + N)
    x, dy = _whole(rng, M, N, K, 100, some)
    want = dy.T @ x
    t, kept = base.rows(dy, DT[dtype]), binding.rl_f8_pack(base.rows(x, DT[dtype]))
    w = binding.rl_f8_pack_weight(torch.zeros(N, K, device="cuda"))
    start = rng.integers(-1000, 1000, size=(N, K)).astype(np.float64)
    into = torch.from_numpy(start).float().cuda()
    for ld in (K, K + 2, K + 32):
        assert np.array_equal(base.f64(_gradient(t, kept, w, ld=ld)), want), ld
        assert np.array_equal(base.f64(_gradient(t, kept, w, into, ld=ld)), want + start), ld


def test_weight_gradient_in_lines_and_in_halves_is_the_same():
    """Ordinary values: the same bits, whichever way the tiles leave, and within the rounding of f32 sums."""
    M, N, K = 700, 520, 640
    rng = np.random.default_rng(1)
    x, dy = rng.normal(size=(M, K)), rng.normal(size=(M, N)) * 1e-3
    t, kept = base.rows(dy, torch.bfloat16), binding.rl_f8_pack(base.rows(x, torch.bfloat16))
    w = binding.rl_f8_pack_weight(torch.zeros(N, K, device="cuda"))
    got = _gradient(t, kept, w)
    assert torch.equal(got, _gradient(t, kept, w, ld=K + 2))
    vx, d = base.f64(binding.rl_f8_unpack(kept, torch.float32)), base.f64(t)
    tol = 2 * (M + 32) * base.U * (np.abs(d).T @ np.abs(vx)) + 1e-38
    assert np.all(np.abs(base.f64(got) - d.T @ vx) <= tol)
