"""Workspace of the 8-bit linear layer's backward pass: a call reserves what it touches, and touches nothing beyond."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2603_16435_amd import binding
from test_norm_linear_abi import DTYPE, NULL, OK, P, SHAPE, WORKSPACE, lib  # noqa: F401  (lib: fixture)

F32, BF16 = 0, 1


def _need(lib, M, N, K, dtype, lddy, aligned, dx, dW):
    n = C.c_size_t(1)
    assert lib.rl_f8_linear_backward_workspace_bytes_for(M, N, K, dtype, lddy, aligned, dx, dW, C.byref(n)) == OK
    return n.value


def _any(lib, M, N, K, dtype):
    n = C.c_size_t(0)
    assert lib.rl_f8_linear_backward_workspace_bytes(M, N, K, dtype, C.byref(n)) == OK
    return n.value


def test_a_call_reserves_what_it_touches(lib):
    M, N, K = 32749, 3584, 3584
    both, dx, dW = (_need(lib, M, N, K, BF16, N, 1, *w) for w in ((1, 1), (1, 0), (0, 1)))
    packed = M * (N + 28) + 512                       # dy in 8 bits
    restored = 32768 * K * 2                          # x of a chunk in bf16
    assert dx <= packed and restored <= dW <= restored + 256 and both <= packed + restored + 256
    copied = _need(lib, M, N, K, BF16, N, 0, 1, 1)    # rows off 16 bytes are copied first
    assert copied == both + 32768 * N * 2 == _need(lib, M, N, K, BF16, N + 1, 1, 1, 1)
    assert _any(lib, M, N, K, BF16) == copied
    assert _need(lib, M, N, K, F32, N, 1, 1, 1) == _any(lib, M, N, K, F32)
    assert _need(lib, 1, 64, 256, BF16, 64, 1, 1, 0) == 0          # one row is packed where it is multiplied
    assert _need(lib, 0, 64, 256, BF16, 64, 1, 1, 1) == 0


def test_the_plain_query_covers_every_call(lib):
    for M in (1, 17, 300, 5003, 40_000):
        for N, K in ((1, 1), (40, 136), (264, 1157), (1157, 1163), (4096, 512)):
            for dtype in (F32, BF16):
                most = _any(lib, M, N, K, dtype)
                need = [_need(lib, M, N, K, dtype, N + pad, al, dx, dW) for pad in (0, 3, 8) for al in (0, 1) for dx in (0, 1) for dW in (0, 1)]
                assert max(need) == most and all(n % 256 == 0 for n in need)


def test_refusals(lib):
    n = C.c_size_t(0)
    q = lib.rl_f8_linear_backward_workspace_bytes_for
    assert q(100, 64, 256, BF16, 64, 1, 1, 1, None) == NULL and q(100, 64, 256, 2, 64, 1, 1, 1, C.byref(n)) == DTYPE
    assert q(-1, 64, 256, BF16, 64, 1, 1, 1, C.byref(n)) == SHAPE and q(100, 64, 256, BF16, 63, 1, 1, 1, C.byref(n)) == SHAPE
    for aligned, dx, dW in ((1, 1, 1), (1, 1, 0), (0, 0, 1)):
        need = _need(lib, 100, 64, 256, BF16, 64, aligned, dx, dW)
        dy = P if aligned else P + 2
        call = [dy, 64, BF16, 100, 64, 256, 1, P, P, 0, P, P, 0, P if dx else None, 256, P if dW else None, 256, 0]
        assert need and lib.rl_f8_linear_backward(*call, P, need - 1, None) == WORKSPACE and lib.rl_f8_linear_backward(*call, None, need, None) == WORKSPACE


@pytest.mark.gpu
@pytest.mark.parametrize("M, N, K", [(1, 64, 256), (40, 72, 130), (300, 264, 264), (700, 520, 640), (33000, 40, 136)])
@pytest.mark.parametrize("dtype, pad", [("bf16", 0), ("bf16", 3), ("f32", 0)])
def test_nothing_beyond_it_is_touched(lib, M, N, K, dtype, pad):
    """The bytes that the query names, between others that stay: the same results as through the binding."""
    rng = np.random.default_rng(M)
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    dy = torch.from_numpy(rng.normal(size=(M, N + pad))).to(t).cuda()[:, :N]
    kept = binding.rl_f8_pack(torch.from_numpy(rng.normal(size=(M, K))).to(t).cuda())
    w = binding.rl_f8_pack_weight(torch.from_numpy(rng.normal(size=(N, K))).to(t).cuda())
    want = binding.rl_f8_linear_backward(dy, kept, w)
    pdy, lddy, dt = binding._rows(dy, "dy")
    cx, sx, fx = kept._pointers("kept")
    ct, st, fw = w.cols._pointers("w")
    for need_dx, need_dw in ((1, 1), (1, 0), (0, 1)):
        need = _need(lib, M, N, K, dt, lddy, int(pdy % 16 == 0), need_dx, need_dw)
        room = torch.full((need + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
        at = 4096 + (-room.data_ptr()) % 256
        dx, dw = torch.zeros((M, K), dtype=t, device="cuda"), torch.zeros((N, K), device="cuda")
        assert lib.rl_f8_linear_backward(pdy, lddy, dt, M, N, K, 1, cx, sx, fx, ct, st, fw, dx.data_ptr() if need_dx else None, K, dw.data_ptr() if need_dw else None, K, 0,
                                         room.data_ptr() + at if need else None, need, binding._stream_handle()) == OK
        assert torch.all(room[:at] == 0xA5) and torch.all(room[at + need:] == 0xA5)
        assert not need_dx or torch.equal(dx, want[0])
        assert not need_dw or torch.equal(dw, want[1])


@pytest.mark.gpu
def test_the_binding_reserves_no_more():
    M, N, K = 4096, 1024, 1024
    dy = torch.randn(M, N, device="cuda").bfloat16()
    kept, w = binding.rl_f8_pack(torch.randn(M, K, device="cuda").bfloat16()), binding.rl_f8_pack_weight(torch.randn(N, K, device="cuda"))
    def peak(**want):
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        binding.rl_f8_linear_backward(dy, kept, w, **want)
        return torch.cuda.max_memory_allocated() - before
    slack = 1 << 16
    assert peak(want_dw=False) <= M * K * 2 + M * (N + 8) + slack                                   # dx, dy in 8 bits
    n = C.c_size_t(0)
    assert binding.lib().rl_f8_linear_backward_workspace_bytes_for(M, N, K, BF16, N, 1, 0, 1, C.byref(n)) == OK
    assert peak(want_dx=False) <= N * K * 4 + n.value + slack
