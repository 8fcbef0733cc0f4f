"""The layer norm where nothing is kept for a backward pass: no statistics are asked for, allocated or written."""
import pytest
import torch

from paper_2603_16435_amd import binding
from paper_2603_16435_amd.head_block import HeadBlock

pytestmark = pytest.mark.gpu


def _allocations(f):
    f()                                               # (what is loaded or kept on the first call)
    torch.cuda.synchronize()
    before = torch.cuda.memory_stats()["allocation.all.allocated"]
    out = f()
    return out, torch.cuda.memory_stats()["allocation.all.allocated"] - before


@pytest.mark.parametrize("R, H", [(0, 64), (1, 4096), (40, 1157), (1100, 1283), (9, 8200)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_statistics_the_same_output(R, H, dtype):
    x, gamma, beta = torch.randn(R, H, device="cuda").to(dtype), torch.randn(H, device="cuda"), torch.randn(H, device="cuda")
    want, stats, _ = binding.rl_layer_norm_forward(x, gamma, beta)
    assert stats.shape == (R, 2)
    (y, none, kept), n = _allocations(lambda: binding.rl_layer_norm_forward(x, gamma, beta, want_stats=False))
    assert none is None and kept is None and torch.equal(y, want) and n == (1 if R else 0)
    _, n = _allocations(lambda: binding.rl_layer_norm_forward(x, gamma, beta, out=y, want_stats=False))
    assert n == 0
    kept = binding.rl_layer_norm_forward(x, gamma, beta, checkpoint="e4m3", want_stats=False)[2]
    assert torch.equal(kept.codes, binding.rl_f8_pack(x).codes)


def test_scoring_a_token_keeps_nothing():
    block = HeadBlock(torch.ones(256, device="cuda"), torch.zeros(256, device="cuda"), torch.randn(384, 256, device="cuda") / 16, torch.zeros(8, 384, device="cuda").bfloat16())
    x = torch.randn(1, 256, device="cuda").bfloat16()
    hidden, n = _allocations(lambda: block.hidden(x))
    assert n == 2 and torch.equal(hidden, block.forward(x)[0])         # the norm's output, and the result
