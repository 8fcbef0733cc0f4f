"""The divergence of a student's block on held-out text: the loss alone, and what the block's step refuses."""
import pytest
import torch

from test_gpu_head_block_distill import example  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [None, 40])
def test_the_loss_alone(example, dtype, rows):  # noqa: F811
    teacher, b, x, _ = example.make(520, 264, 1000, dtype, seed=5)
    student = example.make(520, 264, 1000, dtype, seed=6)[0]
    n = rows or x.shape[0]
    x, ids, mask = x[:n].contiguous(), b.token_ids[:n].contiguous(), b.mask[:n].contiguous()
    cu = torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda")
    top = teacher.top_logprobs(x, ids, mask, 16)
    lists, copy = (top.top_ids, top.top_logprob, mask, cu), x.clone()
    want = student.distill_step(x, *lists, aggregation="token")[0]
    for overwrite in (False, True):
        res, grads = student.distill_step(x, *lists, overwrite=overwrite, aggregation="token", backward=False)
        assert grads is None and res.d_hidden is None and res.d_weight is None and torch.equal(x, copy)
        assert torch.equal(res.loss, want.loss) and torch.equal(res.row_loss, want.row_loss) and torch.equal(res.lse, want.lse) and torch.equal(res.stats, want.stats)
    for backward in (False, True):
        with pytest.raises(ValueError, match="d_hidden"):
            student.distill_step(x, *lists, backward=backward, d_hidden=torch.empty_like(x))
