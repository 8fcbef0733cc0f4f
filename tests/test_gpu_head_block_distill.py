"""A student's block in front of the LM head learns from the lists of a teacher's: scoring, divergence and all gradients together."""
import importlib.util
import os

import pytest
import torch

from paper_2603_16435_amd import binding

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_head_block", os.path.join(ROOT, "examples", "train_head_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [None, 40])
def test_a_step_is_its_calls_one_after_the_other(example, dtype, rows):
    teacher, b, x, _ = example.make(520, 264, 1000, dtype, seed=5)
    student = example.make(520, 264, 1000, dtype, seed=6)[0]
    n = rows or x.shape[0]
    x, ids, mask = x[:n].contiguous(), b.token_ids[:n].contiguous(), b.mask[:n].contiguous()
    cu = torch.tensor([0, n // 3, n], dtype=torch.int32, device="cuda")
    top = teacher.top_logprobs(x, ids, mask, 16, temperature=1.5)
    want = binding.rl_token_top_logprobs(teacher.hidden(x), teacher.lm_head, ids, mask, 16, temperature=1.5)
    assert torch.equal(top.top_ids, want.top_ids) and torch.equal(top.top_logprob, want.top_logprob) and torch.equal(top.logprob, want.logprob)
    options = dict(temperature=1.5, d_weight_dtype=dtype)
    res, g = student.distill_step(x, top.top_ids, top.top_logprob, mask, cu, **options)
    hidden, kept = student.forward(x)
    ref = binding.rl_distill_loss_fwd_bwd(hidden, student.lm_head, top.top_ids, top.top_logprob, mask, cu, **options)
    dx, dgamma, dbeta, dweight = student.backward(ref.d_hidden, kept)
    assert torch.equal(res.loss, ref.loss) and torch.equal(g.dlm_head, ref.d_weight) and torch.equal(res.row_loss, ref.row_loss)
    assert torch.equal(g.dx, dx) and torch.equal(g.dgamma, dgamma) and torch.equal(g.dbeta, dbeta) and torch.equal(g.dweight, dweight)
    assert torch.all(g.dx[mask == 0] == 0) and bool(g.dx[mask != 0].abs().sum(1).gt(0).all()) and res.loss > 0
    copy = x.clone()
    res2, g2 = student.distill_step(copy, top.top_ids, top.top_logprob, mask, cu, overwrite=True, **options)
    assert torch.equal(res2.loss, res.loss) and torch.equal(g2.dx, g.dx) and torch.equal(g2.dlm_head, g.dlm_head) and not torch.equal(copy, x)
