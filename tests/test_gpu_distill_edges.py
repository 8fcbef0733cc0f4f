"""Scoring with top alternatives and distillation where rows, weights or logits are out of the ordinary: rows without a list, numbers that are none, a token that is nearly certain."""
import pytest
import torch

from paper_2603_16435_amd import binding
from test_gpu_distill import Batch, DTYPES, off_grid

pytestmark = pytest.mark.gpu


# few rows (one pass over the weight); tiles, W as it is and W^T, several chunks, hidden states off the 16-byte grid; f32: few rows, small tiles in one launch, several chunks, dX out of dS^T and W
ROUTES = [(40, 128, 3000, "bf16", 0, 0), (300, 136, 2000, "bf16", 256, 0), (300, 128, 1025, "bf16", 0, 0), (40, 136, 700, "bf16", 0, 3), (20, 68, 1000, "f32", 0, 0), (200, 36, 500, "f32", 0, 0),
          (600, 100, 700, "f32", 256, 0), (1100, 260, 3000, "f32", 0, 0), (150, 68, 900, "f32", 0, 1)]


def without_lists(b, ids, lp, rest):
    """Every fifth row without entries, in each of the ways that a row can be; these rows, as a mask."""
    r = torch.arange(b.R, device="cuda")
    gone = r % 5 == 2
    ids[gone] = -1
    ids[gone & (r % 3 == 1)] = b.V
    if rest == "renormalise":
        some = gone & (r % 3 == 2)
        ids[some] = torch.arange(ids.shape[1], dtype=torch.int32, device="cuda")
        lp[some] = -float("inf")
    return gone


@pytest.mark.parametrize("R,H,V,dtype,chunk,off", ROUTES)
@pytest.mark.parametrize("rest", ["bucket", "renormalise"])
@pytest.mark.parametrize("dw", ["own", "f32"])
def test_a_row_without_a_list_has_no_part_in_the_weight_gradient(R, H, V, dtype, chunk, off, rest, dw):
    """Whatever its hidden states are: the gradients are to the bit those of finite ones."""
    b = Batch(R, H, V, dtype, seed=R, masked=0.1)
    ids, lp = b.teacher(5)
    if off:
        b.hidden = off_grid(b.hidden, off)
    gone = without_lists(b, ids, lp, rest)
    run = lambda: b.distill(ids, lp, rest=rest, chunk_rows=chunk, d_weight_dtype=DTYPES[dtype] if dw == "own" else torch.float32)
    want = run()
    assert bool(want.d_weight.isfinite().all()) and bool(want.d_weight.any())
    b.hidden[gone] = float("nan")
    b.hidden[gone & (torch.arange(R, device="cuda") % 2 == 0)] = float("inf")
    got = run()
    for f in ("loss", "row_loss", "d_hidden", "d_weight", "stats"):
        assert torch.equal(getattr(got, f), getattr(want, f)), f
    assert not got.d_hidden[gone].any() and not got.row_loss[gone].any() and int(got.stats[2]) >= int((gone & (b.mask != 0)).sum())


@pytest.mark.parametrize("R,H,V,dtype,chunk,off", ROUTES)
def test_a_row_without_a_list_has_no_gradient_whatever_the_weight_holds(R, H, V, dtype, chunk, off):
    b = Batch(R, H, V, dtype, seed=R + 1, masked=0.1)
    ids, lp = b.teacher(5)
    if off:
        b.weight = off_grid(b.weight, off)
    without_lists(b, ids, lp, "bucket")
    gone = ((ids < 0) | (ids >= V)).all(1)
    b.weight[V // 2, 1], b.weight[V - 1, 0] = float("nan"), float("inf")
    kw = dict(chunk_rows=chunk, d_weight_dtype=DTYPES[dtype])
    r = b.distill(ids, lp, **kw)
    counts = b.mask != 0
    assert not r.d_hidden[gone | ~counts].any() and not r.row_loss[gone | ~counts].any()
    assert bool(r.row_loss[counts & ~gone].isnan().all())
    x = b.hidden.clone()
    over = binding.rl_distill_loss_fwd_bwd(x, b.weight, ids, lp, b.mask, b.cu, d_hidden=x, **kw)
    assert not over.d_hidden[gone | ~counts].any()
    ids.fill_(-1)
    r = b.distill(ids, lp, **kw)
    for f in (r.loss, r.row_loss, r.d_hidden, r.d_weight):
        assert not f.any()
