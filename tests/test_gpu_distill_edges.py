"""Scoring with top alternatives and distillation where rows, weights or logits are out of the ordinary: rows without a list, numbers that are none, a token that is nearly certain."""
import numpy as np
import pytest
import torch

from oracle import distill_oracle as orc
from paper_2603_16435_amd import binding
from test_gpu_distill import Batch, DTYPES, U, host, near, off_grid

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


# a token nearly certain, and the list says so: what is left to learn, 1 - q and its logarithm, is a sum of positive terms over the other tokens, and is right relative to itself.  Column 0 of the weight
# is that token's alone, so that column 0 of d_hidden is its dS times a number.  With e^-d of the others off by 156 u and the sums by 26 u (see test_nearly_certain_tokens), 1 - q and KL are off by
# 182 u of themselves (where another token is the likelier one, 26 u more of a KL above one); then dS and d_hidden round once each.  (1e-13: the oracle's own differences.)
@pytest.mark.parametrize("R,H,V,dtype", [(1, 64, 300, "bf16"), (40, 128, 3000, "bf16"), (300, 136, 5001, "bf16"), (3, 36, 200, "f32"), (100, 68, 5001, "f32"), (200, 68, 777, "f32"), (1100, 100, 900, "f32")])
@pytest.mark.parametrize("lift,tau", [(1.0, 1.0), (1.0, 0.7), (1.25, 1.0), (1.5, 1.0)])
@pytest.mark.parametrize("runner_up", [False, True])
@pytest.mark.parametrize("rest", ["bucket", "renormalise"])
def test_a_list_of_a_nearly_certain_token(R, H, V, dtype, lift, tau, runner_up, rest):
    b = Batch(R, H, V, dtype, seed=R + 7, masked=0.0)
    y = int(b.ids[0])
    b.weight[:, :2], b.hidden[:, :2] = 0.0, 16.0
    b.weight[y, 0] = lift
    if runner_up:                                              # eight below it in the same group
        b.weight[y - 1 if y % 64 else y + 1, 1] = lift - 0.5
    ids, lp = torch.full((R, 1), y, dtype=torch.int32, device="cuda"), torch.zeros(R, 1, device="cuda")
    r = b.distill(ids, lp, rest=rest, temperature=tau, aggregation="token", d_weight_dtype=DTYPES[dtype])
    want = orc.distill(host(b.hidden), host(b.weight), host(ids), host(lp), host(b.mask), host(b.cu), rest, tau, "token")
    kl = want["row_loss"]
    near(r.row_loss, kl, 182 * U * kl + 26 * U * (kl > 1) + 1e-13, "row_loss")
    ref = want["dS"][:, y] * lift
    half = 2.0 ** -8 if dtype == "bf16" else U
    near(r.d_hidden[:, 0], ref, (182 * U + 2.01 * half) * np.abs(ref) + 2e-13 / R, "d_hidden")


# scoring: few tokens in bf16 and in f32, tiles of both, a weight off the 16-byte grid
@pytest.mark.parametrize("R,H,V,dtype,off", [(1, 64, 300, "bf16", 0), (60, 128, 3000, "bf16", 0), (100, 136, 20000, "bf16", 0), (300, 128, 1000, "bf16", 0), (300, 72, 1000, "bf16", 0),
                                             (200, 64, 700, "bf16", 1), (3, 36, 200, "f32", 0), (60, 68, 777, "f32", 0), (200, 68, 777, "f32", 0), (1100, 100, 20011, "f32", 0), (200, 36, 700, "f32", 1)])
@pytest.mark.parametrize("where", ["group", "far"])
def test_a_logit_below_all_numbers_has_no_part_in_the_entropy(R, H, V, dtype, off, where):
    """Logits that overflow to -inf, in the group of the largest and in others; and logits so far apart that their difference overflows.  Their tokens have probability 0.  (A sum
    of e d over the others: an exponential as in test_gpu_distill.py, sums in f64, entropy within 32 u (2 + 2 x 60).)"""
    b = Batch(R, H, V, dtype, seed=R + 5, masked=0.0)
    b.weight[:, 0], b.hidden[:, 0] = 0.0, 4.0
    low = torch.tensor([1, 70, V // 2, V - 1], device="cuda") % V
    if where == "group":
        b.weight[low, 0] = -3e38
        b.weight[low, 1:] = 0.0
    else:
        b.weight[64:128, 0], b.weight[5, 0] = -7.5e37, 7.5e37
    if off:
        b.weight = off_grid(b.weight, off)
    r = b.score(3, 1.0)
    want = orc.top_logprobs(host(b.hidden), host(b.weight), host(b.ids), host(b.mask), host(b.cu), 3, 1.0)
    assert bool(r.entropy.isfinite().all()) and bool(r.lse.isfinite().all())
    near(r.entropy, want["entropy"], 32 * U * (2 + 2 * 60), "entropy")
    assert np.array_equal(host(r.top_ids), want["top_ids"])


@pytest.mark.parametrize("R,H,V,dtype", [(40, 128, 3000, "bf16"), (300, 136, 5001, "bf16"), (20, 36, 700, "f32"), (200, 68, 777, "f32")])
def test_the_lowest_temperatures(R, H, V, dtype):
    """At the lowest that is taken a row's largest logit has all of the probability, shared out among equal ones: numbers everywhere, and those of the definition."""
    tau = 4.3e-39
    b = Batch(R, H, V, dtype, seed=R + 9, masked=0.0)
    r = b.score(2, tau)
    want = orc.top_logprobs(host(b.hidden), host(b.weight), host(b.ids), host(b.mask), host(b.cu), 2, tau)
    assert np.array_equal(host(r.top_ids), want["top_ids"])
    near(r.top_logprob[:, 0], want["top_logprob"][:, 0], 32 * U, "top_logprob")
    near(r.entropy, want["entropy"], 64 * U, "entropy")
    d = b.distill(r.top_ids[:, :1].contiguous(), torch.zeros(R, 1, device="cuda"), temperature=tau, rest="renormalise", aggregation="token")
    near(d.row_loss, -want["top_logprob"][:, 0], 32 * U, "row_loss")
    assert bool(d.d_hidden.isfinite().all()) and bool(d.d_weight.isfinite().all())
