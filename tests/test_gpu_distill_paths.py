"""Distillation and scoring on the paths that only large or oddly cut calls take: weight gradients that several chunks add to, hidden states that span 4 GiB, very many rounds of tiles; and
the loss and the gradient of the kernels against each other."""
import numpy as np
import pytest
import torch

from paper_2603_16435_amd import binding
from test_gpu_distill import Batch, DTYPES, SUM, U, check_distill

pytestmark = pytest.mark.gpu


# every chunk has rows, the last one's tile of d_weight joins what the others left: whole tiles, in whole lines and not, and edges
@pytest.mark.parametrize("R,H,V", [(700, 256, 1024), (513, 256, 512), (1000, 264, 4097), (600, 128, 1500), (780, 520, 769)])
@pytest.mark.parametrize("dw", ["bf16", "f32"])
def test_chunks_that_all_have_rows(R, H, V, dw):
    b = Batch(R, H, V, "bf16", seed=R + V, masked=0.0, B=1)
    ids, lp = b.teacher(9, wild=False)
    r = b.distill(ids, lp, aggregation="token", chunk_rows=256, d_weight_dtype=DTYPES[dw])
    assert int(r.stats[0]) == R
    check_distill(b, r, ids, lp, "bucket", 1.0, "token")


def test_chunks_that_all_have_rows_f32():
    b = Batch(600, 100, 1500, "f32", seed=3, masked=0.0, B=1)
    ids, lp = b.teacher(9, wild=False)
    check_distill(b, b.distill(ids, lp, aggregation="token", chunk_rows=256), ids, lp, "bucket", 1.0, "token")


@pytest.mark.parametrize("H", [512, 520])
def test_rows_more_than_4_gib_apart(H):
    """... give what the same rows give close together, to the bit."""
    near = Batch(340, H, 300, "bf16", seed=91, masked=0.0, cu=[0, 40, 340])
    ids, lp = near.teacher(7, wild=False)
    R = (1 << 32) // (2 * H) + 512                              # 512 rows past the 4 GiB
    at = torch.cat([torch.arange(40), torch.arange(R - 300, R)]).cuda()
    far = []
    for v in (near.hidden, near.ids, near.mask, ids, lp):
        w = torch.zeros(R, *v.shape[1:], dtype=v.dtype, device="cuda")
        w[at] = v
        far.append(w)
    x, y, mask, f_ids, f_lp = far
    cu = torch.tensor([0, 40, R], dtype=torch.int32, device="cuda")
    want, top = near.distill(ids, lp, d_weight_dtype=torch.bfloat16), near.score(7)
    t = binding.rl_token_top_logprobs(x, near.weight, y, mask, 7, cu_seqlens=cu, chunk_rows=1 << 20)
    for f in ("logprob", "lse", "entropy", "top_ids", "top_logprob"):
        assert torch.equal(getattr(t, f)[at], getattr(top, f)), f
    assert int((t.lse != 0).sum()) <= 340 and int((t.top_ids >= 0).any(1).sum()) == 340
    d = binding.rl_distill_loss_fwd_bwd(x, near.weight, f_ids, f_lp, mask, cu, chunk_rows=1 << 20, d_weight_dtype=torch.bfloat16, d_hidden=x)
    for f in ("loss", "d_weight", "stats"):
        assert torch.equal(getattr(d, f), getattr(want, f)), f
    for f in ("row_loss", "lse", "d_hidden"):
        assert torch.equal(getattr(d, f)[at], getattr(want, f)), f
    assert int((d.d_hidden != 0).any(1).sum()) <= 340


@pytest.mark.parametrize("dw", ["bf16", "f32"])
def test_very_many_rounds_of_tiles(dw):
    """A chunk of more than 33280 rows with more than 6144 tiles of d_weight, five in a row: vocabulary entries and rows picked at random, in 64 bits.  Inputs lie on grids on which logits are sums
    without rounding; q is off by SUM and lse's own rounding, dS rounds once to bf16, the contractions as in test_gpu_distill.py."""
    R, H, V, K, tau = 33_400, 1032, 314_900, 4, 1.25
    g = torch.Generator(device="cuda").manual_seed(5)
    sw = 2.0 ** round(np.log2(1.2 / np.sqrt(H) / 10))
    w = ((torch.randn(V, H, generator=g, device="cuda") * (1.2 / np.sqrt(H) / sw)).round().clamp(-31, 31) * sw).bfloat16()
    x = ((torch.randn(R, H, generator=g, device="cuda") * 16).round().clamp(-60, 60) / 16).bfloat16()
    mask = torch.ones(R, dtype=torch.uint8, device="cuda")
    ids = (torch.arange(R * K, device="cuda").view(R, K) * 9973 % V).int()
    lp = torch.log_softmax(torch.randn(R, K, generator=g, device="cuda"), 1)
    r = binding.rl_distill_loss_fwd_bwd(x, w, ids, lp, mask, rest="renormalise", temperature=tau, aggregation="token", chunk_rows=R, d_weight_dtype=DTYPES[dw])
    f = 1.0 / R / float(np.float32(tau))
    p = torch.softmax(lp.double(), 1)

    def check(got, d, gross, other, n):
        want, size = d @ other, (d.abs() @ other.abs())
        err = (2.0 ** -16 * gross + 2.0 ** -8 * d.abs()) @ other.abs()
        half = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
        off = (got.double() - want).abs()
        assert bool((off <= err + (n + 64) * U * size + half * (want.abs() + err) + 1e-37).all()), (off / want.abs().clamp(min=1e-30)).max()

    some = torch.cat([torch.randint(V, (24,), generator=g, device="cuda"), ids[::4800, 1].long(), torch.tensor([0, V - 1], device="cuda")])
    q = torch.exp(x.double() @ w[some].double().t() / tau - r.lse.double()[:, None])
    target = sum(torch.where(ids[:, k:k + 1].long() == some[None], p[:, k:k + 1], 0.0) for k in range(K))
    d = f * (q - target)
    check(r.d_weight[some], d.t().contiguous(), (d.abs() + 2 * f * q).t().contiguous(), x.double(), R)
    rows = torch.cat([torch.randint(R, (14,), generator=g, device="cuda"), torch.tensor([0, 33_279, 33_280, R - 1], device="cuda")])
    wide = w.double()
    z = x[rows].double() @ wide.t() / tau
    q = torch.softmax(z, 1)
    d = f * q.scatter_add(1, ids[rows].long(), -p[rows])
    check(r.d_hidden[rows], d, d.abs() + 2 * f * q, wide, V)
    lse = torch.logsumexp(z, 1)
    assert bool(((r.lse[rows].double() - lse).abs() <= SUM + 2 * U * lse.abs() + 2 * U * 60).all())


@pytest.mark.parametrize("rest,tau", [("bucket", 1.0), ("renormalise", 1.5)])
@pytest.mark.parametrize("R,V", [(30, 150), (150, 700)])
def test_differences_of_the_kernels_own_loss(rest, tau, R, V):
    """f32: (KL(x + h e) - KL(x - h e)) / 2 h of the call itself against its gradient, row by row for the hidden states and in the sum for the weight, along random directions scaled to change no logit by
    more than tau h.  A row's KL (below 16) is off by 2 SUM + 4 u 60 + 16 u on each side (see check_distill), 320 u / h; its third derivative is that of two logarithms of sums, each at most 2^3: 16 h^2 / 6.  The gradient's own
    rounding, 2^-12 of its terms at most, is far below both."""
    b = Batch(R, 16, V, "f32", seed=14, masked=0.0, B=1)
    ids, lp = b.teacher(8, wild=False)
    run = lambda x, w, back=False: binding.rl_distill_loss_fwd_bwd(x, w, ids, lp, b.mask, b.cu, rest=rest, temperature=tau, aggregation="token", backward=back)
    r = run(b.hidden, b.weight, True)
    h, g = 2.0 ** -6, torch.Generator(device="cuda").manual_seed(3)
    tol = 320 * U / h + 16 * h * h / 6
    biggest = 0.0
    for _ in range(4):
        e = torch.randn(R, 16, generator=g, device="cuda")
        e *= tau / (e @ b.weight.t()).abs().amax(1, keepdim=True)
        slope = (run(b.hidden + h * e, b.weight).row_loss.double() - run(b.hidden - h * e, b.weight).row_loss.double()) / (2 * h)
        got = R * (r.d_hidden.double() * e.double()).sum(1)
        assert bool(((slope - got).abs() <= tol + 2.0 ** -12 * R * (r.d_hidden * e).abs().sum(1)).all())
        biggest = max(biggest, float(slope.abs().max()))
        e = torch.randn(V, 16, generator=g, device="cuda")
        e *= tau / (b.hidden @ e.t()).abs().max()
        slope = (run(b.hidden, b.weight + h * e).row_loss.double() - run(b.hidden, b.weight - h * e).row_loss.double()).mean() / (2 * h)
        got = (r.d_weight.double() * e.double()).sum()
        assert (slope - got).abs() <= tol + 2.0 ** -12 * (r.d_weight * e).abs().sum()
    assert biggest > 20 * tol                                    # (there is a slope to be found)
