"""Scoring with top alternatives and distillation through the C ABI, against the float64 oracle.

Inputs lie on grids of powers of two on which every logit is a sum without rounding, so that the order of the alternatives is that of the oracle to the bit, and what is
left in the tolerances is what follows the logits.  With u = 2^-24 (half a step of f32, relative):
  * an exponential: the difference to the maximum and its scaling round once each, which changes e = exp(-d) by 2 u d e, summed at most 2 u sum d e; exp2 itself 2 u.
    A group's 64 are added in chains of 18 at most: 18 u.  Groups are added in f64, their weights are exponentials of the same kind: 2 u d + 2 u.  d e^-d <= 0.37,
    so a sum is off by less than 26 u of itself, its logarithm by 26 u.  SUM = 32 u.
  * lse and log-probabilities: SUM, and their own rounding.   * entropy: ln S (SUM) and sum e d / S, off by 32 u (1 + D) D with D = its value: SUM (2 + 2 D).
  * dS: exponentials of the row's maximum, SUM more from the sum: (32 + 2 d) u of each magnitude that it is the difference of, d < 60 here: 2^-16.  Then one rounding, 2^-8 in bf16.
  * contractions of n terms: n u of the sum of magnitudes; one rounding at the end (2^-8 in bf16, u in f32)."""
import numpy as np
import pytest
import torch

from oracle import distill_oracle as orc
from paper_2603_16435_amd import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SUM = 32 * U
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def off_grid(t, elements):
    """The same values in a tensor that starts `elements` behind a 16-byte boundary."""
    buf = torch.empty(t.numel() + elements, dtype=t.dtype, device=t.device)
    buf[elements:].copy_(t.flatten())
    return buf[elements:].view(t.shape)


class Batch:
    def __init__(self, R, H, V, dtype, seed=0, B=3, w_levels=31, x_levels=60, masked=0.25, cu=None):
        g = torch.Generator().manual_seed(seed)
        sw = 2.0 ** round(np.log2(1.2 / np.sqrt(H) / (w_levels / 3)))
        self.weight = ((torch.randn(V, H, generator=g) * 1.2 / np.sqrt(H) / sw).round().clamp(-w_levels, w_levels) * sw).to(DTYPES[dtype]).cuda()
        x = torch.randn(R, H, generator=g) + (torch.rand(R, 1, generator=g) * 12) * self.weight.float().cpu()[torch.randint(V, (R,), generator=g)]
        self.hidden = ((x * 16).round().clamp(-x_levels, x_levels) / 16).to(DTYPES[dtype]).cuda()
        self.ids = torch.randint(V, (R,), generator=g, dtype=torch.int32).cuda()
        self.mask = (torch.rand(R, generator=g) >= masked).to(torch.uint8)
        if R == 1:
            self.mask[0] = 1
        self.mask = self.mask.cuda()
        cuts = sorted(torch.randint(R + 1, (B - 1,), generator=g).tolist())
        self.cu = torch.tensor([0, *cuts, R] if cu is None else cu, dtype=torch.int32, device="cuda")
        self.R, self.H, self.V, self.dtype, self.g = R, H, V, dtype, g

    def teacher(self, K, spread=1.5, wild=True):
        """Lists out of a perturbed student, some short or empty; wild: tokens named twice or out of range, log-probabilities of -inf, and anything where nothing counts."""
        z = (self.hidden.double() @ self.weight.double().t()).cpu() + spread * torch.randn(self.R, self.V, generator=self.g, dtype=torch.float64)
        top = z.topk(min(K, self.V), 1)
        ids = torch.full((self.R, K), -1, dtype=torch.int32)
        lp = torch.zeros(self.R, K)
        ids[:, :top.indices.shape[1]] = top.indices.int()
        lp[:, :top.indices.shape[1]] = (top.values - torch.logsumexp(z, 1, keepdim=True)).float()
        have = torch.where(torch.rand(self.R, generator=self.g) < 0.3, torch.randint(K + 1, (self.R,), generator=self.g), K)
        gone = torch.arange(K)[None] >= have[:, None]
        ids[gone], lp[gone] = -1, float("nan")
        if wild:
            for r in range(0, self.R, 5):
                a, b = torch.randint(K, (2,), generator=self.g).tolist()
                if a < b and ids[r, a] >= 0 and ids[r, b] >= 0:
                    ids[r, b] = ids[r, a]
            for r, bad in ((1, self.V), (2, -2), (3, 2 ** 31 - 1), (4, -2 ** 31)):
                if r < self.R:
                    ids[r, K // 2] = bad
            if self.R > 6 and ids[6, 0] >= 0:
                lp[6, 0] = -float("inf")
            hide = self.mask.cpu() == 0
            ids[hide], lp[hide] = 7 * self.V, float("nan")
        return ids.cuda(), lp.cuda()

    def score(self, K, tau=1.0, **kw):
        return binding.rl_token_top_logprobs(self.hidden, self.weight, kw.pop("ids", self.ids), self.mask, K, temperature=tau, cu_seqlens=self.cu, **kw)

    def distill(self, ids, lp, **kw):
        return binding.rl_distill_loss_fwd_bwd(self.hidden, self.weight, ids, lp, self.mask, self.cu, **kw)


def host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def near(got, want, tol, what):
    got = host(got).astype(np.float64)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), got[bad][:4], want[bad][:4], np.broadcast_to(tol, want.shape)[bad][:4])


def check_score(b, r, K, tau):
    want = orc.top_logprobs(host(b.hidden), host(b.weight), host(b.ids), host(b.mask), host(b.cu), K, tau)
    assert np.array_equal(host(r.top_ids), want["top_ids"])
    for f in ("lse", "logprob", "top_logprob"):
        near(getattr(r, f), want[f], SUM + 2 * U * np.abs(want[f]) + 2 * U * 60, f)
    near(r.entropy, want["entropy"], SUM * (2 + 2 * 60), "entropy")


def check_distill(b, r, ids, lp, rest, tau, aggregation, scale=1.0):
    want = orc.distill(host(b.hidden), host(b.weight), host(ids), host(lp), host(b.mask), host(b.cu), rest, tau, aggregation, scale)
    assert r.stats_dict() == want["stats"]
    near(r.lse, want["lse"], SUM + 4 * U * 60, "lse")
    # each log p - log q is off by SUM and its own roundings, and the p add up to one
    row = 2 * SUM + 4 * U * 60 + U * np.abs(want["row_loss"])
    near(r.row_loss, want["row_loss"], row, "row_loss")
    near(r.loss, np.array([want["loss"]]), abs(scale) * row.max() + U * abs(want["loss"]), "loss")
    if r.d_hidden is None:
        return
    bf = b.dtype == "bf16"
    ds, x, w = np.abs(want["dS"]), np.abs(host(b.hidden).astype(np.float64)), np.abs(host(b.weight).astype(np.float64))
    err = 2.0 ** -16 * want["gross"] + (2.0 ** -8 * ds if bf else U * ds) + 1e-37
    for got, ref, e, gross, n in ((r.d_hidden, want["d_hidden"], err @ w, ds @ w, b.V), (r.d_weight, want["d_weight"], err.T @ x, ds.T @ x, b.R)):
        half = 2.0 ** -8 if got.dtype == torch.bfloat16 else U
        near(got, ref, e + (n + 64) * U * gross + half * (np.abs(ref) + e) + 1e-37, "gradient")


# bf16: few tokens (64, 128), the hot kernel (H on the grid of 128, off it), whole and partial tiles, one group, several chunks; f32: narrow tiles, 256 x 64, a K tail
SCORE = [(1, 64, 300, "bf16", 1, 0), (1, 512, 20000, "bf16", 20, 0), (63, 128, 129, "bf16", 128, 0), (65, 136, 5000, "bf16", 7, 0), (128, 456, 65537, "bf16", 5, 0),
         (129, 128, 1000, "bf16", 128, 0), (300, 256, 50257, "bf16", 33, 0), (700, 264, 4097, "bf16", 64, 256), (530, 128, 64, "bf16", 64, 512),
         (1, 4, 5, "f32", 5, 0), (16, 36, 64, "f32", 9, 0), (17, 260, 20000, "f32", 3, 0), (33, 516, 3000, "f32", 20, 0), (64, 520, 41000, "f32", 2, 0), (31, 1028, 2000, "f32", 33, 0),
         (65, 68, 777, "f32", 9, 0), (300, 128, 8200, "f32", 128, 256), (1100, 100, 20011, "f32", 11, 0), (2, 64, 130000, "f32", 100, 0)]


@pytest.mark.parametrize("R,H,V,dtype,K,chunk", SCORE)
@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_score(R, H, V, dtype, K, chunk, tau):
    b = Batch(R, H, V, dtype, seed=R + V)
    check_score(b, b.score(K, tau, chunk_rows=chunk), K, tau)


# ties: a few values only, all equal, more equal at the K-th place than there is room for
@pytest.mark.parametrize("R,H,V,dtype,K", [(70, 64, 3000, "bf16", 128), (200, 64, 20000, "bf16", 100), (300, 64, 70000, "f32", 5), (90, 16, 8192, "f32", 128)])
@pytest.mark.parametrize("kind", ["few", "equal", "blocks"])
def test_ties_go_to_the_lower_token(R, H, V, dtype, K, kind):
    b = Batch(R, H, V, dtype, seed=5, w_levels=1, x_levels=16)
    if kind == "equal":
        b.weight.zero_()
    if kind == "blocks":                                       # the same logits over and over, the largest last
        b.weight = b.weight[:97].repeat(V // 97 + 1, 1)[:V].contiguous()
        b.weight[V - 3:] = b.weight[V - 3]
    check_score(b, b.score(K), K, 1.0)


# distillation: the routes of the forward as above, and of the backward (f32: small tiles in one launch, dX out of dS^T and W, several chunks; bf16: W as it is, W^T)
DISTILL = [(1, 64, 300, "bf16", 1, 0), (61, 128, 3000, "bf16", 8, 0), (128, 136, 5000, "bf16", 100, 0), (300, 256, 1025, "bf16", 128, 0), (700, 264, 4097, "bf16", 30, 256),
           (1, 4, 5, "f32", 5, 0), (50, 68, 777, "f32", 9, 0), (600, 128, 1500, "f32", 128, 256), (900, 100, 6001, "f32", 21, 0), (1100, 260, 3000, "f32", 16, 0)]


@pytest.mark.parametrize("R,H,V,dtype,K,chunk", DISTILL)
@pytest.mark.parametrize("rest,tau,aggregation", [("bucket", 1.0, "sequence"), ("renormalise", 1.7, "token"), ("bucket", 0.6, "token")])
def test_distill(R, H, V, dtype, K, chunk, rest, tau, aggregation):
    b = Batch(R, H, V, dtype, seed=R + V + 1)
    ids, lp = b.teacher(K)
    r = b.distill(ids, lp, rest=rest, temperature=tau, aggregation=aggregation, chunk_rows=chunk, d_weight_dtype=DTYPES[dtype])
    check_distill(b, r, ids, lp, rest, tau, aggregation)


# few rows, whose gradients are one pass over the weight: every number of token blocks, columns inside a wavefront's, at its border and past it, vocabularies inside a step, past the
# last whole one, in one run and in many; a weight off the 16-byte grid takes the other route
@pytest.mark.parametrize("R,H,V,dtype", [(1, 8, 33, "bf16"), (16, 128, 64, "bf16"), (17, 136, 1000, "bf16"), (32, 264, 4001, "bf16"), (33, 120, 300, "bf16"), (64, 1160, 9000, "bf16"),
                                         (65, 64, 700, "bf16"), (100, 200, 5001, "bf16"), (128, 1032, 3000, "bf16"), (3, 4, 17, "f32"), (16, 64, 48, "f32"), (17, 68, 1001, "f32"),
                                         (32, 516, 9003, "f32"), (33, 60, 500, "f32")])
@pytest.mark.parametrize("dw,off", [("own", 0), ("f32", 0), ("own", 1)])
def test_few_rows(R, H, V, dtype, dw, off):
    b = Batch(R, H, V, dtype, seed=R + H)
    ids, lp = b.teacher(7)
    if off:
        b.weight, b.hidden = off_grid(b.weight, off), off_grid(b.hidden, off)
    r = b.distill(ids, lp, aggregation="token", d_weight_dtype=DTYPES[dtype] if dw == "own" else torch.float32)
    check_distill(b, r, ids, lp, "bucket", 1.0, "token")


# one token far above all others: it has all of the probability, to the last bit, at any temperature
@pytest.mark.parametrize("R,H,V,dtype", [(1, 64, 300, "bf16"), (40, 128, 3000, "bf16"), (300, 136, 5001, "bf16"), (3, 36, 200, "f32"), (200, 68, 777, "f32")])
@pytest.mark.parametrize("tau", [1.0, 0.7, 1.9])
def test_certain_tokens(R, H, V, dtype, tau):
    b = Batch(R, H, V, dtype, seed=R, masked=0.0)
    b.weight[:, 0], b.hidden[:, 0] = 0.0, 37.0                 # (the others' logits are below 50 in size, this one is above 2000)
    b.ids[:] = b.ids[0].clone()
    b.weight[b.ids[0].long(), 0] = 64.0
    r = b.score(2, tau)
    for f in (r.logprob, r.entropy, r.top_logprob[:, 0]):
        assert torch.equal(f, torch.zeros_like(f))
    assert torch.equal(r.top_ids[:, 0], b.ids)
    z = host(b.hidden).astype(np.float64) @ host(b.weight[b.ids[:1].long()]).astype(np.float64)[0]
    near(r.lse, z / tau, 4 * U * np.abs(z / tau), "lse")
    d = b.distill(b.ids[:, None].contiguous(), torch.zeros(R, 1, device="cuda"), temperature=tau, aggregation="token")
    for f in (d.row_loss, d.loss, d.d_hidden, d.d_weight):
        assert torch.equal(f, torch.zeros_like(f))


# a token nearly certain: entropy and its log-probability are small numbers of their own, not what is left of larger ones.  Both are sums of positive terms d^i e^-d over the others;
# a difference to the maximum is exact, its product with c off by 1.3 u of itself (c 0.33 u at these temperatures), exp2 by 2 u, a group's sum by 24 u: with d below 100 each term by 156 u,
# and 26 u for the sums' own roundings and the result's.  Where another token is the likely one, 26 u more from the logarithm of a sum.  (The oracle's differences in f64: 1e-13)
@pytest.mark.parametrize("R,H,V,dtype", [(1, 64, 300, "bf16"), (40, 128, 3000, "bf16"), (300, 136, 65001, "bf16"), (3, 36, 200, "f32"), (200, 68, 777, "f32")])
@pytest.mark.parametrize("lift,tau", [(1.0, 1.0), (1.5, 0.7), (2.0, 1.0)])
def test_nearly_certain_tokens(R, H, V, dtype, lift, tau):
    b = Batch(R, H, V, dtype, seed=R + 7, masked=0.0)
    b.weight[:, 0], b.hidden[:, 0] = 0.0, 16.0
    b.ids[:] = b.ids[0].clone()
    b.weight[b.ids[0].long(), 0] = lift
    r = b.score(2, tau)
    want = orc.top_logprobs(host(b.hidden), host(b.weight), host(b.ids), host(b.mask), host(b.cu), 2, tau)
    for f in ("entropy", "logprob"):
        near(getattr(r, f), want[f], 182 * U * np.abs(want[f]) + (26 * U if f == "logprob" else 0) * (want[f] < -1) + 1e-13, f)


# lists that name next to nothing: with p, q ~ 1e-3 the divergence is ~ (p - q)^2 / q, far below the terms p (log p - log q) and p_r (log p_r - log q_r) that it is the sum of.  With each
# log q_i off by e_i, at most SUM and 2 u d for the temperature's two roundings, 52 u at d < 10, KL moves by sum e_i (q_i p_r / q_r - p_i), and |p_r / q_r - 1| <= 1.25 sum |p - q|: at most
# 1.25 x 52 u sum |p - q|.  The q_i that make q_r are exponentials, 4 u of each, times p_r / q_r <= 1.25
@pytest.mark.parametrize("R,H,V,dtype", [(1, 64, 3000, "bf16"), (60, 128, 20000, "bf16"), (300, 136, 30001, "bf16"), (20, 68, 5000, "f32"), (150, 36, 7777, "f32")])
@pytest.mark.parametrize("K", [1, 4])
def test_lists_of_next_to_nothing(R, H, V, dtype, K):
    tau = 2.9
    b = Batch(R, H, V, dtype, seed=R + 3, masked=0.0, x_levels=16)
    z = (b.hidden.double() @ b.weight.double().t()) / tau
    lq = z - torch.logsumexp(z, 1, keepdim=True)
    ids = torch.randint(V, (R, K), generator=b.g).cuda()
    lp = (lq.gather(1, ids) + 0.1 * torch.randn(R, K, generator=b.g, dtype=torch.float64).cuda()).float()
    ids = ids.int()
    r = b.distill(ids, lp, temperature=tau, aggregation="token")
    want = orc.distill(host(b.hidden), host(b.weight), host(ids), host(lp), host(b.mask), host(b.cu), "bucket", tau, "token", 1.0)
    p, q = np.exp(host(lp).astype(np.float64)), np.exp(lq.gather(1, ids.long()).cpu().numpy())
    both = (p + q).sum(1)
    assert both.max() < 0.2
    near(r.row_loss, want["row_loss"], 65 * U * np.abs(p - q).sum(1) + 5 * U * both + U * np.abs(want["row_loss"]), "row_loss")
    check_distill(b, r, ids, lp, "bucket", tau, "token")


# f32, up to 128 rows: every number of token blocks, 64 and 32 columns of a wavefront, whole and not, vocabularies inside a step and past the last whole one, and a row more
@pytest.mark.parametrize("R,H,V", [(48, 100, 1001), (49, 516, 300), (64, 64, 48), (65, 36, 777), (80, 1028, 40), (96, 132, 2003), (97, 4, 33), (128, 516, 5003), (128, 32, 16), (120, 92, 30001), (129, 68, 999)])
@pytest.mark.parametrize("off", [0, 1])
def test_few_rows_f32(R, H, V, off):
    b = Batch(R, H, V, "f32", seed=R + H + 1, masked=0.1)
    ids, lp = b.teacher(5)
    if off:
        b.weight, b.hidden = off_grid(b.weight, off), off_grid(b.hidden, off)
    check_distill(b, b.distill(ids, lp), ids, lp, "bucket", 1.0, "sequence")
