"""Scoring with top alternatives and distillation, on the CPU: what the C entry points and the binding refuse (nothing reaches a kernel), and the oracle against
independent statements of the same (torch's own losses, autograd, finite differences, closed forms)."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import distill_oracle as orc
from paper_2603_16435_amd import binding

OK, NULL, SHAPE, DTYPE, RANGE, WORKSPACE = 0, 1, 2, 3, 4, 5
BASE = 1 << 40                                       # addresses that are never dereferenced, a TiB apart


def at(k, off=0):
    return BASE * (k + 1) + off


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_16435_amd import build
        build.build(verbose=False)
    return binding.lib()


def batch(**over):
    b = binding.rl_batch()
    b.R, b.H, b.V, b.B, b.P, b.dtype = 100, 64, 1000, 2, 0, 1
    b.hidden, b.weight, b.token_ids, b.mask, b.cu_seqlens = (at(k) for k in range(5))
    for k, v in over.items():
        setattr(b, k, v)
    return b


TOP = dict(top_k=20, chunk_rows=0, temperature=1.0)
PRM = dict(top_k=20, rest=0, aggregation=0, chunk_rows=0, temperature=1.0, scale=1.0, d_weight_dtype=0)
NAN, INF = float("nan"), float("inf")
SIZES = [(dict(R=0), SHAPE), (dict(R=1 << 31), SHAPE), (dict(H=0), SHAPE), (dict(H=63), SHAPE), (dict(dtype=0, H=66), SHAPE), (dict(V=0), SHAPE), (dict(V=524289), SHAPE),
         (dict(B=0), SHAPE), (dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE)]


def query(fn, b, prm, *more):
    n = C.c_size_t(0)
    return fn(C.byref(b) if b is not None else None, C.byref(prm) if prm is not None else None, *more, C.byref(n)), n.value


def test_workspace_of_scoring(lib):
    q = lambda b, **over: query(lib.rl_token_top_logprobs_workspace_bytes, b, binding.rl_top_params(**dict(TOP, **over)))
    st, need = q(batch())
    assert st == OK and need % 256 == 0 and need > 4 * 256 * 1024          # logits of a chunk
    for over, st in SIZES:
        assert q(batch(**over))[0] == st, over
    for over, st in ((dict(top_k=0), SHAPE), (dict(top_k=-1), SHAPE), (dict(top_k=129), SHAPE), (dict(chunk_rows=-1), SHAPE), (dict(temperature=-1.0), RANGE),
                     (dict(temperature=NAN), RANGE), (dict(temperature=INF), RANGE)):
        assert q(batch(), **over)[0] == st, over
    assert q(batch(V=19))[0] == SHAPE and q(batch(V=20))[0] == OK           # at most as many alternatives as tokens
    assert q(batch(), temperature=0.0) == (OK, need)
    assert query(lib.rl_token_top_logprobs_workspace_bytes, None, binding.rl_top_params(**TOP))[0] == NULL
    assert query(lib.rl_token_top_logprobs_workspace_bytes, batch(), None)[0] == NULL
    assert lib.rl_token_top_logprobs_workspace_bytes(C.byref(batch()), C.byref(binding.rl_top_params(**TOP)), None) == NULL
    big = batch(R=1 << 24, V=256)                                           # a chunk is capped, whatever is asked for
    assert q(big, chunk_rows=(1 << 31) - 1) == q(big, chunk_rows=1 << 20)
    assert q(big, chunk_rows=1) == q(big, chunk_rows=256)
    assert q(big) == q(big, chunk_rows=lib.rl_default_chunk_rows_distill())


def test_workspace_of_distillation(lib):
    q = lambda b, bwd=1, **over: query(lib.rl_distill_workspace_bytes, b, binding.rl_distill_params(**dict(PRM, **over)), bwd)
    st, need = q(batch())
    assert st == OK and need % 256 == 0
    assert q(batch(), bwd=0)[1] < need
    assert q(batch(), d_weight_dtype=1)[1] >= need
    for over, st in SIZES:
        assert q(batch(**over))[0] == st, over
    for over, st in ((dict(top_k=0), SHAPE), (dict(top_k=129), SHAPE), (dict(chunk_rows=-5), SHAPE), (dict(temperature=-0.5), RANGE), (dict(rest=2), RANGE),
                     (dict(rest=-1), RANGE), (dict(aggregation=2), RANGE), (dict(scale=NAN), RANGE), (dict(scale=INF), RANGE), (dict(scale=-INF), RANGE),
                     (dict(d_weight_dtype=2), DTYPE)):
        assert q(batch(), **over)[0] == st, over
    assert q(batch(dtype=0), d_weight_dtype=1)[0] == DTYPE                  # f32 sums of f32 inputs stay f32
    assert q(batch(V=5), top_k=128)[0] == OK                                # a list may have more places than there are tokens
    assert lib.rl_distill_workspace_bytes(C.byref(batch()), C.byref(binding.rl_distill_params(**PRM)), 1, None) == NULL


def top_call(lib, b, out, ws, n, **over):
    return lib.rl_token_top_logprobs(C.byref(b), C.byref(binding.rl_top_params(**dict(TOP, **over))), C.byref(out), ws, n, None)


def test_scoring_refusals(lib):
    full = lambda **over: binding.rl_top_outputs(**dict(dict(logprob=at(5), lse=at(6), entropy=at(7), top_ids=at(8), top_logprob=at(9)), **over))
    need = query(lib.rl_token_top_logprobs_workspace_bytes, batch(), binding.rl_top_params(**TOP))[1]
    ws = at(20)
    for f in ("hidden", "weight", "mask", "cu_seqlens", "token_ids"):
        assert top_call(lib, batch(**{f: None}), full(), ws, need) == NULL, f
    assert top_call(lib, batch(), binding.rl_top_outputs(), ws, need) == NULL
    assert lib.rl_token_top_logprobs(C.byref(batch()), C.byref(binding.rl_top_params(**TOP)), None, ws, need, None) == NULL
    for w, n in ((None, need), (ws + 128, need), (ws, need - 1), (ws, 0)):
        assert top_call(lib, batch(), full(), w, n) == WORKSPACE
    for over in (dict(lse=at(5)), dict(top_ids=at(0, 64)), dict(top_logprob=at(1, 1000 * 64 * 2 - 4)), dict(logprob=at(2)), dict(entropy=at(3, 96)), dict(lse=at(4, 8)),
                 dict(top_logprob=at(8, 100 * 20 * 4 - 4))):
        assert top_call(lib, batch(), full(**over), ws, need) == RANGE, over


def test_distillation_refusals(lib):
    full = lambda **over: binding.rl_distill_outputs(**dict(dict(loss=at(7), row_loss=at(8), lse=at(9), d_hidden=at(10), d_weight=at(11), stats=at(12)), **over))
    prm = lambda **over: C.byref(binding.rl_distill_params(**dict(PRM, **over)))
    need = query(lib.rl_distill_workspace_bytes, batch(), binding.rl_distill_params(**PRM), 1)[1]
    ws = at(20)

    def call(b=None, ids=at(5), lp=at(6), out=None, w=ws, n=need, **over):
        return lib.rl_distill_loss_fwd_bwd(C.byref(b or batch()), ids, lp, prm(**over), C.byref(out or full()), w, n, None)
    for f in ("hidden", "weight", "mask", "cu_seqlens"):
        assert call(batch(**{f: None})) == NULL, f
    assert call(ids=None) == NULL and call(lp=None) == NULL
    for f in ("loss", "d_hidden", "d_weight"):
        assert call(out=full(**{f: None})) == NULL, f
    for w, n in ((None, need), (ws + 8, need), (ws, need - 1)):
        assert call(w=w, n=n) == WORKSPACE
    end_w = 1000 * 64 * 2
    for over in (dict(d_weight=at(1)), dict(d_weight=at(0, 100)), dict(d_hidden=at(0, 2)), dict(d_hidden=at(1, end_w - 2)), dict(d_hidden=at(11, 8)), dict(row_loss=at(5, 40)),
                 dict(lse=at(6)), dict(loss=at(8, 396)), dict(stats=at(3, 96)), dict(d_weight=at(7, -1000 * 64 * 4 + 4))):
        assert call(out=full(**over)) == RANGE, over
    # hidden's place for its gradient is the one exception: refused here for its workspace only
    assert call(out=full(d_hidden=at(0)), n=0) == WORKSPACE


def test_binding_refusals():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
    h, w, m = z(4, 8), z(10, 8), z(4, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        binding.rl_token_top_logprobs(h, w, None, m, 3, cu_seqlens=z(2, dtype=torch.int32))
    with pytest.raises(ValueError, match=r"\[R, K\]"):
        binding.rl_distill_loss_fwd_bwd(h, w, z(4, dtype=torch.int32), z(4), m)
    with pytest.raises(ValueError, match=r"\[R, H\]"):
        binding.rl_token_top_logprobs(z(8), w, None, m, 3)
    with pytest.raises(ValueError, match="one device"):
        binding.rl_token_top_logprobs(h, torch.empty(10, 8, device="meta"), None, m, 3)


# ------------------------------------------------------------------ the oracle
def _case(seed, V=37, K=6, R=9):
    g = np.random.default_rng(seed)
    x, w = g.normal(size=(R, 5)), g.normal(size=(V, 5))
    ids = np.stack([g.permutation(V)[:K] for _ in range(R)])
    t = g.normal(size=(R, V)) * 2
    t = t - np.log(np.exp(t).sum(1, keepdims=True))
    return x, w, ids, np.take_along_axis(t, ids, 1), t


def test_oracle_scores_as_torch_does():
    x, w, _, _, _ = _case(1)
    ids, mask, cu = np.arange(9), np.array([1, 1, 0, 1, 1, 1, 0, 1, 1]), [0, 4, 9]
    out = orc.top_logprobs(x, w, ids, mask, cu, 5, 0.7)
    lp = torch.log_softmax(torch.from_numpy(x @ w.T) / 0.7, 1)
    on = mask.astype(bool)
    top = lp.topk(5)
    assert np.allclose(out["logprob"][on], lp[range(9), ids].numpy()[on]) and np.allclose(out["top_logprob"][on], top.values.numpy()[on])
    assert (out["top_ids"][on] == top.indices.numpy()[on]).all() and (out["top_ids"][~on] == -1).all() and not out["lse"][~on].any()
    assert np.allclose(out["entropy"][on], torch.distributions.Categorical(logits=lp).entropy().numpy()[on])
    assert np.allclose(out["lse"][on], torch.logsumexp(torch.from_numpy(x @ w.T) / 0.7, 1).numpy()[on])
    tie = orc.top_logprobs(np.ones((1, 2)), np.zeros((7, 2)), None, [1], [0, 1], 3)
    assert tie["top_ids"].tolist() == [[0, 1, 2]]


@pytest.mark.parametrize("rest", ["bucket", "renormalise"])
def test_oracle_loss_is_torch_kl_and_its_gradient(rest):
    x, w, ids, lp, t = _case(2)
    mask, cu, tau = np.array([1, 1, 0, 1, 1, 1, 0, 1, 1]), [0, 4, 9], 1.3
    out = orc.distill(x, w, ids, lp, mask, cu, rest, tau, "sequence", 2.0)
    X, W = torch.from_numpy(x).requires_grad_(), torch.from_numpy(w).requires_grad_()
    lq = torch.log_softmax(X @ W.T / tau, 1)
    i = torch.from_numpy(ids)
    if rest == "renormalise":
        p = torch.softmax(torch.from_numpy(lp), 1)
        kl = torch.nn.functional.kl_div(lq.gather(1, i), p, reduction="none").sum(1)
    else:
        on = torch.zeros(9, 37, dtype=torch.bool).scatter_(1, i, True)
        lp_all = torch.cat([torch.from_numpy(lp), torch.log1p(-torch.from_numpy(lp).exp().sum(1, keepdim=True))], 1)
        lq_all = torch.cat([lq.gather(1, i), torch.logsumexp(lq.masked_fill(on, -np.inf), 1, keepdim=True)], 1)
        kl = torch.nn.functional.kl_div(lq_all, lp_all, log_target=True, reduction="none").sum(1)
    on = torch.from_numpy(mask).bool()
    share = torch.tensor([1 / 6] * 4 + [1 / 8] * 5, dtype=torch.float64)
    loss = 2.0 * (kl * share)[on].sum()
    loss.backward()
    assert np.allclose(out["row_loss"], (kl * on).detach().numpy()) and np.isclose(out["loss"], loss.item())
    assert np.allclose(out["d_hidden"], X.grad.numpy()) and np.allclose(out["d_weight"], W.grad.numpy())
    assert (np.abs(out["dS"]) <= out["gross"] + 1e-15).all()


@pytest.mark.parametrize("rest", ["bucket", "renormalise"])
def test_oracle_gradient_by_differences(rest):
    x, w, ids, lp, _ = _case(3, V=11, K=4, R=3)
    ids[1, 2], ids[2, :] = -1, -1
    f = lambda x: orc.distill(x, w, ids, lp, np.ones(3), [0, 2, 3], rest, 0.8, "token")["loss"]
    g = orc.distill(x, w, ids, lp, np.ones(3), [0, 2, 3], rest, 0.8, "token")["d_hidden"]
    h = 1e-6
    for r in range(3):
        for k in range(5):
            d = np.zeros_like(x)
            d[r, k] = h
            assert abs((f(x + d) - f(x - d)) / (2 * h) - g[r, k]) < 1e-8
    assert not g[2].any()


def test_oracle_closed_forms():
    x, w, _, _, _ = _case(4)
    lq = orc._log_softmax(x @ w.T)
    order = np.argsort(-lq, 1)[:, :7]
    # a student that has the teacher's distribution has nothing to learn, whatever part of it is listed
    same = orc.distill(x, w, order, np.take_along_axis(lq, order, 1), np.ones(9), [0, 9])
    assert np.abs(same["row_loss"]).max() < 1e-12 and np.abs(same["dS"]).max() < 1e-12
    # one certain token: cross entropy
    hard = orc.distill(x, w, order[:, 3:4], np.zeros((9, 1)), np.ones(9), [0, 9], "renormalise", aggregation="token")
    assert np.allclose(hard["row_loss"], -np.take_along_axis(lq, order[:, 3:4], 1)[:, 0])
    both = orc.distill(x, w, order[:, 3:4], np.zeros((9, 1)), np.ones(9), [0, 9], "bucket", aggregation="token")
    assert np.allclose(hard["dS"], both["dS"])
    # all tokens listed: both readings are the whole divergence
    every = np.tile(np.arange(37), (9, 1))
    t = np.roll(lq, 1, axis=1)
    a, b = (orc.distill(x, w, every, t, np.ones(9), [0, 9], rest) for rest in ("bucket", "renormalise"))
    assert np.allclose(a["row_loss"], (np.exp(t) * (t - lq)).sum(1)) and np.allclose(a["dS"], b["dS"])
    # entries named again or out of range are left out; a list without any counts and has no part in it
    kept, left_out = orc.row_entries([3, -1, 3, 37, -2, 5], [-1.0] * 6, 37)
    assert [t for t, _ in kept] == [3, 5] and left_out == 3
    none = orc.distill(x, w, np.full((9, 2), -1), np.full((9, 2), np.nan), np.ones(9), [0, 9])
    assert none["loss"] == 0.0 and not none["dS"].any() and none["stats"] == dict(n_tokens=9, n_bad_entry=0, n_empty_row=9, n_bad_seq=0)
