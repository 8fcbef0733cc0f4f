"""What scoring with top alternatives and distillation from a teacher's top entries are timed on, with their plain forms.

Kinds of case
  score    log-probability of a given token, logsumexp, entropy and the K most probable tokens with their log-probabilities, out of hidden
           states and the LM head's weight; ties go to the lowest token
  distill  Kullback-Leibler divergence from a teacher, of whom each token has up to K entries (token, log-probability), to the student
           softmax(W x / temperature): loss, divergence of each row and, in training, the gradients of hidden states and weight

rest = "bucket": what the teacher's entries leave of its probability is one entry that stands for all other tokens; "renormalise": the entries
are the teacher's whole distribution.  Lists shorter than K end in tokens -1, and some are empty."""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ the cases
def _score(name, R, H, V, dtype, K, B=1, padded=False, temperature=1.0):
    return dict(name=name, kind="score", R=R, H=H, V=V, dtype=dtype, K=K, B=B, padded=padded, temperature=temperature)


def _distill(name, R, H, V, dtype, K, B=1, padded=False, temperature=1.0, rest="bucket", aggregation="token", train=True):
    return dict(name=name, kind="distill", R=R, H=H, V=V, dtype=dtype, K=K, B=B, padded=padded, temperature=temperature, rest=rest,
                aggregation=aggregation, train=train)


def listed():
    return [
        # the smallest call: a decode step of 48 sequences on a small vocabulary, five alternatives each; latency
        _score("score_decode_48", 48, 2048, 32000, "bf16", 5, temperature=0.7),
        # one token of one sequence at the 7B head: the weight read once
        _score("score_token_7b", 1, 3584, 152064, "bf16", 20),
        # rollouts scored under a reference model, padded to the longest, with the alternatives that a log of them shows
        _score("score_rollouts_7b", 10240, 3584, 152064, "bf16", 20, B=16, padded=True),
        # a teacher that writes the lists a student learns from, at the 32B width
        _score("score_teacher_32b", 4099, 5120, 151936, "bf16", 128, B=9),
        # a small f32 model, an odd number of rows, a width off the grid of the matrix tiles
        _score("score_odd_f32", 1201, 764, 50257, "f32", 11, B=5, temperature=1.3),
        # a few tokens learnt from at a time: the smallest training step
        _distill("distill_few", 61, 2048, 32000, "bf16", 8, B=3, rest="renormalise", aggregation="sequence"),
        # the small f32 model as a student
        _distill("distill_f32", 1100, 768, 50257, "f32", 32, B=7, aggregation="sequence"),
        # odd sizes: rows, vocabulary and entries off every grid, a temperature above one
        _distill("distill_odd", 2999, 1160, 50257, "bf16", 100, B=11, padded=True, temperature=2.0, rest="renormalise"),
        # the loss alone, on held-out text
        _distill("distill_eval_7b", 3001, 3584, 152064, "bf16", 20, B=4, aggregation="sequence", train=False),
        # a micro-batch of padded rollouts at the 7B head
        _distill("distill_7b", 8192, 3584, 152064, "bf16", 64, B=16, padded=True, aggregation="sequence"),
        # the 32B width, long lists
        _distill("distill_32b", 4099, 5120, 151936, "bf16", 128, B=3),
        # the largest: a batch of packed rollouts at the 7B head
        _distill("distill_large_7b", 20011, 3584, 152064, "bf16", 50, B=24, temperature=1.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["score", "distill"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    H = rng.choice([3584, 5120, 2048, 768, 8 * _log(rng, 8, 640), 8 * _log(rng, 8, 640)])
    V = rng.choice([152064, 151936, 50257, 32000, _log(rng, 300, 152064), _log(rng, 300, 152064)])
    R = _log(rng, 1, 20000)
    most = 2.0e12 if dtype == "f32" else 8.0e12                 # (R V H: a step of 6 of them is a third of a second in f32)
    while R * V * H > most:
        R = R * 3 // 4
    case = dict(kind=kind, R=R, H=H, V=V, dtype=dtype, K=_log(rng, 1, 128), B=_log(rng, 1, min(R, 64)), padded=rng.choice([False, False, True]),
                temperature=rng.choice([1.0, 1.0, 0.7, 2.0, round(rng.uniform(0.5, 3.0), 3)]))
    if kind == "distill":
        case.update(rest=rng.choice(["bucket", "bucket", "renormalise"]), aggregation=rng.choice(["sequence", "token"]), train=rng.random() < 0.8)
    return case


# ------------------------------------------------------------------ inputs
def _layout(case):
    """Offsets of the sequences and how many rows of each count: padded ones have lengths of their own in rows of one size."""
    R, B = case["R"], case["B"]
    cu = [R * i // B for i in range(B + 1)]
    if not case["padded"]:
        return cu, [b - a for a, b in zip(cu, cu[1:])]
    return cu, [math.ceil((b - a) * (0.1 + 0.9 * (0.618034 * (i + 1) % 1.0))) for i, (a, b) in enumerate(zip(cu, cu[1:]))]


def _grid(x, step, most):
    return (x / step).round().clamp(-most, most) * step


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    u = lambda *s: torch.rand(*s, generator=g, device=DEV)
    dt, R, H, V, K = DTYPES[case["dtype"]], case["R"], case["H"], case["V"], case["K"]
    cu, count = _layout(case)
    i32 = dict(dtype=torch.int32, device=DEV)
    starts, counts = torch.tensor(cu, **i32), torch.tensor(count, **i32)
    seq = torch.repeat_interleave(torch.arange(case["B"], device=DEV), starts.diff().long())
    at = torch.arange(R, device=DEV) - starts[:-1][seq]
    ids = (u(R) * V).long().clamp(max=V - 1)
    # logits of a trained model: a spread of about one, and on many rows a token that stands out
    spread = 1.2 / math.sqrt(H)
    w = spread * n(V, H)
    if case["kind"] == "score":
        # weights and states as a quantised model has them, in steps of a power of two: their products add up without rounding, in any
        # order, so that the order of the alternatives is the same for everybody
        w = _grid(w, 2.0 ** round(math.log2(spread / 10)), 31)
    w = w.to(dt)
    x = n(R, H) + (20 * u(R, 1) * (u(R, 1) < 0.7)) * w[ids].float() / 1.44
    s = dict(case=case, weight=w, cu=starts, mask=(at < counts[seq]).to(torch.uint8))
    if case["kind"] == "score":
        pick = u(R) < 0.5                                       # the token that was sampled is not always the one that stands out
        s["ids"] = torch.where(pick, ids, (u(R) * V).long().clamp(max=V - 1)).int()
        s["hidden"] = _grid(x, 1 / 16, 127).to(dt)
        return s
    s["hidden"] = x.to(dt)
    t = (x + 1.6 * n(R, H)).to(dt)                              # the teacher's states at the same tokens
    s["ids"], s["logprob"] = torch.empty(R, K, **i32), torch.empty(R, K, device=DEV)
    for a in range(0, R, 2048):
        z = (t[a:a + 2048] @ w.t()).float() / case["temperature"]
        top = z.topk(K)
        s["ids"][a:a + 2048], s["logprob"][a:a + 2048] = top.indices.int(), top.values - torch.logsumexp(z, 1, keepdim=True)
    have = torch.where(u(R) < 0.2, (u(R) * (K + 1)).long(), torch.full((R,), K, device=DEV))      # lists cut short
    gone = torch.arange(K, device=DEV)[None] >= have[:, None]
    s["ids"][gone], s["logprob"][gone] = -1, 0.0
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2603_16435_amd import binding as b
    case = s["case"]
    if case["kind"] == "score":
        r = b.rl_token_top_logprobs(s["hidden"], s["weight"], s["ids"], s["mask"], case["K"], temperature=case["temperature"], cu_seqlens=s["cu"])
        return dict(logprob=r.logprob, lse=r.lse, entropy=r.entropy, top_ids=r.top_ids, top_logprob=r.top_logprob)
    r = b.rl_distill_loss_fwd_bwd(s["hidden"], s["weight"], s["ids"], s["logprob"], s["mask"], s["cu"], rest=case["rest"],
                                  temperature=case["temperature"], aggregation=case["aggregation"], backward=case["train"],
                                  d_weight_dtype=s["weight"].dtype)
    out = dict(loss=r.loss, row_loss=r.row_loss, lse=r.lse)
    return dict(out, d_hidden=r.d_hidden, d_weight=r.d_weight) if case["train"] else out


def _coefficients(s, rows):
    """What each counting row's divergence is multiplied with in the loss."""
    case = s["case"]
    if case["aggregation"] == "token":
        return torch.full((rows.numel(),), 1.0 / max(1, rows.numel()), dtype=torch.float64, device=DEV)
    seq = torch.bucketize(rows, s["cu"][1:].long(), right=True)
    return 1.0 / (case["B"] * torch.bincount(seq, minlength=case["B"])[seq].double())


def _run_plain(s):
    case, mask = s["case"], s["mask"]
    R, V, K, tau = case["R"], case["V"], case["K"], case["temperature"]
    rows = mask.nonzero()[:, 0]
    x, w = s["hidden"][rows].float(), s["weight"].float()
    z = x @ w.t()
    full = lambda v, fill=0: torch.full((R,) + v.shape[1:], fill, dtype=v.dtype, device=DEV).index_copy_(0, rows, v)
    if case["kind"] == "score":
        bits = (z + 0.0).view(torch.int32)                      # (-0 counts as 0)
        key = ((bits ^ (bits >> 31 & 0x7fffffff)).long() << 32) + (0x7fffffff - torch.arange(V, device=DEV))
        top = 0x7fffffff - (key.topk(K, 1).values & 0xffffffff)
        del bits, key
    z /= tau
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lse = m.double() + torch.log(total.double())
    if case["kind"] == "score":
        ent = torch.log(total) - (e * (z - m)).sum(1, keepdim=True) / total
        lp = z.gather(1, s["ids"][rows].long()[:, None]) - lse
        ids, tlp = top.int(), z.gather(1, top) - lse
        return dict(logprob=full(lp[:, 0].float()), lse=full(lse[:, 0].float()), entropy=full(ent[:, 0]), top_ids=full(ids, -1), top_logprob=full(tlp.float()))
    ids, lt = s["ids"][rows].long(), s["logprob"][rows].double()
    there = ids >= 0
    at = torch.where(there, ids, V)
    p = torch.where(there, torch.exp(lt), 0.0)
    if case["rest"] == "renormalise":
        p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
        left = torch.zeros(rows.numel(), 1, dtype=torch.float64, device=DEV)
    else:
        left = (1 - p.sum(1, keepdim=True)).clamp(min=0)
    listed_ = torch.zeros(rows.numel(), V + 1, dtype=torch.bool, device=DEV).scatter_(1, at, True)[:, :V]
    rest = torch.where(listed_, 0.0, e).sum(1, keepdim=True)
    left = torch.where(rest > 0, left, 0.0)
    lrest = m.double() + torch.log(rest.double())
    lq = torch.where(there, z.gather(1, at.clamp(max=V - 1)) - lse, 0.0)
    kl = torch.where(p > 0, p * (torch.log(p) - lq), 0.0).sum(1) + torch.where(left > 0, left * (torch.log(left) - (lrest - lse)), 0.0)[:, 0]
    c = _coefficients(s, rows)
    out = dict(loss=(c * kl).sum()[None].float(), row_loss=full(kl.float()), lse=full(lse[:, 0].float()))
    if not case["train"]:
        return out
    del e
    whole = (p.sum(1, keepdim=True) + left).float()
    d = torch.exp(z - lse.float()) * whole
    d -= torch.where(listed_ | (left <= 0), 0.0, torch.exp(z - lrest.float()) * left.float())
    d = torch.nn.functional.pad(d, (0, 1)).scatter_add_(1, at, -p.float())[:, :V] * (c / tau).float()[:, None]
    return dict(out, d_hidden=full((d @ w).to(s["hidden"].dtype)), d_weight=(d.t() @ x).to(s["weight"].dtype))


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    T, R, H, V, K = sum(_layout(case)[1]), case["R"], case["H"], case["V"], case["K"]
    once = e * T * H + e * V * H + R + 4 * (case["B"] + 1)      # hidden states of the rows that count, the weight, mask and offsets
    if case["kind"] == "score":
        return dict(bytes=once + 4 * T + 12 * R + 8 * R * K, flops=2 * T * V * H)
    if not case["train"]:
        return dict(bytes=once + 8 * T * K + 8 * R, flops=2 * T * V * H)
    return dict(bytes=once + 8 * T * K + 8 * R + e * R * H + e * V * H, flops=6 * T * V * H)


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    R, V, K, tau, train = case["R"], case["V"], case["K"], case["temperature"], case.get("train", False)
    f64 = dict(dtype=torch.float64, device=DEV)
    w = s["weight"].double()
    mask = s["mask"].bool()
    rows = torch.arange(R, device=DEV)[mask]
    if case["kind"] == "score":
        out = dict(logprob=torch.zeros(R, **f64), lse=torch.zeros(R, **f64), entropy=torch.zeros(R, **f64),
                   top_ids=torch.full((R, K), -1, dtype=torch.int32, device=DEV), top_logprob=torch.zeros(R, K, **f64))
    else:
        out = dict(loss=torch.zeros(1, **f64), row_loss=torch.zeros(R, **f64), lse=torch.zeros(R, **f64))
        if train:
            out.update(d_hidden=torch.zeros(R, case["H"], **f64), d_weight=torch.zeros(V, case["H"], **f64))
        cu = s["cu"].long()
        share = torch.zeros(R, **f64)
        for a, b in zip(cu[:-1].tolist(), cu[1:].tolist()):
            share[a:b] = 1.0 / (case["B"] * max(1, int(mask[a:b].sum())))
        if case["aggregation"] == "token":
            share[:] = 1.0 / max(1, rows.numel())
    for r in torch.split(rows, max(1, 250_000_000 // V)):
        x = s["hidden"][r].double()
        raw = torch.mm(x, w.t())
        z = raw / tau
        lq = torch.log_softmax(z, 1)
        q = lq.exp()
        out["lse"][r] = torch.logsumexp(z, 1)
        if case["kind"] == "score":
            out["logprob"][r] = lq[torch.arange(r.numel(), device=DEV), s["ids"][r].long()]
            out["entropy"][r] = -(q * lq).sum(1)
            order = torch.sort(raw, dim=1, descending=True, stable=True).indices[:, :K] if V <= 4096 else _largest(raw, K)
            out["top_ids"][r] = order.int()
            out["top_logprob"][r] = torch.take_along_dim(lq, order, 1)
            continue
        target = torch.zeros_like(q)                            # the teacher's distribution, spread over the vocabulary
        ids, t = s["ids"][r].long(), s["logprob"][r].double()
        known = torch.zeros_like(q)
        i, j = torch.nonzero(ids >= 0, as_tuple=True)
        target[i, ids[i, j]] = torch.exp(t[i, j])
        known[i, ids[i, j]] = 1.0
        mass = target.sum(1, keepdim=True)
        if case["rest"] == "renormalise":
            target /= torch.where(mass > 0, mass, 1.0)
        else:                                                   # what is left lies on the others as the student has it
            left = (1 - mass).clamp(min=0)
            others = ((1 - known) * q).sum(1, keepdim=True)
            target += torch.where(others > 0, left * (1 - known) * q / others, torch.zeros_like(q))
        kl = torch.where(target > 0, target * (torch.log(target) - lq), torch.zeros_like(q)).sum(1)
        out["row_loss"][r] = kl
        out["loss"] += (share[r] * kl).sum()
        if train:
            d = (q * target.sum(1, keepdim=True) - target) * (share[r] / tau)[:, None]
            out["d_hidden"][r] = torch.mm(d, w)
            out["d_weight"] += torch.mm(d.t(), x)
    return out


def _largest(raw, k):
    """The k largest of each row in order, ties by index: those above the k-th value, and the first of its equals."""
    kth = raw.topk(k, 1).values[:, -1:]
    above, equal = raw > kth, raw == kth
    short = k - above.sum(1, keepdim=True)
    taken = above | (equal & (equal.long().cumsum(1) <= short))
    ids = torch.nonzero(taken)[:, 1].view(-1, k)
    return torch.take_along_dim(ids, torch.sort(torch.take_along_dim(raw, ids, 1), dim=1, descending=True, stable=True).indices, 1)
