"""Float64 CPU oracle of scoring with top alternatives and of distillation from a teacher's top entries.  Straight from the definitions in include/rl_distill.h."""
import numpy as np

from oracle.policy_oracle import compact_rows, widen


def _log_softmax(z):
    m = z.max(axis=1, keepdims=True)
    return z - m - np.log(np.exp(z - m).sum(axis=1, keepdims=True))


def top_logprobs(hidden, weight, token_ids, mask, cu_seqlens, top_k, temperature=1.0):
    """dict(logprob, lse, entropy [R], top_ids, top_logprob [R, K]); token_ids may be None (logprob is then 0)."""
    x, w = widen(hidden), widen(weight)
    R, V = x.shape[0], w.shape[0]
    ids = np.zeros(R, dtype=np.int64) if token_ids is None else np.asarray(token_ids).astype(np.int64)
    out = dict(logprob=np.zeros(R), lse=np.zeros(R), entropy=np.zeros(R), top_ids=np.full((R, top_k), -1, dtype=np.int64), top_logprob=np.zeros((R, top_k)))
    for r in compact_rows(mask, ids, cu_seqlens, V)["row_map"]:
        raw = w @ x[r]
        lp = _log_softmax(raw[None] / temperature)[0]
        out["lse"][r] = raw[0] / temperature - lp[0]
        out["logprob"][r] = 0.0 if token_ids is None else lp[ids[r]]
        out["entropy"][r] = -(np.exp(lp) * lp).sum()
        order = np.lexsort((np.arange(V), -raw))[:top_k]              # by logit, then by token
        out["top_ids"][r], out["top_logprob"][r] = order, lp[order]
    return out


def row_entries(ids, logprob, V):
    """The entries of a list that count: ([(token, log-probability)], how many were left out)."""
    kept, left_out = [], 0
    for i, l in zip(np.asarray(ids).astype(np.int64), np.asarray(logprob).astype(np.float64)):
        if i == -1:
            continue
        if i < 0 or i >= V or any(i == k for k, _ in kept):
            left_out += 1
        else:
            kept.append((int(i), float(l)))
    return kept, left_out


def row_loss(lq, entries, rest):
    """(KL_t, d KL_t / d z [V], whether there was nothing to learn) of log-probabilities lq [V] at the student's temperature."""
    q = np.exp(lq)
    tok = np.array([t for t, _ in entries], dtype=np.int64)
    lt = np.array([l for _, l in entries], dtype=np.float64)
    others = np.ones(lq.size, dtype=bool)
    others[tok] = False
    if rest == "renormalise":
        if not entries or np.all(lt == -np.inf):
            return 0.0, np.zeros_like(q), True
        p = np.exp(lt - lt.max())
        p, left = p / p.sum(), 0.0
    else:
        if not entries:
            return 0.0, np.zeros_like(q), True
        p = np.exp(lt)
        left = max(0.0, 1.0 - p.sum()) if others.any() else 0.0
    kl = sum(a * (np.log(a) - lq[t]) for a, t in zip(p, tok) if a > 0)
    d = q * (p.sum() + left)
    np.subtract.at(d, tok, p)
    if left > 0:
        m = lq[others].max()
        lrest = m + np.log(np.exp(lq[others] - m).sum())
        kl += left * (np.log(left) - lrest)
        d[others] -= left * np.exp(lq[others] - lrest)
    return kl, d, False


def distill(hidden, weight, teacher_ids, teacher_logprob, mask, cu_seqlens, rest="bucket", temperature=1.0, aggregation="sequence", scale=1.0):
    """dict(loss, row_loss, lse [R], dS [R, V], gross [R, V] (the magnitudes that a dS is the difference of), d_hidden, d_weight, stats)."""
    x, w = widen(hidden), widen(weight)
    R, V = x.shape[0], w.shape[0]
    c = compact_rows(mask, np.zeros(R, dtype=np.int64), cu_seqlens, V)
    rows, lens = c["row_map"], c["seq_len"]
    B = len(lens)
    share = np.full(R, 1.0 / max(1, len(rows))) if aggregation == "token" else np.zeros(R)
    if aggregation == "sequence":
        share[rows] = np.repeat(1.0 / (B * np.maximum(1, lens)), lens)
    out = dict(loss=0.0, row_loss=np.zeros(R), lse=np.zeros(R), dS=np.zeros((R, V)), gross=np.zeros((R, V)))
    n_bad = n_empty = 0
    for r in rows:
        z = w @ x[r] / temperature
        lq = _log_softmax(z[None])[0]
        out["lse"][r] = z[0] - lq[0]
        entries, left_out = row_entries(teacher_ids[r], teacher_logprob[r], V)
        kl, d, nothing = row_loss(lq, entries, rest)
        n_bad += left_out
        n_empty += nothing
        out["row_loss"][r] = kl
        out["loss"] += scale * share[r] * kl
        f = scale * share[r] / temperature
        out["dS"][r] = f * d
        out["gross"][r] = abs(f) * (np.abs(d) + (0 if nothing else 2 * np.exp(lq)))
    out["d_hidden"], out["d_weight"] = out["dS"] @ w, out["dS"].T @ x
    out["stats"] = dict(n_tokens=len(rows), n_bad_entry=n_bad, n_empty_row=n_empty, n_bad_seq=c["n_bad_seq"])
    return out
