"""What the norm, the 8-bit checkpoints and the 8-bit linear layer in front of the LM head are timed on, with their plain forms.

Kinds of case
  norm    layer norm: the forward pass alone (serving), or forward and backward (training), the backward from x itself or from the
          8-bit checkpoint that the forward wrote beside its output
  rows    an activation packed into 8-bit rows in the forward pass and restored in the backward
  linear  the linear layer on 8-bit operands, forward only: rows are packed and multiplied with a packed weight
  step    the layer's training step: output, then input gradient and weight gradient from the packed input

8-bit rows: codes [rows, columns rounded up to 128] and, for every 128 columns of a row, a scale that is a power of two, the smallest
under which the block's largest finite magnitude is representable (1 for a block of zeros).  A weight has one scale for 128 x 128 values."""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": 9, "e5m2": 16}                       # the largest value is 0.875 * 2**TOP


# ------------------------------------------------------------------ the cases
def _norm(name, R, H, dtype, mode, params="f32", pad=0, fmt="e4m3"):
    return dict(name=name, kind="norm", R=R, H=H, dtype=dtype, mode=mode, params=params, pad=pad, fmt=fmt)


def _lin(name, kind, M, N, K, dtype, pad=0, fmt="e4m3", grad_fmt="e5m2"):
    return dict(name=name, kind=kind, M=M, N=N, K=K, dtype=dtype, pad=pad, fmt=fmt, grad_fmt=grad_fmt)


def listed():
    return [
        # the smallest call: the final norm of one token in a decode step; latency only
        _norm("norm_token", 1, 4096, "bf16", "forward", params="bf16"),
        # a small model trained in f32 (the width of the f32 loss cases), a batch of some thousand rows
        _norm("norm_train_f32", 2175, 768, "f32", "train"),
        # a micro-batch of rollouts at the 7B width, x kept as it is for the backward pass
        _norm("norm_train_7b", 32768, 3584, "bf16", "train"),
        # the same with x kept in 8 bits: an odd number of rows
        _norm("norm_ckpt_7b", 32749, 3584, "bf16", "checkpoint"),
        # rows of an odd width inside a wider buffer, as after slicing a concatenated state
        _norm("norm_ckpt_odd", 5003, 1157, "bf16", "checkpoint", params="bf16", pad=6),
        # the activations of a batch at the 32B width, packed in the forward and restored in the backward pass
        _lin("rows_32b", "rows", 16381, 0, 5120, "bf16"),
        # a short f32 batch of the small model, packed and restored
        _lin("rows_f32", "rows", 1201, 0, 768, "f32", fmt="e5m2"),
        # serving: one token through the projection in front of the head
        _lin("linear_token", "linear", 1, 3584, 3584, "bf16"),
        # serving: a decode step of 48 sequences through a projection that widens
        _lin("linear_decode_48", "linear", 48, 14336, 3584, "bf16"),
        # the forward pass over a batch of rollouts at the 7B width
        _lin("linear_7b", "linear", 32768, 3584, 3584, "bf16"),
        # the training step of a small layer of odd sizes in f32
        _lin("step_odd_f32", "step", 3001, 1157, 1163, "f32"),
        # the largest: the training step over a batch of rollouts at the 7B width
        _lin("step_7b", "step", 32749, 3584, 3584, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm", "rows", "linear", "linear", "step", "step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, 0, 8, 3])
    fmt = rng.choice(["e4m3", "e4m3", "e5m2"])
    if kind == "norm":
        H = rng.choice([3584, 2048, 4096, 5120, _log(rng, 16, 12000)])
        return dict(kind=kind, R=_log(rng, 1, max(2, min(40000, 120_000_000 // H))), H=H, dtype=dtype, mode=rng.choice(["forward", "train", "checkpoint"]),
                    params=rng.choice(["f32", dtype]), pad=pad, fmt=fmt)
    K, N = (rng.choice([3584, 2048, 4096, 5120, _log(rng, 32, 6000)]) for _ in range(2))
    M = _log(rng, 1, 34000)
    while M * K > 120_000_000 or M * N > 120_000_000 or M * N * K > 4.0e11:
        M = M * 3 // 4
    return dict(kind=kind, M=M, N=0 if kind == "rows" else N, K=K, dtype=dtype, pad=pad, fmt=fmt, grad_fmt=rng.choice(["e5m2", "e5m2", "e4m3"]))


# ------------------------------------------------------------------ inputs
def _scales(amax, fmt):
    """Exponent of each block's scale, from the largest finite magnitude in it."""
    m, e = torch.frexp(amax)
    e = (e - TOP[fmt] + (m > 0.875).int()).clamp(-127, 127)
    return torch.where(amax > 0, e, torch.zeros_like(e))


def _pow2(e):
    """2**e in f32, exactly."""
    return ((e.int().clamp(-126, 127) + 127) << 23).view(torch.float32)


def _round_rows(x, fmt):
    """x rounded to 8-bit rows and back, in f32."""
    R, K = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -K % 128)).view(R, -1, 128)
    a = b.abs()
    e = _scales(torch.where(torch.isfinite(a), a, torch.zeros_like(a)).amax(2), fmt)[..., None]
    v = (b * _pow2(-e)).to(FORMATS[fmt]).float() * _pow2(e)
    return v.view(R, -1)[:, :K]


def _packed_weight(w, fmt):
    """A weight [N, K] in 8-bit rows: (codes [N, Kp], scales [N, Ks]) and the same of its transpose; a scale for 128 x 128 values."""
    N, K = w.shape
    b = torch.nn.functional.pad(w, (0, -K % 128, 0, -N % 128))
    b = b.view(b.shape[0] // 128, 128, b.shape[1] // 128, 128)
    e = _scales(b.abs().amax((1, 3)), fmt)
    codes = (b * _pow2(-e[:, None, :, None])).to(FORMATS[fmt]).view(torch.uint8).view(b.shape[0] * 128, -1)

    def one(codes, e, rows):
        s = torch.full((e.shape[0], -(-e.shape[1] // 4) * 4), 127, dtype=torch.uint8, device=DEV)
        s[:, :e.shape[1]] = (e + 127).to(torch.uint8)
        return codes[:rows].contiguous(), s.repeat_interleave(128, 0)[:rows].contiguous()
    return one(codes, e, N) + one(codes.t(), e.t(), K)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device=DEV)
    u = lambda *s: torch.rand(*s, generator=g, device=DEV)
    dt, pad = DTYPES[case["dtype"]], case["pad"]
    R, H = (case["R"], case["H"]) if case["kind"] == "norm" else (case["M"], case["K"])

    def rows(cols, make):
        """Rows of a buffer that is `pad` columns wider."""
        t = torch.zeros(R, cols + pad, dtype=dt, device=DEV)
        t[:, :cols] = make.to(dt)
        return t[:, :cols]

    def gradient(cols):
        """Tokens that do not count have no gradient; the others' sizes differ."""
        return rows(cols, 1e-3 * n(R, cols) * torch.exp(n(R, 1)) * ((u(R, 1) < 0.8) | (R < 20)))

    # a residual stream: a few wide channels, an offset for each, padding rows of zeros
    x = rows(H, (n(R, H) * (1 + 20 * (u(H) < 0.01)) + 0.2 * n(H)) * ((u(R, 1) < 0.95) | (R < 20)))
    s = dict(case=case, x=x)
    if case["kind"] == "norm":
        p = DTYPES[case["params"]]
        s["gamma"], s["beta"] = (1 + 0.2 * n(H)).to(p), (0.1 * n(H)).to(p)
        if case["mode"] != "forward":
            s["dy"] = gradient(H)
    elif case["kind"] != "rows":
        s["w"], s["w_scales"], s["wt"], s["wt_scales"] = _packed_weight(n(case["N"], H) / math.sqrt(H), "e4m3")
        if case["kind"] == "step":
            s["dy"] = gradient(case["N"])
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2603_16435_amd import binding as b
    case, x = s["case"], s["x"]
    if case["kind"] == "norm":
        kept = case["fmt"] if case["mode"] == "checkpoint" else None
        y, stats, ckpt = b.rl_layer_norm_forward(x, s["gamma"], s["beta"], eps=EPS, checkpoint=kept)
        if case["mode"] == "forward":
            return dict(y=y)
        dx, dgamma, dbeta = b.rl_layer_norm_backward(s["dy"], ckpt if kept else x, stats, s["gamma"])
        return dict(y=y, dx=dx, dgamma=dgamma, dbeta=dbeta)
    if case["kind"] == "rows":
        return dict(restored=b.rl_f8_unpack(b.rl_f8_pack(x, case["fmt"]), x.dtype))
    w = b.F8Weight(b.F8Rows(s["w"], s["w_scales"], case["K"], "e4m3"), b.F8Rows(s["wt"], s["wt_scales"], case["N"], "e4m3"))
    y, kept = b.rl_f8_linear_forward(x, w, fmt=case["fmt"], keep=case["kind"] == "step")
    if case["kind"] == "linear":
        return dict(y=y)
    dx, dw = b.rl_f8_linear_backward(s["dy"], kept, w, fmt=case["grad_fmt"])
    return dict(y=y, dx=dx, dw=dw)


def _run_plain(s):
    case, x = s["case"], s["x"]
    dt = x.dtype
    if case["kind"] == "norm":
        xf, gamma, beta = x.float(), s["gamma"].float(), s["beta"].float()
        mean = xf.mean(1, keepdim=True)
        xc = xf - mean
        rstd = torch.rsqrt((xc * xc).mean(1, keepdim=True) + EPS)
        y = (xc * rstd * gamma + beta).to(dt)
        if case["mode"] == "forward":
            return dict(y=y)
        if case["mode"] == "checkpoint":
            xc = _round_rows(x, case["fmt"]) - mean
        xh, dy = xc * rstd, s["dy"].float()
        g = dy * gamma
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return dict(y=y, dx=dx.to(dt), dgamma=(dy * xh).sum(0), dbeta=dy.sum(0))
    x8 = _round_rows(x, case["fmt"])
    if case["kind"] == "rows":
        return dict(restored=x8.to(dt))
    N, K = case["N"], case["K"]
    e = s["w_scales"][:, :-(-K // 128)].int() - 127
    w = (s["w"].view(torch.float8_e4m3fn).float().view(N, -1, 128) * _pow2(e)[..., None]).view(N, -1)[:, :K]
    y = (x8 @ w.t()).to(dt)
    if case["kind"] == "linear":
        return dict(y=y)
    return dict(y=y, dx=(_round_rows(s["dy"], case["grad_fmt"]) @ w).to(dt), dw=s["dy"].float().t() @ x8)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        n = case["R"] * case["H"]
        passes = {"forward": 2 * e, "train": 5 * e, "checkpoint": 4 * e + 2}[case["mode"]]     # checkpoint: codes written and read instead of x again
        return dict(bytes=passes * n, flops=(8 if case["mode"] == "forward" else 24) * n)
    M, N, K = case["M"], case["N"], case["K"]
    if case["kind"] == "rows":
        return dict(bytes=(2 * e + 2) * M * K, flops=4 * M * K)
    if case["kind"] == "linear":
        return dict(bytes=e * M * K + N * K + e * M * N, flops=2 * M * N * K)
    # x, W both ways, y; dy, dx, the packed input written and read, dW
    return dict(bytes=2 * e * M * K + 2 * M * K + 2 * N * K + 2 * e * M * N + 4 * N * K, flops=6 * M * N * K)


# ------------------------------------------------------------------ the definition, in 64 bits
def _values(fmt):
    """The non-negative finite values of a format by code, from its bits."""
    man, bias, codes = (3, 7, 127) if fmt == "e4m3" else (2, 15, 124)
    v = [(c & ((1 << man) - 1)) * 2.0 ** (1 - bias - man) if c >> man == 0 else
         (1 + (c & ((1 << man) - 1)) / (1 << man)) * 2.0 ** ((c >> man) - bias) for c in range(codes)]
    return torch.tensor(v, dtype=torch.float64, device=DEV)


def _exp2(e):
    """2**e in 64 bits for whole e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(x, fmt):
    """Finite x in 64 bits to the nearest value of its block's scale, ties to the even code."""
    t = _values(fmt)
    mid = (t[1:] + t[:-1]) / 2
    out = torch.empty_like(x)
    for k in range(0, x.shape[1], 128):
        b = x[:, k:k + 128]
        a = b.abs().amax(1, keepdim=True)
        s = torch.ones_like(a)
        up = a > 0
        s[up] = _exp2(torch.ceil(torch.log2(a[up] / t[-1])).clamp(-127, 127))
        s = torch.where(s * t[-1] < a, 2 * s, torch.where(up & (s / 2 * t[-1] >= a) & (s > 2.0 ** -127), s / 2, s))       # log2 next to a whole number
        v = b.abs() / s
        i = torch.bucketize(v.contiguous(), mid)
        j = i.clamp(max=mid.numel() - 1)
        i = i + ((v == mid[j]) & (i % 2 == 1)).long()
        out[:, k:k + 128] = torch.copysign(t[i] * s, b)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["kind"] == "norm":
        gamma, beta, H = s["gamma"].double(), s["beta"].double(), x.shape[1]
        mu = x.sum(1, keepdim=True) / H
        r = 1 / torch.sqrt(((x - mu) ** 2).sum(1, keepdim=True) / H + EPS)
        y = (x - mu) * r * gamma + beta
        if case["mode"] == "forward":
            return dict(y=y)
        xh = ((_nearest(x, case["fmt"]) if case["mode"] == "checkpoint" else x) - mu) * r
        dy = s["dy"].double()
        a, b = (dy @ gamma)[:, None] / H, ((dy * xh) @ gamma)[:, None] / H
        return dict(y=y, dx=(dy * gamma - a - xh * b) * r, dgamma=torch.einsum("rh,rh->h", dy, xh), dbeta=dy.sum(0))
    x8 = _nearest(x, case["fmt"])
    if case["kind"] == "rows":
        return dict(restored=x8)
    t = _values("e4m3")
    c = s["w"][:, :case["K"]].long()
    w = torch.where(c >= 128, -1.0, 1.0) * t[c & 127]
    k = torch.arange(case["K"], device=DEV) // 128
    w = w * _exp2(s["w_scales"].double() - 127)[:, k]
    if case["kind"] == "linear":
        return dict(y=x8 @ w.t())
    dy = s["dy"].double()
    return dict(y=x8 @ w.t(), dx=_nearest(dy, case["grad_fmt"]) @ w, dw=dy.t() @ x8)
