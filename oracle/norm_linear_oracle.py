"""Float64 CPU oracle of the layers in front of the LM head: 8-bit rows, layer norm, linear layer.  Straight from the definitions."""
import numpy as np

MAN, BIAS, CODES = {"e4m3": 3, "e5m2": 2}, {"e4m3": 7, "e5m2": 15}, {"e4m3": 127, "e5m2": 124}     # codes below this are finite


def values(fmt):
    """The finite non-negative values of a format, by code."""
    m, out = MAN[fmt], []
    for c in range(CODES[fmt]):
        e, f = c >> m, c & ((1 << m) - 1)
        out.append(f * 2.0 ** (1 - BIAS[fmt] - m) if e == 0 else (1 + f / 2.0 ** m) * 2.0 ** (e - BIAS[fmt]))
    return np.array(out)


def scale_exponent(amax, fmt):
    """Smallest e >= -127 with amax <= largest * 2^e; 0 for amax = 0."""
    if amax == 0:
        return 0
    top, e = values(fmt)[-1], -127
    while top * 2.0 ** e < amax:
        e += 1
    return e


def round_block(b, fmt, e=None):
    """Values of one block (any shape) after packing and restoring, and the scale's exponent."""
    finite = np.isfinite(b)
    if e is None:
        e = scale_exponent(np.abs(np.where(finite, b, 0.0)).max(initial=0.0), fmt)
    t = values(fmt)
    v = np.abs(np.where(finite, b, 0.0)) / 2.0 ** e
    i = np.clip(np.searchsorted(t, v), 1, len(t) - 1)                    # t[i-1] < v <= t[i], or v = 0
    lo, hi = v - t[i - 1], t[i] - v
    code = np.where((lo < hi) | ((lo == hi) & (i % 2 == 1)), i - 1, i)   # ties to the even code
    most = t[t * 2.0 ** e <= np.finfo(np.float32).max][-1]               # a restored value is one of f32
    out = np.copysign(np.minimum(t[code], most) * 2.0 ** e, b)
    bad = np.where(np.isinf(b) & (fmt == "e5m2"), b, np.nan)
    return np.where(finite, out, bad), e


def round_rows(x, fmt):
    """x [R, K] packed into 8-bit rows and restored; exponents [R, blocks]."""
    R, K = x.shape
    out, nb = np.empty((R, K)), -(-K // 128)
    es = np.zeros((R, nb), dtype=np.int64)
    for r in range(R):
        for b in range(nb):
            out[r, b * 128:(b + 1) * 128], es[r, b] = round_block(x[r, b * 128:(b + 1) * 128], fmt)
    return out, es


def round_weight(w, fmt):
    """w [N, K] with one scale for 128 x 128 values."""
    out = np.empty_like(w)
    for n in range(0, w.shape[0], 128):
        for k in range(0, w.shape[1], 128):
            out[n:n + 128, k:k + 128], _ = round_block(w[n:n + 128, k:k + 128], fmt)
    return out


def norm_forward(x, gamma, beta, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + (0 if beta is None else beta), mean, rstd


def norm_backward(dy, x, mean, rstd, gamma):
    """x: what the backward pass reads, mean and rstd: of the forward pass."""
    xh, g = (x - mean) * rstd, dy * gamma
    dx = rstd * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)
