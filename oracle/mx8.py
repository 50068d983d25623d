"""Microscaled 8-bit rows, the root-mean-square norm, tables of rows and the
verification of drafted tokens, in float64.

Plain restatements used by the tests: E4M3 codes with one E8M0 scale for every 32
coordinates (rows padded to 128), the norm's gradient, the gradient of a table's
lookup, and the rule by which drafted tokens stand or fall.
"""

import numpy as np


def _levels():
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, np.ldexp(m / 8.0, -6), np.ldexp(1 + m / 8.0, e - 7))


E4M3 = _levels()                                  # of codes 0 .. 126, ascending
_BORDERS = (E4M3[1:] + E4M3[:-1]) / 2             # exact in float64


def e4m3(v):
    """Codes of the values v (float64, |v| <= 448): nearest, ties to the even code;
    bit 7 the sign (a zero of either sign has code 0)."""
    v = np.asarray(v, dtype=np.float64)
    low = np.searchsorted(_BORDERS, np.abs(v), side="left")     # a tie stays with the lower code
    high = np.searchsorted(_BORDERS, np.abs(v), side="right")   # or goes to the upper
    return (np.where(low % 2 == 0, low, high) + 128 * (v < 0)).astype(np.uint8)


def quantize(x):
    """Codes (n x dim) and scales (n x ceil(dim / 32)) of the rows of x."""
    x = np.asarray(x, dtype=np.float64)
    n, dim = x.shape
    nb = -(-dim // 32)
    p = np.zeros((n, nb * 32))
    p[:, :dim] = x
    p = p.reshape(n, nb, 32)
    bad = ~np.isfinite(p).all(-1)
    top = np.where(bad, 1.0, np.abs(np.where(np.isfinite(p), p, 0.0)).max(-1))
    f, e = np.frexp(top)          # top = f 2^e, 1/2 <= f < 1; 448 = 7/8 2^9
    s = np.where(top > 0, np.maximum(e - 9 + (f > 0.875) + 127, 0), 0)
    with np.errstate(invalid="ignore"):
        c = e4m3(np.where(bad[..., None], 0.0, p / np.ldexp(1.0, s - 127)[..., None]))
    return c.reshape(n, nb * 32)[:, :dim], np.where(bad, 255, s).astype(np.uint8)


def pack(codes, scales, dim):
    """The stored form: n x 128 steps bytes of codes and n x 4 steps scales."""
    n, steps = codes.shape[0], -(-dim // 128)
    c = np.zeros((n, 128 * steps), dtype=np.uint8)
    c[:, :dim] = codes
    s = np.zeros((n, 4 * steps), dtype=np.uint8)
    s[:, :scales.shape[1]] = scales
    return c, s


def values(codes, scales, dim):
    """float64 values of the stored form."""
    n = codes.shape[0]
    level = np.concatenate([E4M3, [np.nan]])
    v = level[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(n, -1, 32) * scale[..., None]).reshape(n, -1)[:, :dim]


def rmsnorm(h, weight, eps):
    """(y, rstd) of rows h, in float64."""
    h = np.asarray(h, dtype=np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * weight, rstd


def rmsnorm_grad(h, weight, eps, dy, dh):
    """(dx, dweight) from the gradients of y and of h."""
    _, rstd = rmsnorm(h, weight, eps)
    u = h * rstd[:, None]
    g = dy * weight
    dx = rstd[:, None] * (g - u * (g * u).mean(1, keepdims=True)) + dh
    return dx, (dy * u).sum(0)


def embed_grad(dout, ids, rows, scale):
    """(gradient, sum of the terms' magnitudes, number of terms) of a table of `rows` rows."""
    dout = np.asarray(dout, dtype=np.float64)
    d, t, c = np.zeros((rows, dout.shape[1])), np.zeros((rows, dout.shape[1])), np.zeros(rows, dtype=np.int64)
    on = (ids >= 0) & (ids < rows)
    np.add.at(d, ids[on], dout[on])
    np.add.at(t, ids[on], np.abs(dout[on]))
    np.add.at(c, ids[on], 1)
    return d * scale, t * abs(scale), c


def _softmax(scores, scale):
    """(p, log p) of a row of scores; None for a row without a probability."""
    x = np.asarray(scores, dtype=np.float64)
    if np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
        return None, None
    d = (x - x.max()) * scale
    e = np.exp(d)
    return e / e.sum(), d - np.log(e.sum())


def verify(target, tokens, uniforms, draft=None, counts=None, scale=1.0, draft_scale=None):
    """(tokens, accepted, logprob) for target (b x (k + 1) x n), tokens (b x k), uniforms
    (b x (k + 1))."""
    b, k1, n = target.shape
    k = k1 - 1
    draft_scale = scale if draft_scale is None else draft_scale
    out, accepted, logprob = np.full((b, k1), -1, dtype=np.int64), np.zeros(b, dtype=np.int32), np.zeros((b, k1))
    for s in range(b):
        count = k if counts is None else min(max(int(counts[s]), 0), k)
        i, q = 0, None
        while True:
            p, logs = _softmax(target[s, i], scale)
            if i == count:
                break
            x = int(tokens[s, i])
            q = _softmax(draft[s, i], draft_scale)[0] if draft is not None else None
            inside = 0 <= x < n
            qx = 1.0 if draft is None else q[x] if q is not None and inside else np.nan
            if not (inside and p is not None and float(uniforms[s, i]) * qx < p[x]):
                break
            out[s, i], logprob[s, i] = x, logs[x]
            i += 1
        accepted[s] = i
        if p is None:
            continue
        r = p
        if i < count:
            if draft is None:
                over = np.where(np.arange(n) == tokens[s, i], 0.0, p)
            else:
                over = np.maximum(p - q, 0.0) if q is not None else np.zeros(n)
            r = over if over.sum() > 0 else p
        u = np.float32(uniforms[s, k])
        u = float(min(max(u if u == u else np.float32(0), np.float32(0)), np.float32(1 - 2.0 ** -24)))
        c = np.cumsum(r)
        t = int(np.searchsorted(c, u * c[-1], side="right"))
        out[s, i], logprob[s, i] = t, logs[t]
    return out, accepted, logprob
