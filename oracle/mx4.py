"""Microscaled 4-bit rows and log probabilities over scores, in float64.

Plain restatements used by the tests: E2M1 codes with one E8M0 scale for every
32 coordinates (stored two codes to a byte, low nibble first, rows padded to
128 coordinates), and the softmax statistics of rows of scores with their
gradient.
"""

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e2m1(v):
    """Codes of the values v (float64): nearest magnitude, ties to the even
    code, saturated; bit 3 the sign (a zero of either sign has code 0)."""
    v = np.asarray(v, dtype=np.float64)
    d = np.abs(np.abs(v)[..., None] - E2M1)
    best = d.min(-1, keepdims=True)
    tied = d == best
    # of two equally near neighbours the even code
    even = np.where(tied & (np.arange(8) % 2 == 0), 0, np.where(tied, 1, 2))
    return (even.argmin(-1) + 8 * (v < 0)).astype(np.uint8)


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
    _, e = np.frexp(top)          # top = f 2^e, 1/2 <= f < 1
    s = np.where(top > 0, np.maximum(e - 1 - 2 + 127, 0), 0)
    with np.errstate(invalid="ignore"):
        c = e2m1(np.where(bad[..., None], 0.0, p / np.ldexp(1.0, s - 127)[..., None]))
    return c.reshape(n, nb * 32)[:, :dim], np.where(bad, 255, s).astype(np.uint8)


def pack(codes, scales, dim):
    """The stored form: n x 64 steps bytes of codes and n x 4 steps scales."""
    n, steps = codes.shape[0], -(-dim // 128)
    c = np.zeros((n, 128 * steps), dtype=np.uint8)
    c[:, :dim] = codes
    s = np.zeros((n, 4 * steps), dtype=np.uint8)
    s[:, :scales.shape[1]] = scales
    return c[:, 0::2] | (c[:, 1::2] << 4), s


def values(codes, scales, dim):
    """float64 values of the stored form."""
    n = codes.shape[0]
    c = np.empty((n, 2 * codes.shape[1]), dtype=np.uint8)
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    v = E2M1[c & 7] * np.where(c & 8, -1.0, 1.0)
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(n, -1, 32) * scale[..., None]).reshape(n, -1)[:, :dim]


def logprob(scores, scale, target=None, k=0):
    """dict(lse, logprob, entropy, top, ids, logs, p) of rows of scores.  An entry
    that scale takes below float32's range is masked, as is -infinity."""
    x = np.asarray(scores, dtype=np.float64)
    z = x * scale
    z = np.where(z < -np.finfo(np.float32).max, -np.inf, z)
    m, n = z.shape
    masked = z == -np.inf
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        top = z.max(1, keepdims=True)
        ref = np.where(np.isneginf(top), 0.0, top)
        lz = np.log(np.exp(z - ref).sum(1, keepdims=True))
        lse = lz + ref
        logs = np.where(masked, -np.inf, z - ref - lz)
        p = np.where(masked, 0.0, np.exp(logs))
        plogs = np.where(masked, 0.0, p * logs)
        entropy = -plogs.sum(1) + 0.0
    out = dict(lse=lse[:, 0], entropy=entropy, logs=logs, p=p, masked=masked)
    if target is not None:
        t = np.asarray(target)
        on = (t >= 0) & (t < n)
        out["logprob"] = np.where(on, logs[np.arange(m), np.where(on, t, 0)], 0.0)
    key = np.where(np.isnan(x), -np.inf, x)
    ids = np.lexsort((np.broadcast_to(np.arange(n), (m, n)), -key))[:, :k]
    if ids.shape[1] < k:
        ids = np.pad(ids, ((0, 0), (0, k - ids.shape[1])), constant_values=-1)
    dead = (ids < 0) | np.isneginf(np.take_along_axis(np.where(np.isnan(z), -np.inf, z), np.maximum(ids, 0), 1))
    out["ids"] = np.where(dead, -1, ids)
    out["top"] = np.where(dead, -np.inf, np.take_along_axis(logs, np.maximum(ids, 0), 1))
    return out


def logprob_grad(scores, scale, target, dlogprob, dentropy):
    """Gradient of the scores from those of logprob and entropy."""
    r = logprob(scores, scale, target)
    m, n = r["p"].shape
    t = np.asarray(target)
    on = (t >= 0) & (t < n)
    hit = np.zeros((m, n))
    hit[np.arange(m)[on], t[on]] = 1.0
    dl = np.where(on, np.asarray(dlogprob, dtype=np.float64), 0.0)[:, None]
    dh = np.asarray(dentropy, dtype=np.float64)[:, None]
    logs = np.where(r["masked"], 0.0, r["logs"])
    d = dl * (hit - r["p"]) - dh * r["p"] * (logs + r["entropy"][:, None])
    return np.where(r["masked"], 0.0, d * scale)
