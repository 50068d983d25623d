"""The float64 restatements of 8-bit rows, norms, tables and verification, against
closed forms, differences and counting."""

import numpy as np
import pytest

from oracle import mx8


def test_levels():
    assert mx8.E4M3[0] == 0 and mx8.E4M3[1] == 2.0 ** -9 and mx8.E4M3[8] == 2.0 ** -6 and mx8.E4M3[126] == 448
    assert (np.diff(mx8.E4M3) > 0).all()


def test_codes_are_nearest_ties_even():
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 500), rng.standard_normal(500) * 2.0 ** -8, (mx8.E4M3[1:] + mx8.E4M3[:-1]) / 2])
    c = mx8.e4m3(v)
    got = mx8.E4M3[c & 127] * np.where(c & 128, -1, 1)
    d = np.abs(np.abs(v)[:, None] - mx8.E4M3)
    assert np.array_equal(np.abs(np.abs(v) - np.abs(got)), d.min(1))
    tied = (d == d.min(1, keepdims=True)).sum(1) == 2
    assert tied.sum() >= 126 and (c[tied] % 2 == 0).all()
    assert (np.sign(got[got != 0]) == np.sign(v[got != 0])).all()


@pytest.mark.parametrize("top", [1.0, 448.0, 448.1, 449.0, 512.0, 3e-39, 1.7e38])
def test_scale_is_the_least_that_holds_the_largest(top):
    c, s = mx8.quantize(np.array([[top, -top / 3]]))
    s = int(s[0, 0])
    assert top <= 448 * 2.0 ** (s - 127) and (s == 0 or top > 448 * 2.0 ** (s - 128))
    v = mx8.values(*mx8.pack(c, np.array([[s]], dtype=np.uint8), 2), 2)
    assert np.abs(v - [top, -top / 3]).max() <= max(2.0 ** -4 * top, 2.0 ** -137)


def test_norm_gradient_by_differences():
    rng = np.random.default_rng(1)
    h, w = rng.standard_normal((4, 9)), rng.standard_normal(9)
    dy, dh = rng.standard_normal((4, 9)), rng.standard_normal((4, 9))
    dx, dw = mx8.rmsnorm_grad(h, w, 1e-3, dy, dh)

    def loss(h, w):
        return (mx8.rmsnorm(h, w, 1e-3)[0] * dy).sum() + (h * dh).sum()

    for i in np.ndindex(h.shape):
        e = np.zeros_like(h)
        e[i] = 1e-6
        assert abs((loss(h + e, w) - loss(h - e, w)) / 2e-6 - dx[i]) < 1e-7
    for i in range(9):
        e = np.zeros_like(w)
        e[i] = 1e-6
        assert abs((loss(h, w + e) - loss(h, w - e)) / 2e-6 - dw[i]) < 1e-7


@pytest.mark.parametrize("draft", [True, False])
def test_verified_tokens_have_the_targets_distribution(draft):
    """Drafts drawn from q (or one certain draft) and a grid of uniforms: the first token
    comes out as often as p says."""
    rng = np.random.default_rng(2)
    n, grid = 6, 60
    z, d = rng.standard_normal(n), rng.standard_normal(n)
    p = np.exp(z) / np.exp(z).sum()
    q = np.exp(d) / np.exp(d).sum() if draft else np.eye(n)[2]
    u = (np.arange(grid) + 0.5) / grid
    u0, u1 = (a.reshape(-1) for a in np.meshgrid(u, u))
    found = np.zeros(n)
    for x in range(n):
        if q[x] == 0:
            continue
        b = len(u0)
        out, accepted, logprob = mx8.verify(np.broadcast_to(z, (b, 2, n)), np.full((b, 1), x), np.stack([u0, u1], 1),
                                            draft=np.broadcast_to(d, (b, 1, n)) if draft else None)
        assert ((accepted == 0) | (out[:, 0] == x)).all() and (out[:, 1][accepted == 0] == -1).all()
        assert np.abs(logprob[:, 0] - np.log(p[out[:, 0]])).max() < 1e-12
        found += q[x] * np.bincount(out[:, 0], minlength=n) / b
    assert np.abs(found - p).max() < 4 / grid
