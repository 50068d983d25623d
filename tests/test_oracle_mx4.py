"""Pins of the float64 restatement of the 4-bit rows and the log
probabilities, and the refusals of their entry points (no GPU needed)."""

import ctypes as C

import numpy as np
import pytest

from oracle import mx4
from paper_2608_30384_amd import _lib as L


def test_e2m1_grid_and_ties():
    # every value of the format, both signs (bit layout s e e m, bias 1)
    for code in range(16):
        s, e, f = code >> 3, (code >> 1) & 3, code & 1
        v = (f * 0.5 if e == 0 else (1 + f / 2) * 2.0 ** (e - 1)) * (-1) ** s
        assert mx4.E2M1[code & 7] == abs(v)
        assert mx4.e2m1(np.array([v]))[0] == code or (v == 0 and mx4.e2m1(np.array([v]))[0] in (0, 8))
    # midpoints go to the even code, and what lies beyond 6 saturates
    for v, code in [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (7.99, 7), (1e9, 7),
                    (0.2500001, 1), (0.7499999, 1), (5.0000001, 7)]:
        assert mx4.e2m1(np.array([v]))[0] == code
        assert mx4.e2m1(np.array([-v]))[0] == code + 8


def test_scale_rule():
    # the largest coordinate of a block falls in [4, 8) of the codes' units
    for top, s in [(1.0, 125), (1.99, 125), (2.0, 126), (6.0, 127), (2.0 ** -126, 0), (2.0 ** -140, 0), (0.0, 0),
                   (2.0 ** 127, 252)]:
        x = np.zeros((1, 32))
        x[0, 7] = -top
        c, sc = mx4.quantize(x)
        assert sc[0, 0] == s
        if top >= 2.0 ** -124:
            assert 4 <= top / 2.0 ** (s - 127.0) < 8
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones((1, 64))
        x[0, 40] = bad
        c, sc = mx4.quantize(x)
        assert list(sc[0]) == [125, 255]
        v = mx4.values(*mx4.pack(c, sc, 64), 64)
        assert np.isfinite(v[0, :32]).all() and np.isnan(v[0, 32:]).all()


def test_pack_round_trip_and_error():
    rng = np.random.default_rng(0)
    for dim in (1, 31, 32, 33, 100, 128, 129, 300):
        x = rng.standard_normal((5, dim)) * np.exp(rng.standard_normal((5, 1)))
        c, s = mx4.quantize(x)
        pc, ps = mx4.pack(c, s, dim)
        v = mx4.values(pc, ps, dim)
        assert pc.shape == (5, 64 * -(-dim // 128)) and ps.shape == (5, 4 * -(-dim // 128))
        c2, s2 = mx4.quantize(v)
        # values are fixed points, unless the largest was rounded up to the next power of two
        assert np.array_equal(mx4.values(*mx4.pack(c2, s2, dim), dim), v)
        # nearest: within half of the widest gap of the block's grid, or saturated from below 8
        unit = np.repeat(np.ldexp(1.0, s.astype(int) - 127), 32, axis=1)[:, :dim]
        assert np.all(np.abs(v - x) <= np.where(np.abs(x) > 6 * unit, 2.0, 1.0) * unit)


def test_logprob_and_gradient_by_differences():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 9)) * 2
    x[1, 3] = x[2, :5] = -np.inf
    x[3] = x[3, 0]
    t = np.array([2, 3, 7, -1])
    scale = 1.7
    r = mx4.logprob(x, scale, t, 12)
    live = ~r["masked"]
    assert np.allclose(r["p"].sum(1), 1.0) and r["logprob"][1] == -np.inf and r["logprob"][3] == 0.0
    assert np.allclose(r["entropy"][3], np.log(9))
    assert list(r["ids"][3]) == list(range(9)) + [-1] * 3          # ties by index, padding
    assert list(r["ids"][2][:4]) == sorted(range(5, 9), key=lambda j: -x[2, j]) and r["ids"][2][4] == -1
    t[1] = 0
    dl, dh = rng.standard_normal(4), rng.standard_normal(4)
    g = mx4.logprob_grad(x, scale, t, dl, dh)

    def f(y):
        q = mx4.logprob(y, scale, t)
        return q["logprob"] @ dl + q["entropy"] @ dh

    for i in range(4):
        for j in range(9):
            if not live[i, j]:
                assert g[i, j] == 0.0
                continue
            up, dn = x.copy(), x.copy()
            up[i, j] += 1e-5
            dn[i, j] -= 1e-5
            assert abs((f(up) - f(dn)) / 2e-5 - g[i, j]) < 1e-8
    e = mx4.logprob(np.full((1, 5), -np.inf), 1.0, np.array([2]), 2)
    assert e["lse"][0] == -np.inf and e["entropy"][0] == 0.0 and list(e["ids"][0]) == [-1, -1]


P = C.c_void_p(0x10000)      # aligned, never read: every call below is refused
Z = C.c_void_p(0)
ODD = C.c_void_p(0x10001)


def test_mx4_calls_validate_arguments_without_device():
    lib = L.lib()
    q = lib.rslm_mx4_quantize
    assert q(None, Z, 0, 0, 96, 96, Z, Z, Z) == 0                        # nothing to do
    for bad in [(P, 3, 4, 96, 96, P, P), (P, -1, 4, 96, 96, P, P), (P, 0, -1, 96, 96, P, P), (P, 0, 4, 0, 96, P, P),
                (P, 0, 4, 65537, 96, P, P), (P, 0, 4, 96, -1, P, P), (Z, 0, 4, 96, 96, P, P), (P, 0, 4, 96, 96, Z, P),
                (P, 0, 4, 96, 96, P, Z), (ODD, 2, 4, 96, 96, P, P), (P, 0, 4, 96, 96, C.c_void_p(0x10008), P),
                (P, 0, 4, 96, 96, P, C.c_void_p(0x10002)), (P, 0, 1 << 31, 96, 96, P, P)]:
        assert q(None, *bad, Z) == 1, bad
    d = lib.rslm_mx4_dequantize
    assert d(Z, Z, 0, 96, Z, 0, 96, Z) == 0
    for bad in [(P, P, 4, 96, P, 3, 96), (P, P, 4, 96, P, 0, 95), (P, P, 4, 0, P, 0, 96), (Z, P, 4, 96, P, 0, 96),
                (P, Z, 4, 96, P, 0, 96), (P, P, 4, 96, Z, 0, 96), (P, P, 4, 96, ODD, 1, 96)]:
        assert d(*bad, Z) == 1, bad
    mm = lib.rslm_mx4_matmul
    assert mm(Z, Z, 0, P, P, 4, 96, P, 0, 4, Z) == 0 and mm(P, P, 4, Z, Z, 0, 96, P, 0, 4, Z) == 0
    for bad in [(P, P, -1, P, P, 4, 96, P, 0, 4), (P, P, 4, P, P, -4, 96, P, 0, 4), (P, P, 4, P, P, 4, 0, P, 0, 4),
                (P, P, 4, P, P, 4, 96, P, 5, 4), (P, P, 4, P, P, 4, 96, P, 0, 3), (Z, P, 4, P, P, 4, 96, P, 0, 4),
                (P, P, 4, P, Z, 4, 96, P, 0, 4), (P, P, 4, P, P, 4, 96, Z, 0, 4), (P, P, 1 << 23, P, P, 4, 96, P, 0, 4)]:
        assert mm(*bad, Z) == 1, bad
    sc = lib.rslm_mx4_score
    assert sc(Z, 0, 0, 96, P, P, 4, 96, P, 0, 4, Z, 0, Z) == 0 and sc(P, 0, 4, 96, Z, Z, 0, 96, P, 0, 4, Z, 0, Z) == 0
    assert sc(P, 1, 4, 96, P, P, 4, 96, P, 2, 4, Z, 0, Z) == 2 and sc(P, 0, 4, 96, P, P, 4, 96, P, 1, 4, Z, 0, Z) == 2
    need = lib.rslm_mx4_score_workspace(100, 1000, 96, 0)
    assert need > 0 and lib.rslm_mx4_score_workspace(1, 1000, 96, 0) == 0 and lib.rslm_mx4_score_workspace(100, 1000, 96, 9) == 0
    assert sc(P, 0, 100, 96, P, P, 1000, 96, P, 0, 1000, P, need - 1, Z) == 4
    assert sc(P, 0, 100, 96, P, P, 1000, 96, P, 0, 1000, ODD, need, Z) == 1
    for bad in [(P, 7, 4, 96, P, P, 4, 96, P, 0, 4), (P, 0, 4, -96, P, P, 4, 96, P, 0, 4), (Z, 0, 4, 96, P, P, 4, 96, P, 0, 4),
                (P, 0, 4, 96, P, P, 4, 96, P, 0, 3), (P, 0, 4, 96, ODD, P, 4, 96, P, 0, 4), (P, 0, 4, 96, P, P, 4, 70000, P, 0, 4)]:
        assert sc(*bad, P, 1 << 30, Z) == 1, bad
    bw = lib.rslm_mx4_score_backward
    need = lib.rslm_mx4_score_backward_workspace(256, 131072, 768, 0)
    assert need > 0
    assert lib.rslm_mx4_score_backward_workspace(0, 131072, 768, 0) == 0
    assert bw(P, 0, 256, 131072, P, P, 131072, 768, P, 0, 768, P, need - 1, Z) == 4
    assert bw(P, 0, 256, 131072, P, P, 131072, 768, P, 0, 768, Z, need, Z) == 1
    assert bw(P, 0, 256, 131072, P, P, 131072, 768, P, 0, 767, P, need, Z) == 1
    assert bw(P, 1, 256, 131072, P, P, 131072, 768, P, 2, 768, P, need, Z) == 2
    assert bw(P, 0, 0, 131072, P, P, 131072, 768, Z, 0, 768, Z, 0, Z) == 0


def test_logprob_calls_validate_arguments_without_device():
    lib = L.lib()
    f = lib.rslm_logprob
    ok = [P, 0, 4, 100, 100, 1.0, P, 5, P, P, P, P, P, P, P, 1 << 20]
    assert f(Z, 0, 0, 100, 100, 1.0, Z, 0, Z, Z, Z, Z, Z, Z, Z, 0, Z) == 0
    for i, v in [(0, Z), (1, 3), (2, -1), (3, 0), (4, -1), (5, 0.0), (5, -1.0), (5, float("inf")), (5, float("nan")),
                 (6, Z), (7, -1), (7, 1025), (11, Z), (12, Z), (13, Z), (0, ODD), (6, C.c_void_p(0x10004)),
                 (9, C.c_void_p(0x10002)), (2, 1 << 24), (3, 1 << 31)]:
        a = list(ok)
        a[i] = v
        assert f(*a, Z) == 1, (i, v)
    need = lib.rslm_logprob_workspace(1, 1 << 20, 20)
    assert need > 0 and lib.rslm_logprob_workspace(1 << 16, 100, 20) == 0
    a = list(ok)
    a[2], a[3], a[4], a[7], a[15] = 1, 1 << 20, 1 << 20, 20, need - 1
    assert f(*a, Z) == 4
    a[14], a[15] = Z, need
    assert f(*a, Z) == 1
    b = lib.rslm_logprob_backward
    ok = [P, 0, 4, 100, 100, 1.0, P, P, P, P, P, P, 100]
    assert b(Z, 0, 0, 100, 100, 1.0, Z, Z, Z, Z, Z, Z, 100, Z) == 0
    for i, v in [(0, Z), (1, 4), (3, 0), (5, -2.0), (6, Z), (7, Z), (8, Z), (11, Z), (12, 99), (11, ODD)]:
        a = list(ok)
        a[i] = v
        assert b(*a, Z) == 1, (i, v)


def test_binding_refuses_wrong_tensors():
    import torch

    import paper_2608_30384_amd as R

    x = torch.zeros(4, 96)
    with pytest.raises(ValueError):
        R.rslm_mx4_quantize(x)                                      # not on a device
    with pytest.raises(ValueError):
        R.Mx4Rows(torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8), 96)
    with pytest.raises(ValueError):
        R.rslm_logprob(x)
