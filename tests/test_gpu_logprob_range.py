"""Log probabilities at the ends of float32's range, against float64.

Tolerances, in units of U = 2^-24: z is known to 3 of them and a row of few entries
has a log-sum-exp good to 8 (log n + 4); what is compared is at most 100 in
magnitude, so 4 (100 + 8 (log n + 4)) U = 4e-5 covers values and, relative to the
largest entry, gradients.
"""

import numpy as np
import pytest

from oracle import mx4

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

TOL = 4e-5


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def check(R, x, scale, target, dl=None, dh=None, k=3):
    """x: float32 array of scores whose z is within float32."""
    t = torch.from_numpy(x).cuda()
    tt = torch.tensor(target, device="cuda")
    r = R.rslm_logprob(t, tt, k, scale=scale)
    s32 = float(np.float32(scale))
    want = mx4.logprob(x, s32, target, k)
    room = lambda w: TOL * np.maximum(1.0, np.abs(np.where(np.isfinite(w), w, 0.0)))
    for name, got in (("lse", r.lse), ("entropy", r.entropy), ("logprob", r.logprob), ("top", r.top_logprob)):
        with np.errstate(invalid="ignore", over="ignore"):
            g, w = got.double().cpu().numpy(), want[name].astype(np.float32).astype(np.float64)
            assert ((g == w) | (np.abs(g - w) <= room(w))).all(), (name, g, w)
    assert np.array_equal(r.top_ids.cpu().numpy(), want["ids"])
    if dl is not None:
        d = [torch.tensor(v, dtype=torch.float32, device="cuda") for v in (dl, dh)]
        g = R.rslm_logprob_backward(t, tt, r, d[0], d[1], scale=scale).double().cpu().numpy()
        w = mx4.logprob_grad(x, s32, target, d[0].double().cpu().numpy(), d[1].double().cpu().numpy())
        assert np.isfinite(g).all() and (np.abs(g - w) <= TOL * np.abs(w).max(1, keepdims=True)).all(), (g, w)
    return r


@pytest.mark.parametrize("n", [5, 9000])
def test_largest_scale(R, n):
    """2^127 is taken, and anything above it refused: its product with log2(e) is no float32."""
    scale = 2.0 ** 127
    x = np.full((3, n), -1.9, dtype=np.float32)
    x[0, :3] = 0.25, 0.5, 0.5                        # z of 2^125 and 2^126: two equal ones
    x[1, :4] = np.float32(np.array([0.0, -1.0, -2.0, -50.0]) / scale)
    x[2, :2] = 0.0
    check(R, x, scale, [1, 1, 0])
    t = torch.from_numpy(x).cuda()
    r = R.rslm_logprob(t, k=2, scale=scale)
    for bad in (float(np.nextafter(np.float32(scale), np.float32(np.inf))), 3e38, float("inf"), 0.0, -1.0, float("nan")):
        with pytest.raises(R.RslmError):
            R.rslm_logprob(t, k=2, scale=bad)
        r.scale = bad
        with pytest.raises(R.RslmError):
            R.rslm_logprob_backward(t, None, r)


@pytest.mark.parametrize("n", [5, 9000, 70001])
@pytest.mark.parametrize("scale", [1e-38, 2e-38, 0.5, 1.0, 1.5])
def test_scores_further_apart_than_the_largest_float(R, n, scale):
    """z stays within float32 although differences of the scores do not."""
    rng = np.random.default_rng(n)
    x = rng.uniform(-3.3e38, 3.3e38, (4, n)).astype(np.float32) / np.float32(max(1.0, scale))
    x[1] = np.where(np.arange(n) % 2, x.min(), x.max())
    x[2, 0], x[2, n - 1] = x.max(), x.min()
    x[3, 1:] = -np.inf
    check(R, x, scale, [0, 1, n - 1, 0], [1e10, -1e10, 0.0, 1e10], [0.0, 1e10, 1e10, 0.0])


@pytest.mark.parametrize("n", [5, 9000])
@pytest.mark.parametrize("size,scale", [(1e33, 1.0), (3e37, 4.0), (1.0, 1e37), (1e-20, 1e36), (1e-33, 1.0), (1e-10, 1e-20),
                                        (1e20, 1e-20)])
def test_gradients_as_large_and_as_small_as_a_float(R, n, size, scale):
    """Entry by entry: probabilities below float32's normal range too, where the
    product with a large gradient is a normal number again.  An entry is off by the
    error of z - lse (at most 150: 3 (150 + 8 (log n + 4)) U) relative to its terms'
    magnitudes, and by float32's least normal number."""
    rng = np.random.default_rng(n)
    z = rng.uniform(-90.0, 0.0, (4, n))
    x = (z / scale).astype(np.float32)
    x[0, 1] = 0.0
    t = [1, n - 1, 0, 2]
    dl, dh = np.array([1.0, -1.0, 0.0, 0.5]) * size, np.array([0.0, 0.01, -0.01, 0.0]) * size
    tt = torch.tensor(t, device="cuda")
    xt = torch.from_numpy(x).cuda()
    d = [torch.tensor(v, dtype=torch.float32, device="cuda") for v in (dl, dh)]
    r = R.rslm_logprob(xt, tt, scale=scale)
    g = R.rslm_logprob_backward(xt, tt, r, d[0], d[1], scale=scale).double().cpu().numpy()
    s32 = float(np.float32(scale))
    d = [v.double().cpu().numpy() for v in d]
    want = mx4.logprob_grad(x, s32, t, d[0], d[1])
    ref = mx4.logprob(x, s32, t)
    hit = np.zeros((4, n))
    hit[np.arange(4), t] = 1.0
    terms = s32 * (np.abs(d[0])[:, None] * (hit + ref["p"]) + np.abs(d[1])[:, None] * ref["p"] * (np.abs(ref["logs"]) + ref["entropy"][:, None] + 1))
    tol = 2.0 ** -24 * 3 * (150 + 8 * (np.log(n) + 4)) * terms + 2.0 ** -126
    assert np.isfinite(g).all()
    assert (np.abs(g - want) <= tol).all(), (g, want, tol)


@pytest.mark.parametrize("n", [6, 9000])
def test_z_past_the_largest_float(R, n):
    """Finite scores whose z is not: the log-sum-exp alone is infinite, and entries whose z
    is below float32 are masked."""
    x = np.full((3, n), -3e38, dtype=np.float32)
    x[0, :4] = 3e38, 3e38, 1e38, -1e38
    x[1, 0] = 2e38
    check(R, x, 2.0, [1, 0, 2], [1.0, -2.0, 1.0], [0.0, 1.0, 1.0])
