"""Norms of more rows than the kernels launch workgroups for (65,536 forward, 512 or more strips
backward), so that a workgroup takes several, and of strips that get none.  Against float64 on
the same device; tolerances as in tests/test_gpu_norm.py, with D = 80 + dim / 128, and of
dweight n + 8 units of 2^-24 of the sum of magnitudes.
"""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def pieces(n, dim):
    """Runs of rows of some 64 million values."""
    step = max(1, (1 << 26) // dim)
    return [slice(i, min(n, i + step)) for i in range(0, n, step)]


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,dim", [(1_048_600, 20), (262_200, 130), (262_200, 700), (65_700, 1030), (65_600, 4100), (65_545, 9000),
                                   (65_700, 5), (140_000, 3), (513, 5), (1500, 5), (513, 16_392), (1500, 16_392)])
def test_rows(R, n, dim, dt):
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    normal = lambda: torch.randn((n, dim), generator=g, device="cuda", dtype=torch.float32).to(DT[dt])  # noqa: E731
    x, residual, dy, dh = normal(), normal(), normal(), normal()
    weight = 1 + 0.3 * torch.randn((dim,), generator=g, device="cuda")
    r = R.rslm_rmsnorm(x, weight, residual=residual, eps=EPS, rows=True)
    dx, dw = R.rslm_rmsnorm_backward(dy, r, weight, dh=dh)
    values = R.rslm_mx8_dequantize(r.rows)
    depth, w = 80 + dim / 128, weight.double()
    sums, terms = torch.zeros(dim, dtype=torch.float64, device="cuda"), torch.zeros(dim, dtype=torch.float64, device="cuda")
    for p in pieces(n, dim):
        h = (x[p].float() + residual[p].float()).to(DT[dt])
        assert torch.equal(r.h[p], h)
        h = h.double()
        rstd = 1 / torch.sqrt((h * h).mean(1) + EPS)
        assert ((r.rstd[p].double() - rstd).abs() <= (depth / 2 + 4) * U * rstd).all()
        y = h * rstd[:, None] * w
        tol = (depth / 2 + 6) * U * y.abs()
        assert ((r.y[p].double() - y).abs() <= tol + HALF[dt] * (y.abs() + tol)).all()
        # 8 bits: half a unit, or half the least step, 2^-10 of a scale that is above the largest / 448 and below the largest / 224
        top = torch.nn.functional.pad(y.abs(), (0, -dim % 32)).view(len(y), -1, 32).amax(-1).repeat_interleave(32, 1)[:, :dim]
        assert ((values[p].double() - y).abs() <= torch.maximum(2.0 ** -4 * (y.abs() + tol), 2.0 ** -10 / 224 * 1.001 * top) + tol).all()
        # the gradients, of the rstd that the call was given
        rstd = r.rstd[p].double()[:, None]
        u, gg, d = h * rstd, dy[p].double() * w, dh[p].double()
        mean, size = (gg * u).mean(1, keepdim=True), (gg * u).abs().mean(1, keepdim=True)
        want = rstd * (gg - u * mean) + d
        tol = U * (rstd * (4 * gg.abs() + u.abs() * ((depth + 8) * size + 4 * mean.abs())) + 2 * want.abs() + d.abs())
        assert ((dx[p].double() - want).abs() <= tol + HALF[dt] * (want.abs() + tol)).all()
        sums += (dy[p].double() * u).sum(0)
        terms += (dy[p].double() * u).abs().sum(0)
        del h, y, u, gg, d, want, tol, top
    tol = U * (n + 8) * terms
    assert ((dw.double() - sums).abs() <= tol + U * (sums.abs() + tol)).all()
    again = R.rslm_rmsnorm_backward(dy, r, weight, dh=dh)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
