"""The root-mean-square norm of values whose squares' sum passes float32 while their mean,
which the calls take up to float32's largest, does not.

Tolerances: those of tests/test_gpu_norm.py.  The sum is taken of values times 2^-8, which is
exact, so its depth D = 80 + dim / 128 units of 2^-24 is the same; what squares below 2^-126
lose there is far below a unit of a sum above 2^112.
"""

import numpy as np
import pytest

from oracle import mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("n,dim", [(5, 5), (9, 100), (6, 300), (1100, 1000), (6, 1000), (6, 2049), (6, 4096), (6, 9000), (6, 16384),
                                   (6, 16392), (6, 65536)])
def test_large_values(R, n, dim, residual, dt):
    g = torch.Generator().manual_seed(dim)
    # magnitudes of 0.6 to 1.2 10^19: a mean of about 8 10^37, a sum past 3.4 10^38 from 5 values on
    x = 1.2e19 * (0.5 + 0.5 * torch.rand((n, dim), generator=g)) * (2 * torch.randint(0, 2, (n, dim), generator=g) - 1)
    x[1::3] = torch.randn((len(x[1::3]), dim), generator=g)      # ordinary rows beside them
    x = x.to(DT[dt]).cuda()
    # halves that add up to x exactly
    r = R.rslm_rmsnorm(x / 2, residual=x / 2, rows=True) if residual else R.rslm_rmsnorm(x, rows=True)
    assert torch.equal(r.h, x)
    y, rstd = mx8.rmsnorm(f64(x), np.ones(dim), 1e-6)
    depth = 80 + dim / 128
    assert (np.abs(f64(r.rstd) - rstd) <= (depth / 2 + 4) * U * rstd).all()
    tol = (depth / 2 + 6) * U * np.abs(y)
    assert (np.abs(f64(r.y) - y) <= tol + HALF[dt] * (np.abs(y) + tol)).all()
    got = mx8.values(r.rows.codes.cpu().numpy(), r.rows.scales.cpu().numpy(), dim)
    unit = np.repeat(np.ldexp(1.0, r.rows.scales.cpu().numpy().astype(int) - 127), 32, axis=1)[:, :dim] * 2.0 ** -10
    assert (np.abs(got - y) <= np.maximum(2.0 ** -4 * (np.abs(y) + tol), unit) + tol).all()


@pytest.mark.parametrize("dim", [100, 300, 2049, 9000, 16392])
def test_past_the_mean_of_float32(R, dim):
    """Beside a large row: one whose mean is past float32 too, one with an infinity, one with a
    NaN, and a row of zeros."""
    x = torch.full((5, dim), 1e19, device="cuda")
    x[1] = 3e19
    x[2, dim - 1] = float("inf")
    x[3, 0] = float("nan")
    x[4] = 0
    r = R.rslm_rmsnorm(x, eps=1e-6)
    assert (r.y[0] - 1).abs().max() <= (44 + dim / 256) * U
    assert r.rstd[1] == 0 and (r.y[1] == 0).all()
    assert r.rstd[2] == 0 and r.y[2, dim - 1].isnan() and (r.y[2, :dim - 1] == 0).all()
    assert r.y[3].isnan().all()
    assert (r.y[4] == 0).all() and abs(float(r.rstd[4]) - 1e3) < 1e-3


@pytest.mark.parametrize("n,dim", [(200_000, 1030), (140_000, 5)])
def test_large_rows_among_many(R, n, dim):
    """More rows than workgroups, large and ordinary ones in turns that differ from workgroup to
    workgroup: each has its own sum."""
    g = torch.Generator(device="cuda").manual_seed(dim)
    x = torch.randn((n, dim), generator=g, device="cuda")
    large = torch.rand((n,), generator=g, device="cuda") < 0.5
    x[large] = 1.2e19 * (0.5 + 0.5 * torch.rand((int(large.sum()), dim), generator=g, device="cuda"))
    r = R.rslm_rmsnorm(x, y=False, rows=True)
    rstd = 1 / torch.sqrt(x.double().square().mean(1) + 1e-6)
    assert ((r.rstd.double() - rstd).abs() <= (44 + dim / 256) * U * rstd).all()
    assert torch.equal(R.rslm_rmsnorm(x[:70], y=False, rows=True).rows.codes, r.rows.codes[:70])
    assert torch.equal(R.rslm_rmsnorm(x[-70:], y=False, rows=True).rows.codes, r.rows.codes[-70:])
