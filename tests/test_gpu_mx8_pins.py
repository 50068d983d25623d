"""Products of 8-bit with 4-bit rows where the sum of magnitudes, which the other tests'
tolerances go by, says little: terms that cancel, and whether a call repeats itself.
"""

import numpy as np
import pytest

from oracle import mx4, mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# one of each arrangement: few rows (shared out or not, held in LDS or not), tiles of either height
SIZES = [(1, 300, 96), (16, 100, 4096), (16, 70000, 200), (15, 50, 4200), (130, 1030, 500), (300, 5000, 640), (1000, 17000, 1536)]


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,dim", SIZES)
def test_terms_that_cancel(R, m, n, dim, dt):
    """Products 64, -64 and c beside each other, once in a row: the result is c.  A float32 one
    is c itself.  Of a 16-bit one's c what lies below 2^-13 of the largest product, 2^-7, is cut
    off: all of c = 2^-9, nothing of c = 1."""
    rng = np.random.default_rng(dim)
    at = 8 * rng.integers(0, dim // 8, m)
    small = np.arange(m) % 2 == 1
    one, big = 0x38, 0x58                                   # 1 and 16
    ac = np.zeros((m, dim), dtype=np.uint8)
    rows = np.arange(m)
    ac[rows, at], ac[rows, at + 1], ac[rows, at + 2] = big, big | 0x80, np.where(small, 1, one)     # 2^-9, or 1
    bc = np.zeros((n, dim), dtype=np.uint8)
    # 4, 4, 1 and zeros
    phase = np.arange(dim) % 8
    bc[:] = np.where(phase < 2, 6, np.where(phase == 2, 2, 0)).astype(np.uint8)
    bs = np.full((n, -(-dim // 32)), 127, dtype=np.uint8)
    asc = np.full((m, -(-dim // 32)), 127, dtype=np.uint8)
    a, b = mx8.pack(ac, asc, dim), mx4.pack(bc, bs, dim)
    want = mx8.values(*a, dim) @ mx4.values(*b, dim).T
    c = np.where(small, 2.0 ** -9, 1.0)[:, None]
    assert (want == c).all()                                # 16 x 4 - 16 x 4 + c
    got = R.rslm_mx8_score(R.Mx8Rows(*map(dev, a), dim), R.Mx4Rows(*map(dev, b), dim), dtype=DT[dt]).double().cpu().numpy()
    if dt == "f32":
        assert (got == want).all()
    else:
        assert (got[~small] == 1).all()
        assert (np.abs(got - want) <= 64 * 2.0 ** -13).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,dim", SIZES + [(2048, 8192, 4096)])
def test_a_call_repeats_itself(R, m, n, dim, dt):
    """The same bits each time, with products of other rows in the same memory between."""
    g = torch.Generator(device="cuda").manual_seed(m + n)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    sides = [(R.rslm_mx8_quantize(normal(m, dim)), R.rslm_mx4_quantize(normal(n, dim))) for _ in range(2)]
    first = [R.rslm_mx8_score(a, b, dtype=DT[dt]) for a, b in sides]
    for _ in range(8):
        for (a, b), want in zip(sides, first):
            assert torch.equal(R.rslm_mx8_score(a, b, dtype=DT[dt]), want)
