"""Products of 8-bit with 4-bit rows whose codes lie past 4 GiB from their start.

All values are -1 and 1, so that every partial sum of 65,536 products is a whole number that
float32 holds and nothing is cut off: float32 results are equal to the products, bfloat16
ones to these rounded.  The rows that an offset short of its 33rd bit would read hold the
negatives of those looked at, whose products are not all zero, so that no such row passes
for another, nor a result of zeros.
"""

import numpy as np
import pytest

from oracle import mx4, mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DIM = 65536


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def signs(r, bits):
    """Codes of -1 and 1 whose signs are those bits of r: E4M3's (8) or E2M1's (4)."""
    return r & 0x80 | 0x38 if bits == 8 else r & 0x88 | 0x22


def far_rows(kind, bits, n, looked, rng):
    """n rows, those in `looked` from rng, the others random."""
    rows = kind.empty(n, DIM, torch.device("cuda", 0))
    rows.codes.random_(0, 256, generator=torch.Generator(device="cuda").manual_seed(bits))
    for part in rows.codes.split(16384):
        part.copy_(signs(part, bits))
    rows.scales.fill_(127)
    codes = signs(rng.integers(0, 256, (len(looked), rows.codes.shape[1])).astype(np.uint8), bits)
    wrap = (1 << 32) // rows.codes.shape[1]
    for i, c in zip(looked, codes):
        rows.codes[i] = torch.from_numpy(c).cuda()
        if i >= wrap:
            assert i - wrap not in looked
            rows.codes[i - wrap] = torch.from_numpy(c ^ (0x80 if bits == 8 else 0x88)).cuda()
    scales = np.full((len(looked), DIM // 32), 127, dtype=np.uint8)
    return rows, (mx8 if bits == 8 else mx4).values(codes, scales, DIM)


def places(n):
    return sorted({0, n // 2, max(n - 2, 0), n - 1})


SIZES = [(1, 140_000), (16, 140_000), (20, 140_000), (300, 140_000), (70_000, 20), (70_000, 300)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n", SIZES)
def test_score(R, m, n, dtype):
    i, j, rng = places(m), places(n), np.random.default_rng(m + n + 1)
    a, x = far_rows(R.Mx8Rows, 8, m, i, rng)
    b, y = far_rows(R.Mx4Rows, 4, n, j, rng)
    assert max(a.codes.numel(), b.codes.numel()) > 1 << 32
    want = x @ y.T
    # neither zeros nor another looked-at row's products are a row's own, beyond bfloat16's rounding
    assert (want != 0).any(0).all() and (want != 0).any(1).all()
    for w in (want, want.T):
        for p in range(len(w)):
            for q in range(p):
                assert (np.abs(w[p] - w[q]) > 2.0 ** -7 * np.abs(w[p])).any()
    got = R.rslm_mx8_score(a, b, dtype=dtype)
    assert torch.equal(got[i][:, j].cpu(), torch.from_numpy(want).float().to(dtype))
