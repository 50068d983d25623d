"""4-bit (MX4) rows on the GPU at the ends of what the calls take."""

import numpy as np
import pytest

from oracle import mx4

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


@pytest.mark.parametrize("n", [1 << 30, (1 << 30) - 63])
def test_one_row_against_as_many_rows_as_threads_of_a_grid(R, n):
    """The form with one wavefront to 16 rows of b would have 2^32 threads (73 GB of codes)."""
    b = R.Mx4Rows.empty(n, 32, "cuda")
    b.codes.zero_()
    b.scales.fill_(127)
    at = torch.tensor([0, 63, 1 << 26, n - 65, n - 1], device="cuda")
    b.codes[at, 3] = torch.arange(1, 6, device="cuda", dtype=torch.uint8)
    a = R.rslm_mx4_quantize(torch.full((1, 32), 2.0, device="cuda"))
    out = R.rslm_mx4_matmul(a, b, dtype=torch.bfloat16)
    value = 2.0 * torch.tensor(mx4.E2M1[1:6], device="cuda", dtype=torch.float32)
    assert torch.equal(out[0, at].float(), value)
    assert torch.count_nonzero(out) == 5
