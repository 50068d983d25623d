"""Verification of batches so large that a wavefront takes several slices of a row, in the sums
and in the draw, where the slices do not divide evenly among them.  As in
tests/test_gpu_verify.py: tokens and how many stand are equal to float64's.
"""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from .test_gpu_verify import DT, R, check  # noqa: E402,F401

pytestmark = pytest.mark.gpu

SLICE, MOST_SLICES, WAVES = 1024, 256, 4
SUMS, DRAWS = 6144, 1024        # workgroups from which on a wavefront takes several slices


def make(b, k, n, dt, seed, masked):
    """As tests/test_gpu_verify.py's, made on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    z = 3 * normal(b, k + 1, n)
    z.masked_fill_(torch.rand((b, 1, n), generator=g, device="cuda") < masked, -float("inf"))
    d = (z[:, :k] + 0.7 * normal(b, k, n)).to(DT[dt])
    noise = -torch.log(-torch.log(torch.rand((b, k, n), generator=g, device="cuda").clamp(1e-6, 1 - 1e-6)))
    tokens = (d.float() + noise).argmax(-1)
    return z.to(DT[dt]).cpu(), d.cpu(), tokens.cpu(), torch.rand((b, k + 1), generator=g, device="cuda").cpu()


@pytest.mark.parametrize("b,k,n,dt,draft,masked", [
    (64, 4, 131_072, "bf16", True, 0.05), (200, 2, 70_001, "f32", True, 0.0), (200, 2, 130_000, "f16", False, 0.3),
    (67, 2, 300_001, "bf16", True, 0.0), (4200, 1, 5000, "f32", True, 0.0)])
def test_several_slices_to_a_wavefront(R, b, k, n, dt, draft, masked):  # noqa: F811
    blocks = -(-n // (SLICE * MOST_SLICES))
    slices = -(-n // (SLICE * blocks))
    rows = b * (k + 1 + (k if draft else 0))
    # else the sizes reach nothing that tests/test_gpu_verify.py does not
    assert rows * slices >= 2 * WAVES * SUMS and b * slices >= 2 * WAVES * DRAWS
    z, d, tokens, u = make(b, k, n, dt, n, masked)
    check(R, z, d if draft else None, tokens, u, scale=1.25)
    counts = torch.from_numpy(np.random.default_rng(b).integers(0, k + 1, b).astype(np.int32))
    check(R, z, d if draft else None, tokens, u, counts, scale=0.6, draft_scale=0.9 if draft else None)
