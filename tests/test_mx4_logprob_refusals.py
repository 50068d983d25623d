"""Refusals of the 4-bit and log probability entry points at the ends of their
ranges (no GPU needed: every call is refused before any launch)."""

import ctypes as C

import numpy as np
import pytest

from paper_2608_30384_amd import _lib as L

P = C.c_void_p(0x10000)      # aligned, never read
Z = C.c_void_p(0)


@pytest.mark.parametrize("scale", [float(np.nextafter(np.float32(2.0 ** 127), np.float32(np.inf))), 2.4e38, 3.4e38])
def test_scales_whose_product_with_log2e_is_no_float32(scale):
    lib = L.lib()
    assert lib.rslm_logprob(P, 0, 4, 100, 100, scale, P, 5, P, P, P, P, P, P, P, 1 << 20, Z) == 1
    assert lib.rslm_logprob_backward(P, 0, 4, 100, 100, scale, P, P, P, P, P, P, 100, Z) == 1
