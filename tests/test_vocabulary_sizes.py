"""Numbers of sequences whose products pass 64 bits are refused as large ones are (no GPU
needed: nothing is launched)."""

import ctypes as C

import pytest

from paper_2608_30384_amd import _lib as L

P = C.c_void_p(0x10000)      # aligned, never read
Z = C.c_void_p(0)


def sequences(k):
    """Numbers b below 2^63 whose product with 2 k + 1 is small in 64 bits."""
    inverse = pow(2 * k + 1, -1, 2 ** 64)
    return [b for b in (inverse * p % 2 ** 64 for p in range(1, 9)) if 2 ** 32 < b < 2 ** 63]


@pytest.mark.parametrize("k", [1, 2, 4, 63, 64])
def test_verification(k):
    lib = L.lib()
    some = sequences(k)
    assert some
    for b in some + [2 ** 63 - 1, 2 ** 40, 0x7fffffff // 256 // (2 * k + 1) + 1]:
        assert lib.rslm_verify_workspace(b, k, 100, 1) == 0, b
        assert lib.rslm_verify(P, 0, b, k, 100, 0, 0, 1.0, P, 0, 0, 1.0, P, P, Z, P, P, Z, P, 0, Z) == 1, b
    assert lib.rslm_verify_workspace(0x7fffffff // 256 // (2 * k + 1), k, 100, 1) > 0
