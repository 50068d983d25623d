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


def test_tensors_and_streams_of_another_device(monkeypatch):
    """A launch goes to the current device, whatever its tensors are on."""
    import types

    import torch

    from paper_2608_30384_amd import api

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)
    here, other = torch.device("cuda", 0), torch.device("cuda", 1)
    s0, s1 = (types.SimpleNamespace(device_index=i, cuda_stream=200 + i) for i in (0, 1))
    assert api._launch_stream(None, here) == 100 and api._launch_stream(s0, here) == 200
    for stream, device in ((None, other), (s1, other), (s1, here), (s0, other)):
        with pytest.raises(ValueError, match="current device"):
            api._launch_stream(stream, device)

    class Rows:
        is_cuda, dtype, shape, device = True, torch.float32, (4, 96), here
        dim, stride = (lambda self: 2), (lambda self, i=0: (96, 1)[i])

    with pytest.raises(ValueError, match="plan's device"):
        api.rslm_mx4_quantize(Rows(), types.SimpleNamespace(dim=96, device=other))
