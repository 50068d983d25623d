"""Rows of 4 bits in an object of the caller's own, with the attributes that the calls read,
are taken as they are; what holds too little, or is no rows at all, is refused.  No GPU needed."""

import types

import pytest

torch = pytest.importorskip("torch")

from paper_2608_30384_amd import api

from .test_written_tensors import DIM, N, ROWS, library, t  # noqa: F401

U8 = torch.uint8


def own(n, dim=DIM, codes=64, scales=4, flat=False):
    steps = -(-dim // 128)
    c, s = t(n, codes * steps, dtype=U8), t(n, scales * steps, dtype=U8)
    return types.SimpleNamespace(codes=c.view(-1) if flat else c, scales=s.view(-1) if flat else s, n=n, dim=dim, device=c.device)


CALLS = {
    "quantize": lambda r: api.rslm_mx4_quantize(t(N, DIM), rows=r(N)),
    "dequantize": lambda r: api.rslm_mx4_dequantize(r(N)),
    "matmul": lambda r: api.rslm_mx4_matmul(r(N), r(ROWS)),
    "score": lambda r: api.rslm_mx4_score(t(N, DIM), r(ROWS)),
    "score_backward": lambda r: api.rslm_mx4_score_backward(t(N, ROWS), r(ROWS)),
}


@pytest.mark.parametrize("name", CALLS)
def test_rows_of_another_class(name):
    call = CALLS[name]
    call(own)
    call(lambda n: own(n, flat=True))
    call(lambda n: own(n, codes=65))        # room for more
    for small in (dict(codes=63), dict(scales=3)):
        with pytest.raises(ValueError, match="hold"):
            call(lambda n: own(n, **small))
    for none in (torch.zeros(N, 64, dtype=U8), (1, 2), None):
        if name != "quantize" or none is not None:
            with pytest.raises(TypeError):
                call(lambda n: none)
    # the other kind's rows, whose class says so
    with pytest.raises(TypeError):
        call(lambda n: api.Mx8Rows(t(n, 128, dtype=U8), t(n, 4, dtype=U8), DIM))


def test_8_bit_rows_of_another_class():
    a = lambda codes: types.SimpleNamespace(**vars(own(N, codes=codes)))
    api.rslm_mx8_score(a(128), own(ROWS))
    with pytest.raises(ValueError, match="hold"):
        api.rslm_mx8_score(a(64), own(ROWS))
