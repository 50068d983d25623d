"""Refusals of the 8-bit rows', norms', tables' and verification's entry points (no GPU
needed: every call is refused before any launch)."""

import ctypes as C
import types

import pytest

from paper_2608_30384_amd import _lib as L

torch = pytest.importorskip("torch")

P = C.c_void_p(0x10000)      # aligned, never read
Q = C.c_void_p(0x10001)      # not aligned to anything
Z = C.c_void_p(0)
BIG = 2 ** 31 - 255


def test_8_bit_rows():
    lib = L.lib()
    ok = [Z, P, 0, 4, 96, 96, P, P, Z]
    for at, bad in ((1, Z), (1, Q), (2, 3), (2, -1), (3, -1), (3, BIG), (4, 0), (4, 65537), (5, -1), (6, Z), (6, C.c_void_p(8)),
                    (7, Q)):
        assert lib.rslm_mx8_quantize(*[bad if i == at else v for i, v in enumerate(ok)]) == 1, at
    ok = [P, P, 4, 96, P, 0, 96, Z]
    for at, bad in ((0, Z), (0, C.c_void_p(8)), (1, Q), (2, -1), (2, BIG), (3, 0), (3, 65537), (4, Z), (4, Q), (5, 7), (6, 95)):
        assert lib.rslm_mx8_dequantize(*[bad if i == at else v for i, v in enumerate(ok)]) == 1, at
    ok = [P, P, 4, P, P, 5, 96, P, 0, 5, Z]
    for at, bad in ((0, Z), (0, C.c_void_p(8)), (1, Q), (2, -1), (2, 4194241), (3, Z), (4, Z), (4, Q), (5, -1), (5, BIG), (6, 0),
                    (6, 65537), (7, Q), (8, 3), (9, 4)):
        assert lib.rslm_mx8_score(*[bad if i == at else v for i, v in enumerate(ok)]) == 1, at
    assert lib.rslm_mx8_score(Z, Z, 0, Z, Z, 5, 96, Z, 0, 5, Z) == 0


def test_norm():
    lib = L.lib()
    ok = [P, 0, 4, 96, 96, P, 96, P, 0, 1e-6, P, 96, P, 96, P, P, P, Z]
    nan, inf = float("nan"), float("inf")
    for at, bad in ((0, Z), (0, Q), (1, 3), (2, -1), (2, BIG), (3, 0), (3, 65537), (4, -1), (5, Q), (6, -1), (7, Q), (8, 3), (9, 0.0),
                    (9, -1.0), (9, nan), (9, inf), (10, Z), (10, Q), (11, 95), (12, Q), (13, 95), (14, Z), (14, C.c_void_p(8)), (15, Z),
                    (16, Z), (16, Q)):
        assert lib.rslm_rmsnorm(*[bad if i == at else v for i, v in enumerate(ok)]) == 1, at
    size = lib.rslm_rmsnorm_backward_workspace(4, 96)
    ok = [P, 0, 4, 96, 96, P, 96, P, P, 0, P, 96, P, 96, P, P, size, Z]
    for at, bad, want in ((0, Z, 1), (0, Q, 1), (1, 3, 1), (2, -1, 1), (3, 0, 1), (4, -1, 1), (5, Z, 1), (6, -1, 1), (7, Z, 1), (8, Q, 1),
                          (9, 4, 1), (10, Q, 1), (11, -1, 1), (12, Q, 1), (13, 95, 1), (14, Q, 1), (15, Z, 1), (15, C.c_void_p(8), 1),
                          (16, size - 1, 4)):
        assert lib.rslm_rmsnorm_backward(*[bad if i == at else v for i, v in enumerate(ok)]) == want, at
    assert lib.rslm_rmsnorm(Z, 0, 0, 96, 96, Z, 96, Z, 0, 1e-6, Z, 96, Z, 96, Z, Z, Z, Z) == 0


def test_tables():
    lib = L.lib()
    ok = [P, 0, 50, 96, 96, P, 8, 4, 1.0, P, 0, 96, Z]
    for at, bad in ((0, Z), (0, Q), (1, 3), (2, -1), (2, BIG), (3, 0), (3, 65537), (4, -1), (5, Z), (5, C.c_void_p(0x10004)), (6, 2),
                    (7, -1), (7, BIG), (9, Z), (9, Q), (10, 5), (11, 95)):
        assert lib.rslm_embed(*[bad if i == at else v for i, v in enumerate(ok)]) == 1, at
    ok = [P, P, 50, 96, P, 4, 4, 1.0, P, 0, 96, Z]
    for at, bad in ((0, Z), (0, C.c_void_p(8)), (1, Z), (1, Q), (2, -1), (3, 0), (4, Z), (4, C.c_void_p(0x10002)), (5, 16), (6, -1),
                    (8, Q), (9, -1), (10, 95)):
        assert lib.rslm_mx4_embed(*[bad if i == at else v for i, v in enumerate(ok)]) == 1, at
    size = lib.rslm_embed_backward_workspace(4, 50, 96)
    ok = [P, 1, 4, 96, 96, P, 8, 50, 1.0, 0, P, 1, 96, P, size, Z]
    for at, bad, want in ((0, Z, 1), (0, Q, 1), (1, 3, 1), (2, -1, 1), (2, BIG, 1), (3, 0, 1), (4, -1, 1), (5, Z, 1), (6, 3, 1), (7, -1, 1),
                          (7, BIG, 1), (10, Z, 1), (10, Q, 1), (11, 2, 2), (11, 9, 1), (12, 95, 1), (13, Z, 1), (13, C.c_void_p(8), 1),
                          (14, size - 1, 4)):
        assert lib.rslm_embed_backward(*[bad if i == at else v for i, v in enumerate(ok)]) == want, at
    # sizes at the ends have a workspace, and one that grows with them
    assert lib.rslm_embed_backward_workspace(BIG - 1, BIG - 1, 65536) > lib.rslm_embed_backward_workspace(BIG - 1, 1, 1) > 16 * (BIG - 1)
    assert lib.rslm_embed_backward_workspace(0, 50, 96) == 0


def test_verification():
    lib = L.lib()
    size = lib.rslm_verify_workspace(3, 2, 100, 1)
    nan, big = float("nan"), 2.4e38
    ok = [P, 0, 3, 2, 100, 300, 100, 1.0, P, 200, 100, 1.0, P, P, P, P, P, P, P, size, Z]
    for at, bad, want in ((0, Z, 1), (0, Q, 1), (1, 3, 1), (2, -1, 1), (3, -1, 1), (3, 65, 1), (4, 0, 1), (4, 2 ** 31 - 1, 1), (5, -1, 1),
                          (6, -1, 1), (7, 0.0, 1), (7, -1.0, 1), (7, nan, 1), (7, big, 1), (8, Q, 1), (9, -1, 1), (10, -1, 1), (11, 0.0, 1),
                          (11, big, 1), (12, Z, 1), (12, C.c_void_p(0x10004), 1), (13, Z, 1), (13, Q, 1), (14, Q, 1), (15, Z, 1), (15, Q, 1),
                          (16, Z, 1), (17, Q, 1), (18, Z, 1), (18, C.c_void_p(8), 1), (19, size - 1, 4)):
        assert lib.rslm_verify(*[bad if i == at else v for i, v in enumerate(ok)]) == want, at
    assert lib.rslm_verify(Z, 0, 2 ** 23, 0, 100, 100, 100, 1.0, Z, 0, 0, 1.0, Z, Z, Z, Z, Z, Z, Z, 0, Z) == 1
    assert lib.rslm_verify(Z, 0, 0, 2, 100, 0, 0, 1.0, Z, 0, 0, 1.0, Z, Z, Z, Z, Z, Z, Z, 0, Z) == 0


# ------------------------------------------------------------------ from Python, without a device
class Fake:
    """What the checks look at of a device tensor."""

    is_cuda, requires_grad = True, False

    def __init__(self, shape, dtype=torch.float32, device=0, stride=None, grad=False):
        self.shape, self.dtype, self.device, self.requires_grad = torch.Size(shape), dtype, torch.device("cuda", device), grad
        self._stride = stride or tuple(int(torch.Size(shape[i + 1:]).numel()) for i in range(len(shape)))

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self._stride if i is None else self._stride[i]

    def is_contiguous(self):
        return self._stride == tuple(int(torch.Size(self.shape[i + 1:]).numel()) for i in range(len(self.shape)))

    def data_ptr(self):
        raise AssertionError("a call that has to be refused came to its launch")


I64 = torch.int64


def rows_of(kind, n, dim, device=0):
    from paper_2608_30384_amd import api

    r = getattr(api, kind).__new__(getattr(api, kind))
    steps = -(-dim // 128)
    r.codes = Fake((n, r._bytes * steps), torch.uint8, device)
    r.scales, r.dim = Fake((n, 4 * steps), torch.uint8, device), dim
    return r


def test_python_refusals(monkeypatch):
    from paper_2608_30384_amd import api

    x, w, h = Fake((4, 96)), Fake((96,)), Fake((4, 96))
    a, b, ids = rows_of("Mx8Rows", 4, 96), rows_of("Mx4Rows", 9, 96), Fake((4,), I64)
    norm = types.SimpleNamespace(h=h, rstd=Fake((4,)))
    z, tokens, u = Fake((2, 3, 50)), Fake((2, 2), I64), Fake((2, 3))
    for error, call in (
            # rows of the other kind would be read past their end
            (TypeError, lambda: api.rslm_mx8_score(b, b)),
            (TypeError, lambda: api.rslm_mx8_score(a, a)),
            (TypeError, lambda: api.rslm_mx8_dequantize(b)),
            (TypeError, lambda: api.rslm_mx4_dequantize(a)),
            (TypeError, lambda: api.rslm_mx4_matmul(a, b)),
            (TypeError, lambda: api.rslm_mx4_matmul(b, a)),
            (TypeError, lambda: api.rslm_mx4_score(x, a)),
            (TypeError, lambda: api.rslm_mx4_score_backward(Fake((4, 4)), a)),
            (TypeError, lambda: api.rslm_mx8_quantize(x, rows=b)),
            (TypeError, lambda: api.rslm_mx4_quantize(x, rows=a)),
            (ValueError, lambda: api.rslm_mx8_quantize(x, rows=rows_of("Mx8Rows", 5, 96))),
            (ValueError, lambda: api.rslm_mx8_score(a, rows_of("Mx4Rows", 9, 97))),
            (ValueError, lambda: api.rslm_mx8_score(a, rows_of("Mx4Rows", 9, 96, 1))),
            (ValueError, lambda: api.rslm_mx8_score(a, b, out=Fake((4, 8)))),
            (TypeError, lambda: api.rslm_mx8_score(a, b, dtype=torch.float64)),
            # norms
            (ValueError, lambda: api.rslm_rmsnorm(Fake((96,)))),
            (TypeError, lambda: api.rslm_rmsnorm(Fake((4, 96), torch.float64))),
            (ValueError, lambda: api.rslm_rmsnorm(Fake((4, 0)))),
            (ValueError, lambda: api.rslm_rmsnorm(Fake((4, 96), stride=(1, 4)))),
            (ValueError, lambda: api.rslm_rmsnorm(x, Fake((95,)))),
            (ValueError, lambda: api.rslm_rmsnorm(x, Fake((96,), stride=(2,)))),
            (ValueError, lambda: api.rslm_rmsnorm(x, Fake((96,), device=1))),
            (TypeError, lambda: api.rslm_rmsnorm(x, residual=Fake((4, 96), torch.float16))),
            (ValueError, lambda: api.rslm_rmsnorm(x, residual=Fake((3, 96)))),
            (ValueError, lambda: api.rslm_rmsnorm(x, h=h)),
            (TypeError, lambda: api.rslm_rmsnorm(x, residual=x, h=Fake((4, 96), torch.float16))),
            (ValueError, lambda: api.rslm_rmsnorm(Fake((4, 96), grad=True))),
            (ValueError, lambda: api.rslm_rmsnorm(x, Fake((96,), grad=True))),
            (TypeError, lambda: api.rslm_rmsnorm_backward(Fake((4, 96), torch.float16), norm)),
            (ValueError, lambda: api.rslm_rmsnorm_backward(Fake((5, 96)), norm)),
            (ValueError, lambda: api.rslm_rmsnorm_backward(x, types.SimpleNamespace(h=h, rstd=Fake((3,))))),
            (ValueError, lambda: api.rslm_rmsnorm_backward(x, norm, Fake((97,)))),
            (ValueError, lambda: api.rslm_rmsnorm_backward(x, norm, w, dh=Fake((4, 95)))),
            (ValueError, lambda: api.rslm_rmsnorm_backward(x, norm, w, dh=Fake((4, 96), grad=True))),
            # tables
            (TypeError, lambda: api.rslm_embed(x, Fake((4,)))),
            (ValueError, lambda: api.rslm_embed(x, Fake((4, 1), I64))),
            (ValueError, lambda: api.rslm_embed(x, Fake((4,), I64, device=1))),
            (ValueError, lambda: api.rslm_embed(b, Fake((4,), I64, device=1))),
            (ValueError, lambda: api.rslm_embed(x, Fake((4,), I64, stride=(2,)))),
            (ValueError, lambda: api.rslm_embed(Fake((4, 96), grad=True), ids)),
            (ValueError, lambda: api.rslm_embed(x, ids, out=Fake((4, 95)))),
            (TypeError, lambda: api.rslm_embed(a, ids)),
            (ValueError, lambda: api.rslm_embed_backward(x, Fake((5,), I64), 50)),
            (ValueError, lambda: api.rslm_embed_backward(x, ids, 50, accumulate=True)),
            (ValueError, lambda: api.rslm_embed_backward(x, ids, 50, out=Fake((49, 96)))),
            (ValueError, lambda: api.rslm_embed_backward(Fake((4, 96), grad=True), ids, 50)),
            # drafted tokens
            (ValueError, lambda: api.rslm_verify(Fake((2, 50)), tokens, u)),
            (ValueError, lambda: api.rslm_verify(Fake((2, 66, 50)), Fake((2, 65), I64), Fake((2, 66)))),
            (ValueError, lambda: api.rslm_verify(Fake((2, 0, 50)), tokens, u)),
            (ValueError, lambda: api.rslm_verify(Fake((2, 3, 0)), tokens, u)),
            (ValueError, lambda: api.rslm_verify(Fake((2, 3, 50), stride=(150, 1, 3)), tokens, u)),
            (TypeError, lambda: api.rslm_verify(z, Fake((2, 2), torch.int32), u)),
            (ValueError, lambda: api.rslm_verify(z, Fake((2, 3), I64), u)),
            (ValueError, lambda: api.rslm_verify(z, tokens, Fake((2, 2)))),
            (TypeError, lambda: api.rslm_verify(z, tokens, u, counts=Fake((2,), I64))),
            (ValueError, lambda: api.rslm_verify(z, tokens, u, counts=Fake((3,), torch.int32))),
            (TypeError, lambda: api.rslm_verify(z, tokens, u, draft=Fake((2, 2, 50), torch.float16))),
            (ValueError, lambda: api.rslm_verify(z, tokens, u, draft=Fake((2, 3, 50)))),
            (ValueError, lambda: api.rslm_verify(z, tokens, Fake((2, 3), device=1))),
            (ValueError, lambda: api.rslm_verify(Fake((2, 3, 50), grad=True), tokens, u))):
        with pytest.raises(error):
            call()
