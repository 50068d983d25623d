"""Tensors that reach past 2^31 elements and 4 GiB from their start."""

import numpy as np
import pytest

from oracle import mx4, mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def far(shape, strides, seed):
    """A bfloat16 tensor of these strides, with numbers."""
    size = 1 + sum((n - 1) * s for n, s in zip(shape, strides))
    t = torch.empty((size,), dtype=torch.bfloat16, device="cuda").as_strided(shape, strides)
    t.copy_(torch.randn(shape, generator=torch.Generator().manual_seed(seed)))
    return t


def test_norm(R):
    n, dim, stride = 3, 300, 1_500_000_000
    x, residual, dy = (far((n, dim), (stride, 1), i) for i in range(3))
    near = [t.contiguous() for t in (x, residual, dy)]
    want = R.rslm_rmsnorm(near[0], residual=near[1], rows=True)
    dwant, _ = R.rslm_rmsnorm_backward(near[2], want, dh=near[1])
    got = R.rslm_rmsnorm(x, residual=residual, rows=True, h=x)
    assert torch.equal(x, want.h) and torch.equal(got.y, want.y) and torch.equal(got.rows.codes, want.rows.codes)
    dx, _ = R.rslm_rmsnorm_backward(dy, got, dh=residual, out=dy)
    assert torch.equal(dy, dwant)


def test_embed(R):
    rows, dim, stride = 4, 200, 1_100_000_000
    table = far((rows, dim), (stride, 1), 0)
    ids = torch.tensor([3, 0, 2, 3, -1], device="cuda")
    out = far((5, dim), (700_000_000, 1), 1)
    R.rslm_embed(table, ids, out=out)
    assert torch.equal(out[:4], table[ids[:4]]) and (out[4] == 0).all()
    grad = R.rslm_embed_backward(out, ids, rows, out=table)
    near = R.rslm_embed_backward(out.contiguous(), ids, rows)
    assert grad is table and torch.equal(table, near)


def test_verify(R):
    b, k, n = 2, 1, 1000
    z, d = far((b, k + 1, n), (2_400_000_000, 1_200_000_000, 1), 0), far((b, k, n), (2_400_000_000, 5, 1), 1)
    tokens, u = torch.tensor([[3], [999]]), torch.rand((b, k + 1), generator=torch.Generator().manual_seed(2))
    r = R.rslm_verify(z, tokens.cuda(), u.cuda(), draft=d)
    want = mx8.verify(z.double().cpu().numpy(), tokens.numpy(), u.numpy(), d.double().cpu().numpy())
    assert np.array_equal(r.tokens.cpu().numpy(), want[0]) and np.array_equal(r.accepted.cpu().numpy(), want[1])


def random_rows(kind, n, dim, seed):
    """Rows of random codes of both kinds, and scales near 1."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = kind.empty(n, dim, torch.device("cuda", 0))
    r.codes.random_(0, 256, generator=g)
    r.codes.bitwise_and_(0xBB)      # neither NaN (8 bits) nor of the largest exponents
    r.scales.random_(126, 129, generator=g)
    return r


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n", [(1, 140_000), (20, 140_000), (70_000, 20), (16, 140_000)])
def test_score(R, m, n, dtype):
    """65,536 coordinates: 32 KiB a row of 4-bit codes, 64 KiB of 8-bit ones."""
    dim = 65536
    a, b = random_rows(R.Mx8Rows, m, dim, 1), random_rows(R.Mx4Rows, n, dim, 2)
    assert max(a.codes.numel(), b.codes.numel()) > 1 << 32
    got = R.rslm_mx8_score(a, b, dtype=dtype)
    i, j = sorted({0, m // 2, m - 1}), sorted({0, n // 2, n - 2, n - 1})
    x = mx8.values(a.codes[i].cpu().numpy(), a.scales[i].cpu().numpy(), dim)
    y = mx4.values(b.codes[j].cpu().numpy(), b.scales[j].cpu().numpy(), dim)
    want, terms = x @ y.T, np.abs(x) @ np.abs(y).T
    tol = 2 * (3 * dim + 16) * 2.0 ** -24 * terms
    if dtype == torch.bfloat16:
        tol = tol + 7 * 2.0 ** -13 * terms
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    assert (np.abs(got[i][:, j].double().cpu().numpy() - want) <= tol).all()
