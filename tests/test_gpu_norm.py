"""The root-mean-square norm on the GPU against float64.

Tolerances.  rstd: no thread of the kernels adds more than 64 + dim / 128 squares one
after the other, and its sum goes through at most 16 additions more; all terms are
positive, so the mean is off by at most D = 80 + dim / 128 units of 2^-24, rstd by half of
that and 4 roundings, y by 2 more and half a unit of its type.  mean(g u) is off by D + 8
units (times 2^-24) of mean |g u|.  dweight sums n terms, each of 3 roundings: n + 8 units
of the sum of their magnitudes, for any order.
"""

import numpy as np
import pytest

from oracle import mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
U = 2.0 ** -24


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def f64(t):
    return t.double().cpu().numpy()


def wide(g, n, dim, extra, dt, amp=1.0):
    t = (amp * torch.randn((n, dim + extra), generator=g)).to(DT[dt]).cuda()
    return t[:, :dim]


def depth(dim):
    return 80 + dim / 128


def check_forward(r, x, residual, weight, dt, eps, rows):
    dim = x.shape[1]
    h = x.cpu() if residual is None else (x.cpu().float() + residual.cpu().float()).to(DT[dt])
    assert torch.equal(r.h.cpu(), h)
    w = np.ones(dim) if weight is None else f64(weight)
    y, rstd = mx8.rmsnorm(f64(h), w, eps)
    assert (np.abs(f64(r.rstd) - rstd) <= (depth(dim) / 2 + 4) * U * rstd).all()
    tol = (depth(dim) / 2 + 6) * U * np.abs(y)
    if r.y is not None:
        least = 2.0 ** -25 if dt == "f16" else 0.0
        assert (np.abs(f64(r.y) - y) <= tol + HALF[dt] * (np.abs(y) + tol) + least).all()
    if rows:
        got = mx8.values(r.rows.codes.cpu().numpy(), r.rows.scales.cpu().numpy(), dim)
        scale = np.ldexp(1.0, r.rows.scales.cpu().numpy().astype(int) - 127)
        unit = np.repeat(scale, 32, axis=1)[:, :dim] * 2.0 ** -10
        assert (np.abs(got - y) <= np.maximum(2.0 ** -4 * (np.abs(y) + tol), unit) + tol).all()
        top = np.abs(np.pad(y, ((0, 0), (0, -dim % 128)))).reshape(len(y), -1, 32).max(-1)
        assert (top * (1 - (depth(dim) / 2 + 8) * U) <= 448 * scale).all()
        assert ((top * (1 + (depth(dim) / 2 + 8) * U) > 224 * scale) | (r.rows.scales.cpu().numpy() == 0)).all()
        assert (r.rows.codes.cpu().numpy()[:, dim:] == 0).all()


SIZES = [(1, 1, 0), (2, 7, 1), (5, 8, 0), (3, 33, 2), (40, 96, 0), (17, 128, 0), (9, 129, 7), (4, 512, 0), (33, 768, 1),
         (1, 1024, 0), (300, 2049, 15), (2, 2048, 0), (1, 4096, 0), (3, 4100, 3), (2, 8192, 0), (1, 8200, 0), (2, 16384, 0),
         (1, 16392, 1), (1, 20001, 0), (1, 65536, 0), (3, 1100, 0), (2, 5120, 1), (2, 9000, 3), (1, 12288, 0), (1100, 640, 1)]


@pytest.mark.parametrize("dt,wt", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("n,dim,extra", SIZES)
def test_forward_and_gradient(R, dt, wt, n, dim, extra):
    g = torch.Generator().manual_seed(n + dim)
    eps = 1e-5
    x, residual = wide(g, n, dim, extra, dt), wide(g, n, dim, 2 * extra, dt, 2.0)
    weight = (1 + 0.3 * torch.randn((dim,), generator=g)).to(DT[wt]).cuda()
    r = R.rslm_rmsnorm(x, weight, residual=residual, eps=eps, rows=True)
    check_forward(r, x, residual, weight, dt, eps, True)
    plain = R.rslm_rmsnorm(x, eps=eps, y=False, rows=True)
    assert plain.y is None and plain.h is x
    check_forward(plain, x, None, None, dt, eps, True)

    dy, dh = wide(g, n, dim, extra, dt), wide(g, n, dim, 0, dt)
    for w, dhs in ((weight, dh), (weight, None), (None, dh)):
        dx, dw = R.rslm_rmsnorm_backward(dy, r, w, dh=dhs)
        h, rstd = f64(r.h), f64(r.rstd)[:, None]
        w64, dh64 = np.ones(dim) if w is None else f64(w), 0.0 if dhs is None else f64(dhs)
        u, gg = h * rstd, f64(dy) * w64
        mean, size = (gg * u).mean(1, keepdims=True), np.abs(gg * u).mean(1, keepdims=True)
        want = rstd * (gg - u * mean) + dh64
        tol = U * (rstd * (4 * np.abs(gg) + np.abs(u) * ((depth(dim) + 8) * size + 4 * np.abs(mean))) + 2 * np.abs(want) + np.abs(dh64))
        tol = tol + HALF[dt] * (np.abs(want) + tol) + (2.0 ** -25 if dt == "f16" else 0.0)
        assert (np.abs(f64(dx) - want) <= tol).all()
        if w is None:
            assert dw is None
            continue
        terms = np.abs(f64(dy) * u).sum(0)
        tol = U * (n + 8) * terms
        want = (f64(dy) * u).sum(0)
        tol = tol + HALF[wt] * (np.abs(want) + tol) + (2.0 ** -25 if wt == "f16" else 0.0)
        assert dw.dtype == DT[wt] and (np.abs(f64(dw) - want) <= tol).all()
    # the kernel's formula is the derivative: against the oracle's, which is checked by differences
    dx64, _ = mx8.rmsnorm_grad(f64(r.h), f64(weight), eps, f64(dy), f64(dh))
    dx, _ = R.rslm_rmsnorm_backward(dy, r, weight, dh=dh)
    assert np.abs(f64(dx) - dx64).max() <= 2 * HALF[dt] * np.abs(dx64).max() + 1e-5 * np.abs(dx64).max()


@pytest.mark.parametrize("n,dim", [(700, 64), (5000, 96), (2000, 300), (1500, 1024), (1030, 2049), (600, 4096), (1300, 1100), (300, 5120), (270, 9000)])
def test_many_rows(R, n, dim):
    """More rows than workgroups: every row and every row's part of dweight, in bfloat16
    whose 8-bit rows are those of the float32 norm."""
    g = torch.Generator().manual_seed(n)
    x, dy = wide(g, n, dim, 0, "f32"), wide(g, n, dim, 0, "f32")
    weight = (1 + 0.3 * torch.randn((dim,), generator=g)).cuda()
    r = R.rslm_rmsnorm(x, weight, rows=True)
    check_forward(r, x, None, weight, "f32", 1e-6, True)
    c, s = mx8.quantize(f64(r.y))
    pc, ps = mx8.pack(c, s, dim)
    got = r.rows.codes.cpu().numpy()
    assert np.array_equal(r.rows.scales.cpu().numpy(), ps) and ((got == pc) | (((got | pc) & 127) == 0)).all()
    dx, dw = R.rslm_rmsnorm_backward(dy, r, weight)
    u = f64(x) * f64(r.rstd)[:, None]
    assert (np.abs(f64(dw) - (f64(dy) * u).sum(0)) <= U * (n + 9) * np.abs(f64(dy) * u).sum(0)).all()
    again = R.rslm_rmsnorm_backward(dy, r, weight)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])


@pytest.mark.parametrize("dim", [5, 40, 768, 4096, 8200, 16392])
def test_in_place(R, dim):
    g = torch.Generator().manual_seed(dim)
    x, residual = wide(g, 6, dim, 0, "bf16"), wide(g, 6, dim, 0, "bf16")
    want = R.rslm_rmsnorm(x, residual=residual, rows=True)
    for into in (0, 1):
        both = [x.clone(), residual.clone()]
        got = R.rslm_rmsnorm(both[0], residual=both[1], rows=True, h=both[into])
        assert got.h is both[into] and torch.equal(got.h, want.h) and torch.equal(got.y, want.y)
        assert torch.equal(got.rows.codes, want.rows.codes) and torch.equal(got.rstd, want.rstd)
    # the gradient into dy, dh or h, whose other readers (the weight's gradient) come first
    dy, weight = wide(g, 6, dim, 0, "bf16"), torch.rand((dim,), generator=g).cuda()
    dx, dw = R.rslm_rmsnorm_backward(dy, want, weight, dh=x)
    for into in range(3):
        all3 = [dy.clone(), x.clone(), want.h.clone()]
        again = type(want)(all3[2], None, None, want.rstd)
        got = R.rslm_rmsnorm_backward(all3[0], again, weight, dh=all3[1], out=all3[into])
        assert got[0] is all3[into] and torch.equal(got[0], dx) and torch.equal(got[1], dw)


def test_rows_of_zeros_and_of_no_numbers(R):
    x = torch.randn((6, 300), device="cuda")
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 299] = float("inf")
    x[4] = 1e18
    r = R.rslm_rmsnorm(x, eps=1e-6, rows=True)
    values = R.rslm_mx8_dequantize(r.rows)
    assert (r.y[1] == 0).all() and (values[1] == 0).all() and abs(float(r.rstd[1]) - 1e3) < 1e-3
    assert r.y[2].isnan().all() and values[2].isnan().all()
    assert r.y[3, 299].isnan() and (r.y[3, :299] == 0).all()
    assert (r.y[4] - 1).abs().max() < 1e-5
    clean = R.rslm_rmsnorm(x[[0, 5]].contiguous(), eps=1e-6)
    assert torch.equal(r.y[[0, 5]], clean.y)


def test_no_rows(R):
    x, w = torch.empty((0, 50), device="cuda"), torch.ones((50,), device="cuda")
    r = R.rslm_rmsnorm(x, w, residual=x, rows=True)
    assert r.h.shape == r.y.shape == (0, 50) and r.rows.n == 0
    dx, dw = R.rslm_rmsnorm_backward(x, r, w)
    assert dx.shape == (0, 50) and (dw == 0).all()


def test_other_stream(R):
    x, w = torch.randn((70, 768), device="cuda"), torch.rand((768,), device="cuda")
    want = R.rslm_rmsnorm(x, w, residual=x, rows=True)
    grads = R.rslm_rmsnorm_backward(x, want, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = R.rslm_rmsnorm(x, w, residual=x, rows=True, stream=s)
    back = R.rslm_rmsnorm_backward(x, got, w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got.y, want.y) and torch.equal(got.rows.codes, want.rows.codes)
    assert torch.equal(back[0], grads[0]) and torch.equal(back[1], grads[1])


def test_captured(R):
    x, w, dy = torch.randn((300, 768), device="cuda"), torch.rand((768,), device="cuda"), torch.randn((300, 768), device="cuda")
    h, dx = torch.empty_like(x), torch.empty_like(x)

    def step():
        r = R.rslm_rmsnorm(x, w, residual=dy, h=h, rows=True)
        return r, R.rslm_rmsnorm_backward(dy, r, w, out=dx)[1]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, dw = step()
    for seed in range(3):
        x.copy_(torch.randn((300, 768), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        got = [t.clone() for t in (r.y, r.rows.codes, dx, dw)]
        e = R.rslm_rmsnorm(x, w, residual=dy, rows=True)
        edx, edw = R.rslm_rmsnorm_backward(dy, e, w)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, (e.y, e.rows.codes, edx, edw)))
