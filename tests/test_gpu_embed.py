"""Rows of tables for given ids, and the table's gradient, on the GPU.

The rows are exact: one float32 product, rounded once.  Gradients of whole numbers whose
sums float32 holds are exact too, whatever the order; of others a row with c terms is off
by at most (c + 2) 2^-24 of the sum of their magnitudes, and half a unit of its type.
"""

import numpy as np
import pytest

from oracle import mx4, mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def some_ids(kind, n, rows, seed):
    rng = np.random.default_rng(seed)
    if kind == "one":
        return np.full(n, rows // 2)
    if kind == "none":
        return np.full(n, -1)
    if kind == "sorted":
        return np.sort(rng.integers(0, rows, n))
    if kind == "falling":
        return np.sort(rng.integers(0, rows, n))[::-1].copy()
    if kind == "outside":
        return rng.choice([-1, -5, 0, rows - 1, rows, rows + 1, 2 ** 31 - 1, -2 ** 31], n)
    if kind == "few":
        return rng.integers(0, min(rows, 3), n)
    ids = np.minimum(np.exp(rng.uniform(0, np.log(rows + 1), n)).astype(np.int64) - 1, rows - 1)
    return np.where(rng.random(n) < 0.05, -1, ids)


@pytest.mark.parametrize("it", [torch.int32, torch.int64])
@pytest.mark.parametrize("dt,to", [("f32", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("n,rows,dim,extra", [(1, 1, 1, 0), (5, 3, 7, 2), (64, 100, 96, 0), (17, 50, 128, 1), (300, 9, 129, 0),
                                              (33, 1000, 768, 5), (2, 40, 2049, 0), (1000, 20, 520, 0), (1, 2, 65536, 0)])
def test_lookup(R, it, dt, to, n, rows, dim, extra):
    g = torch.Generator().manual_seed(n + dim)
    table = torch.randn((rows, dim + extra), generator=g).to(DT[dt])[:, :dim]
    ids = torch.from_numpy(some_ids("outside" if n > 3 else "zipf", n, rows, n)).to(it)
    on = (ids >= 0) & (ids < rows)
    want = torch.where(on[:, None], table[ids.long().clamp(0, rows - 1)].float() * 1.7, 0.0).to(DT[to])
    out = torch.full((n, dim + 2), 3.0, dtype=DT[to], device="cuda")
    got = R.rslm_embed(table.cuda(), ids.cuda(), scale=1.7, dtype=DT[to], out=out[:, :dim])
    assert torch.equal(got.cpu(), want) and (out[:, dim:] == 3).all()


@pytest.mark.parametrize("to", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,rows,dim", [(1, 1, 1), (7, 5, 33), (64, 300, 96), (40, 9, 129), (256, 1000, 768), (3, 4, 2049)])
def test_lookup_of_4_bit_rows(R, to, n, rows, dim):
    g = torch.Generator(device="cuda").manual_seed(n + dim)
    table = R.rslm_mx4_quantize(torch.randn((rows, dim), generator=g, device="cuda"))
    ids = torch.from_numpy(some_ids("outside" if n > 3 else "zipf", n, rows, n))
    on = (ids >= 0) & (ids < rows)
    values = torch.from_numpy(mx4.values(table.codes.cpu().numpy(), table.scales.cpu().numpy(), dim)).float()
    want = torch.where(on[:, None], values[ids.clamp(0, rows - 1)] * 0.3, 0.0).to(DT[to])
    got = R.rslm_embed(table, ids.cuda(), scale=0.3, dtype=DT[to])
    assert torch.equal(got.cpu(), want)
    assert R.rslm_embed(table, ids.cuda()).dtype == torch.float32


def test_lookup_of_nothing(R):
    table = torch.randn((5, 12), device="cuda")
    assert R.rslm_embed(table, torch.empty((0,), dtype=torch.int64, device="cuda")).shape == (0, 12)
    ids = torch.tensor([0, -1, 3], device="cuda")
    assert (R.rslm_embed(torch.empty((0, 12), device="cuda"), ids) == 0).all()
    assert (R.rslm_embed(R.Mx4Rows.empty(0, 12, "cuda"), ids) == 0).all()
    # rows that overlap
    one = torch.randn((12,), device="cuda")
    assert torch.equal(R.rslm_embed(one.expand(4, 12), ids)[2], one)


def whole(rng, n, dim):
    return rng.integers(-8, 9, (n, dim)).astype(np.float32)


@pytest.mark.parametrize("kind", ["zipf", "one", "none", "sorted", "falling", "outside", "few"])
@pytest.mark.parametrize("n,rows,dim", [(1, 1, 1), (2, 5, 8), (63, 4, 7), (64, 700, 96), (65, 511, 33), (1000, 512, 130),
                                        (4095, 513, 64), (4096, 70000, 8), (4097, 262143, 4), (10007, 262144, 3),
                                        (9000, 100, 520), (30000, 1000, 40), (2049, 600, 20), (8192, 262144, 3),
                                        (8191, 5, 64), (8193, 70000, 12), (9, 4, 96), (16, 40, 96), (17, 3, 96)])
def test_gradient_is_exact_for_whole_numbers(R, kind, n, rows, dim):
    rng = np.random.default_rng(n + rows)
    dout, ids = whole(rng, n, dim), some_ids(kind, n, rows, n)
    want, _, _ = mx8.embed_grad(dout, ids, rows, 0.5)
    tids = torch.from_numpy(ids.astype(np.int64)).cuda()
    got = R.rslm_embed_backward(torch.from_numpy(dout).cuda(), tids, rows, scale=0.5)
    assert np.array_equal(got.double().cpu().numpy(), want)
    # bfloat16 terms (whole numbers up to 8 are exact) to float32, from 32-bit ids, added to what is there
    base = torch.ones((rows, dim + 3), device="cuda")
    got = R.rslm_embed_backward(torch.from_numpy(dout).cuda().bfloat16(), tids.int(), rows, scale=0.5, dtype=torch.float32,
                                out=base[:, :dim], accumulate=True)
    assert np.array_equal(got.double().cpu().numpy(), want + 1) and (base[:, dim:] == 1).all()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,rows,dim,extra", [(300, 40, 768, 0), (5000, 3000, 129, 7), (20000, 50, 513, 1), (257, 1000, 2049, 0)])
def test_gradient(R, dt, n, rows, dim, extra):
    g = torch.Generator().manual_seed(n)
    dout = torch.randn((n, dim + extra), generator=g).to(DT[dt])[:, :dim]
    ids = some_ids("zipf", n, rows, n)
    want, terms, count = mx8.embed_grad(dout.double().numpy(), ids, rows, 1.3)
    tol = (count[:, None] + 2) * 2.0 ** -24 * terms
    tol = tol + HALF[dt] * (np.abs(want) + tol) + (2.0 ** -25 if dt == "f16" else 0.0)
    wide = dout.new_empty((n, dim + extra)).cuda()
    wide[:, :dim] = dout.cuda()
    tids = torch.from_numpy(ids).cuda()
    got = R.rslm_embed_backward(wide[:, :dim], tids, rows, scale=1.3)
    assert got.dtype == DT[dt] and (np.abs(got.double().cpu().numpy() - want) <= tol).all()
    assert torch.equal(R.rslm_embed_backward(wide[:, :dim], tids, rows, scale=1.3), got)
    # differences: the sum of out * dout is linear in the table
    out = torch.full((rows, dim + 1), 2.0, dtype=DT[dt], device="cuda")
    R.rslm_embed_backward(wide[:, :dim], tids, rows, scale=1.3, out=out[:, :dim])
    assert torch.equal(out[:, :dim], got) and (out[:, dim:] == 2).all()


def test_gradient_of_very_many_tokens(R):
    """More than 256 workgroups' rounds of the sort."""
    n, rows, dim = 1_100_003, 5000, 4
    rng = np.random.default_rng(1)
    ids = rng.integers(-1, rows, n)
    dout = rng.integers(-2, 3, (n, dim)).astype(np.float32)
    want, _, _ = mx8.embed_grad(dout, ids, rows, 1.0)
    got = R.rslm_embed_backward(torch.from_numpy(dout).cuda(), torch.from_numpy(ids).cuda(), rows)
    assert np.array_equal(got.double().cpu().numpy(), want)


def test_gradient_past_32_bits_of_bytes(R):
    """A table and rows of dout beyond 4 GiB from its start."""
    rows, dim, n = 300_000, 8192, 40
    ids = np.array([0, rows - 1, 270_000, 5, rows - 1] * 8)
    dout = whole(np.random.default_rng(3), n, dim)
    out = R.rslm_embed_backward(torch.from_numpy(dout).cuda().bfloat16(), torch.from_numpy(ids).cuda(), rows)
    for v in (0, 5, 270_000, rows - 1):
        assert np.array_equal(out[v].double().cpu().numpy(), dout[ids == v].sum(0).astype(np.float64))
    used = torch.zeros((rows,), dtype=torch.bool, device="cuda")
    used[torch.from_numpy(ids).cuda()] = True
    assert not out[~used].any()
    back = R.rslm_embed(out, torch.tensor([rows - 1, 270_000], device="cuda"))
    assert torch.equal(back[0], out[rows - 1]) and torch.equal(back[1], out[270_000])


def test_gradient_of_nothing(R):
    ids = torch.empty((0,), dtype=torch.int64, device="cuda")
    dout = torch.empty((0, 12), device="cuda")
    assert (R.rslm_embed_backward(dout, ids, 7) == 0).all()
    out = torch.ones((7, 12), device="cuda")
    assert (R.rslm_embed_backward(dout, ids, 7, out=out, accumulate=True) == 1).all()
    assert R.rslm_embed_backward(dout, ids, 0).shape == (0, 12)
    assert R.rslm_embed_backward(torch.ones((3, 12), device="cuda"), torch.zeros((3,), dtype=torch.int64, device="cuda"), 0).shape == (0, 12)


def test_gradient_of_rows_that_are_one(R):
    """dout of one row for all tokens, as the gradient of a sum over them is."""
    ids = torch.tensor([3, 1, 3, 3, -1, 0] * 500, device="cuda")
    one = torch.arange(40, device="cuda", dtype=torch.float32)
    got = R.rslm_embed_backward(one.expand(3000, 40), ids, 5)
    assert torch.equal(got, torch.stack([500 * one, 500 * one, 0 * one, 1500 * one, 0 * one]))


def test_other_stream(R):
    table, ids = torch.randn((300, 96), device="cuda"), torch.randint(-1, 300, (5000,), device="cuda")
    want = R.rslm_embed(table, ids)
    grad = R.rslm_embed_backward(want, ids, 300)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = R.rslm_embed(table, ids, stream=s)
    back = R.rslm_embed_backward(got, ids, 300, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want) and torch.equal(back, grad)


def test_two_captured_graphs_with_eager_calls_between(R):
    """Each captured call's workspace is its own: replays of both, with eager calls of other
    sizes between them, give what eager calls give."""
    graphs = []
    for n, rows, dim in ((6000, 700, 96), (300, 5000, 40)):
        dout, ids = torch.empty((n, dim), device="cuda"), torch.empty((n,), dtype=torch.int64, device="cuda")
        dout.normal_(), ids.random_(0, rows)
        R.rslm_embed_backward(dout, ids, rows)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = R.rslm_embed_backward(dout, ids, rows)
        graphs.append((graph, dout, ids, out, rows))
    for turn in range(3):
        for graph, dout, ids, out, rows in graphs:
            dout.normal_(), ids.random_(-1, rows)
        for graph, *_ in graphs:
            graph.replay()
        for graph, dout, ids, out, rows in graphs:
            R.rslm_embed_backward(torch.ones((20000, 64), device="cuda"), torch.zeros((20000,), dtype=torch.int64, device="cuda"), 9)
            assert torch.equal(out, R.rslm_embed_backward(dout, ids, rows))
