"""8-bit (MX8) rows on the GPU against float64: codes and values bit for bit, products
with 4-bit rows.

Tolerances.  A float32 product sums dim exact terms in float32 and an unknown order:
|error| <= 2 (3 L + 16) 2^-24 sum |terms| for L terms (as for the 4-bit products).  A
16-bit one also loses, of each product in a group of eight, less than 2^-13 of the
group's largest: at most 7 2^-13 of each group's largest, which is at most the group's
sum of magnitudes; and is rounded once more, by 2^-11 (float16) or 2^-8 (bfloat16) of
the value and float16's least subnormal.
"""

import numpy as np
import pytest

from oracle import mx4, mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def check_rows(rows, x64):
    """Codes and scales of MX8 rows against those of float64 values, and the padding."""
    c, s = mx8.quantize(x64)
    pc, ps = mx8.pack(c, s, x64.shape[1])
    got_c, got_s = rows.codes.cpu().numpy(), rows.scales.cpu().numpy()
    assert np.array_equal(got_s, ps)
    bad = np.repeat(ps == 255, 32, axis=1)      # codes under a NaN scale mean nothing
    # a value that rounds to zero keeps its sign
    same = (got_c == pc) | (((got_c | pc) & 127) == 0)
    assert same[~bad].all()
    assert (got_c[:, x64.shape[1]:] == 0).all()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,dim,extra,off", [
    (1, 1, 0, 0), (3, 31, 1, 0), (2, 32, 0, 1), (5, 33, 7, 3), (17, 96, 0, 0), (16, 127, 2, 1), (4, 128, 0, 0),
    (33, 129, 0, 0), (1, 768, 0, 0), (300, 768, 8, 1), (9, 2049, 15, 0), (2, 4100, 0, 5), (1, 65536, 0, 0)])
def test_quantize(R, dt, n, dim, extra, off):
    g = torch.Generator().manual_seed(n * dim + extra)
    wide = torch.randn((n * (dim + extra) + off,), generator=g) * torch.exp(2 * torch.randn((1,), generator=g))
    wide = wide.to(DT[dt])
    x = wide[off:].view(n, dim + extra)[:, :dim]
    rows = R.rslm_mx8_quantize(wide.cuda()[off:].view(n, dim + extra)[:, :dim])
    check_rows(rows, x.double().numpy())
    want = mx8.values(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), dim)
    assert np.array_equal(R.rslm_mx8_dequantize(rows).double().cpu().numpy(), want)


def test_quantize_at_the_ends_of_the_range(R):
    """Zeros of both signs, ties, all levels, a largest value at and past 448 steps, float32's
    least and largest, subnormals, infinities and NaN."""
    level = np.concatenate([mx8.E4M3, (mx8.E4M3[1:] + mx8.E4M3[:-1]) / 2])
    blocks = [np.resize(v, 32) for v in np.array_split(np.concatenate([level, -level]), 16)]
    blocks += [np.resize([0.0, -0.0], 32), np.resize([448.0, 1.0], 32), np.resize([448.00003, 447.9, -3.1], 32),
               np.resize([2.0 ** -149, -2.0 ** -148], 32), np.resize([2.0 ** -126, 2.0 ** -130, 2.0 ** -127], 32),
               np.resize([2.0 ** -118 * 1.76, 2.0 ** -127], 32), np.resize([3.4e38, -1e38, 1.0], 32)]
    blocks += [np.resize([np.inf, 1.0], 32), np.resize([2.0, np.nan], 32)]
    blocks += [b * 2.0 ** -20 for b in blocks[:16]]
    x = np.stack(blocks).astype(np.float32).reshape(1, -1)
    rows = R.rslm_mx8_quantize(dev(x))
    check_rows(rows, x.astype(np.float64))
    want = mx8.values(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), x.shape[1])
    got = R.rslm_mx8_dequantize(rows).cpu().numpy()
    # 3.4e38 is nearest to 256 2^120 = 2^128, past float32's end: infinity in float32
    with np.errstate(over="ignore"):
        assert np.array_equal(got, want.astype(np.float32), equal_nan=True)
    assert np.isnan(got).sum() == 64


@pytest.mark.parametrize("dim", [1, 5, 64, 100, 127, 128, 129, 256, 384, 768, 1000, 2049, 4096])
@pytest.mark.parametrize("passes", [1, 2])
def test_quantize_rotated_is_that_of_the_rotation(R, dim, passes):
    g = torch.Generator(device="cuda").manual_seed(dim)
    x = torch.randn((37, dim), generator=g, device="cuda")
    plan = R.Plan(dim, 4, passes=passes)
    rows = R.rslm_mx8_quantize(x, plan)
    plain = R.rslm_mx8_quantize(R.rslm_fwht(plan, x))
    assert torch.equal(rows.scales, plain.scales) and torch.equal(rows.codes, plain.codes)


def test_quantize_edges(R):
    rows = R.rslm_mx8_quantize(torch.empty((0, 40), device="cuda"))
    assert rows.n == 0 and R.rslm_mx8_dequantize(rows).shape == (0, 40)
    x = torch.randn((1, 70), device="cuda")
    check_rows(R.rslm_mx8_quantize(x.expand(5, 70)), x.expand(5, 70).double().cpu().numpy())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = R.rslm_mx8_quantize(x, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other.codes, R.rslm_mx8_quantize(x).codes)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_dequantize_every_code_and_scale(R, dt):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 8, 1)
    want = mx8.values(codes, scales, 256)
    rows = R.Mx8Rows(dev(codes), dev(scales), 256)
    wide = torch.full((256, 259), 7.0, dtype=DT[dt], device="cuda")
    got = R.rslm_mx8_dequantize(rows, dtype=DT[dt], out=wide[:, :256])
    assert (wide[:, 256:] == 7).all()
    assert torch.equal(got.cpu().isnan(), torch.from_numpy(want).to(DT[dt]).isnan())
    ok = ~np.isnan(want)
    # float32 first: that is where the values are exact
    assert np.array_equal(got.cpu().double().numpy()[ok], torch.from_numpy(want).float().to(DT[dt]).double().numpy()[ok])


def sides(m, n, dim, seed, spread=3):
    rng = np.random.default_rng(seed)
    ac, asc = rng.integers(0, 256, (m, dim)).astype(np.uint8), rng.integers(127 - spread, 128 + spread, (m, -(-dim // 32)))
    ac[(ac & 127) == 127] ^= 1
    bc, bsc = rng.integers(0, 16, (n, dim)).astype(np.uint8), rng.integers(127 - spread, 128 + spread, (n, -(-dim // 32)))
    return mx8.pack(ac, asc.astype(np.uint8), dim), mx4.pack(bc, bsc.astype(np.uint8), dim)


def product(a, b, dim):
    """The product in float64, the sum of the terms' magnitudes, and of the largest of each eight
    (of large products that sum again, which is more)."""
    x, y = mx8.values(*a, dim), mx4.values(*b, dim)
    pad = -dim % 8
    xs, ys = np.pad(np.abs(x), ((0, 0), (0, pad))), np.pad(np.abs(y), ((0, 0), (0, pad)))
    if x.shape[0] * y.shape[0] * dim > 1 << 28:
        terms = np.abs(x) @ np.abs(y).T
        return x @ y.T, terms, terms
    top = np.zeros((x.shape[0], y.shape[0]))
    for o in range(0, dim, 8):
        top += (xs[:, None, o:o + 8] * ys[None, :, o:o + 8]).max(-1)
    return x @ y.T, np.abs(x) @ np.abs(y).T, top


def check_product(got, want, terms, top, dim, dt):
    tol = 2 * (3 * dim + 16) * 2.0 ** -24 * terms
    if dt != "f32":
        tol = tol + 7 * 2.0 ** -13 * top
        tol = tol + HALF_ULP[dt] * (np.abs(want) + tol) + (2.0 ** -24 if dt == "f16" else 0.0)
    g = got.double().cpu().numpy()
    over = np.abs(want) > 65000 if dt == "f16" else np.zeros_like(want, dtype=bool)
    assert g.shape == want.shape and (np.abs(g - want) <= tol)[~over].all(), (np.abs(g - want) / tol)[~over].max()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,dim", [
    (1, 1, 1), (1, 3, 31), (2, 17, 32), (3, 16, 33), (1, 300, 96), (15, 64, 100), (16, 255, 128), (17, 257, 129),
    (5, 1000, 768), (32, 65, 200), (33, 70, 300), (64, 129, 256), (65, 300, 129), (100, 513, 260), (128, 256, 384),
    (130, 1030, 500), (257, 700, 96), (300, 2049, 640), (1, 5000, 2049), (9, 33, 4096), (16, 100, 4096),
    (16, 70000, 200), (15, 50, 4200), (70, 300, 2000), (260, 70001, 1500), (250, 66001, 1541), (1000, 17000, 1536),
    (17, 60000, 31), (33, 40001, 129), (65, 30003, 300), (129, 9001, 96), (257, 4001, 260), (40, 19000, 2049)])
def test_score(R, dt, m, n, dim):
    a, b = sides(m, n, dim, m + 7 * n + dim, spread=1 if dt == "f16" else 3)
    if dt == "f16":
        a[1][a[1] > 0] -= 8     # within float16
    wide = torch.full((m, n + 3), 5.0, dtype=DT[dt], device="cuda")
    got = R.rslm_mx8_score(R.Mx8Rows(*map(dev, a), dim), R.Mx4Rows(*map(dev, b), dim), dtype=DT[dt], out=wide[:, :n])
    check_product(got, *product(a, b, dim), dim, dt)
    assert (wide[:, n:] == 5).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,dim", [(1, 40, 64), (16, 40, 300), (40, 300, 300), (256, 4096, 128), (256, 8192, 768), (64, 16000, 100)])
def test_score_at_the_ends_of_the_scales(R, dt, m, n, dim):
    """Scales of 0 and 254 on either side with the other's making up for it, and NaN scales
    and codes, whose rows and columns are NaN and no others."""
    a, b = sides(m, n, dim, 3, spread=1)
    nb = -(-dim // 32)
    a[1][0, :nb], b[1][:, :nb] = 200, 100
    a[1][m // 2, :nb] = 3
    b[1][n - 1, :nb] = 250
    b[1][3, 1] = 255
    a[0][m - 1, dim - 1] = 0xff
    if m > 2:
        a[1][1, nb - 1] = 255
    want, terms, top = product(a, b, dim)
    got = R.rslm_mx8_score(R.Mx8Rows(*map(dev, a), dim), R.Mx4Rows(*map(dev, b), dim), dtype=DT[dt])
    # the last row of b, of 2^(250 - 127) and more, has terms past float32's 2^128 with all but
    # the smallest row of a: infinities of either sign, or NaN where both meet
    held = np.isnan(terms) | (terms < 2.0 ** 127)
    assert held[:, :n - 1].all() and held[m // 2].all()
    assert np.array_equal(got.isnan().cpu().numpy()[held], np.isnan(want)[held])
    ok = ~np.isnan(want) & held
    g = got.double().cpu().numpy()
    small = 2.0 ** -125 * dim      # bfloat16 and float32 end at 2^-126; values of a below 2^-130 are rounded
    tol = 2 * (3 * dim + 16) * 2.0 ** -24 * terms + small
    if dt == "bf16":
        tol = tol + 7 * 2.0 ** -13 * top
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    assert (np.abs(g - want) <= tol)[ok].all()


def test_score_of_nothing(R):
    for m, n in ((0, 5), (5, 0), (0, 0)):
        a, b = R.Mx8Rows.empty(m, 40, "cuda"), R.Mx4Rows.empty(n, 40, "cuda")
        assert R.rslm_mx8_score(a, b).shape == (m, n)


def test_score_is_that_of_quantised_rows(R):
    """Through the calls: rotated queries in 8 bits against a rotated collection in 4."""
    g = torch.Generator(device="cuda").manual_seed(5)
    plan = R.Plan(768, 4)
    x, c = torch.randn((20, 768), generator=g, device="cuda"), torch.randn((900, 768), generator=g, device="cuda")
    a, b = R.rslm_mx8_quantize(x, plan), R.rslm_mx4_quantize(c, plan)
    exact = R.rslm_mx8_dequantize(a).double() @ R.rslm_mx4_dequantize(b).double().t().contiguous()
    got = R.rslm_mx8_score(a, b)
    terms = R.rslm_mx8_dequantize(a).double().abs() @ R.rslm_mx4_dequantize(b).double().abs().t().contiguous()
    assert ((got.double() - exact).abs() <= 2 * (3 * 768 + 16) * 2.0 ** -24 * terms).all()
    # and near the product of the vectors: each code is off by 2^-4 of its value at most, MX4's
    # by 2^-2, and the rotation keeps products, so that all terms are off by 0.33 of theirs
    true = R.rslm_fwht(plan, x).double() @ R.rslm_fwht(plan, c).double().t().contiguous()
    assert (got.double() - true).abs().mean() < 0.33 * terms.mean()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1, 40, 300])
def test_score_captured(R, dt, m):
    a, b = sides(m, 4100, 256, m)
    ra, rb = R.Mx8Rows(*map(dev, a), 256), R.Mx4Rows(*map(dev, b), 256)
    out = torch.empty((m, 4100), dtype=DT[dt], device="cuda")
    R.rslm_mx8_score(ra, rb, dtype=DT[dt], out=out)
    want = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.rslm_mx8_score(ra, rb, dtype=DT[dt], out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want)
        R.rslm_mx8_score(ra, rb, dtype=DT[dt])
        torch.cuda.synchronize()
