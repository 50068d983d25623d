"""Every arrangement of the products of 4-bit rows on the GPU: each height of tiles,
sums in one part and in several, odd and even numbers of groups of 128, and sizes that end
inside a tile.  Which arrangement a size takes is checked in test_mx4_choice.py.

Exact tests: a float row has a single value, with every bit of its significand in use,
and the 4-bit rows hold powers of two, so each result is one product, which the
type holds: any part of the value that is lost, or any place that is read wrong, shows.
Tests of whole sums: the bound of test_gpu_mx4.py, 2 (3 L + 16) 2^-24 sum |terms|, and half
a unit of a 16-bit result.
"""

import numpy as np
import pytest

from oracle import mx4

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BITS = {"f32": 24, "f16": 11, "bf16": 8}
HALF_ULP = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}

# m, n, dim
SCORE = [(1, 515, 768), (7, 300, 130), (16, 100, 200), (3, 1000, 33),               # few rows
         (16, 515, 2049), (32, 1030, 641), (17, 20011, 130), (64, 515, 1030), (40, 20011, 130),
         (100, 700, 513), (128, 20011, 384), (129, 257, 33), (200, 515, 2049),
         (385, 2049, 1030), (257, 4099, 641), (257, 8193, 300), (513, 8193, 130), (385, 16385, 513),
         (139, 13001, 1030), (2947, 105, 4096), (130, 34400, 130)]
BACKWARD = [(1, 70, 33), (4, 10007, 96), (16, 515, 300), (20, 5001, 100), (32, 129, 257), (50, 20011, 130), (64, 77, 4096),
            (100, 3001, 300), (129, 129, 700), (128, 256, 8192),
            (257, 5000, 513), (513, 10007, 1025), (2049, 100, 4096), (2049, 600, 4096), (2049, 1000, 4096),
            (154, 34507, 300), (133, 50001, 130)]
# the forms of 4-bit by 4-bit, of which 256 and 128 run ahead of their use from 5 groups on
MATMUL = [(4097, 4100, 513, "f32"), (4100, 4090, 640, "bf16"), (4090, 4100, 768, "f16"), (4101, 4097, 1000, "f32"),
          (4096, 4103, 1100, "bf16"), (4097, 4097, 1281, "bf16"), (1030, 2051, 1100, "f32"), (700, 4100, 1300, "f16"),
          (513, 4097, 2049, "bf16"), (40, 70000, 641, "f32"), (33, 30011, 300, "bf16"), (20, 3001, 1100, "f32")]


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def powers(R, n, dim, seed):
    """4-bit rows of powers of two (0.5 to 32) of either sign, and their values on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    steps = -(-dim // 128)
    pick = torch.tensor([1, 2, 4, 6, 9, 10, 12, 14], device="cuda", dtype=torch.uint8)   # 0.5, 1, 2, 4
    c = pick[torch.randint(0, 8, (n, 128 * steps), generator=g, device="cuda")]
    c[:, dim:] = 0
    s = torch.randint(126, 130, (n, 4 * steps), generator=g, device="cuda").to(torch.uint8)
    s[:, -(-dim // 32):] = 0
    rows = R.Mx4Rows(c[:, 0::2] | (c[:, 1::2] << 4), s, dim)
    return rows, R.rslm_mx4_dequantize(rows)


def places(m, length, turn):
    """A place for each of m rows: the ends of the sum and of its groups of 32 and 128, then any."""
    ends = [0, length - 1] + [p for b in (32, 128, 256, 512, 1024) for q in range(b, length, b) for p in (q - 1, q)]
    rng = np.random.default_rng(turn)
    ends = [ends[i] for i in rng.permutation(len(ends))] if turn else ends
    p = np.concatenate([ends[:m - m // 3], rng.integers(0, length, m)])[:m]
    return torch.from_numpy(p.astype(np.int64)).cuda()


def significands(m, dt, seed):
    """Odd whole numbers of as many bits as the type's significand, with either sign and some range."""
    rng = np.random.default_rng(seed)
    b = BITS[dt]
    v = (rng.integers(2 ** (b - 2), 2 ** (b - 1), m) * 2 + 1) * rng.choice([-1.0, 1.0], m) * 2.0 ** (rng.integers(-3, 3, m) - b)
    return torch.from_numpy(v).cuda().to(DT[dt])


def exact_case(R, call, m, n, dim, dt, backward):
    b, vb = powers(R, n, dim, m + n)
    length = n if backward else dim
    for turn in range(max(1, 24 // m)):
        at, v = places(m, length, turn), significands(m, dt, turn)
        assert torch.equal(v.double().to(DT[dt]), v) and (v != 0).all()
        x = torch.zeros(m, length, dtype=DT[dt], device="cuda")
        x[torch.arange(m, device="cuda"), at] = v
        want = v.float()[:, None] * (vb[at] if backward else vb[:, at].t())
        for out in {"f32", dt}:
            got = call(x, b, dtype=DT[out])
            assert torch.equal(got.float(), want), (turn, out, (got.float() != want).nonzero()[:5])
        if dim > 1 and turn == 0:      # rows that begin anywhere
            wide = torch.zeros(m, length + 3, dtype=DT[dt], device="cuda")
            wide[:, 1:length + 1] = x
            assert torch.equal(call(wide[:, 1:length + 1], b, dtype=torch.float32), want)


@pytest.mark.parametrize("m,n,dim", SCORE)
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_score_is_exact_for_one_product(R, m, n, dim, dt):
    exact_case(R, R.rslm_mx4_score, m, n, dim, dt, False)


@pytest.mark.parametrize("m,n,dim", BACKWARD)
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_gradient_is_exact_for_one_product(R, m, n, dim, dt):
    exact_case(R, R.rslm_mx4_score_backward, m, n, dim, dt, True)


def random_rows(R, n, dim, seed):
    rng = np.random.default_rng(seed)
    pc, ps = mx4.pack(rng.integers(0, 16, (n, dim)).astype(np.uint8),
                      rng.integers(124, 130, (n, -(-dim // 32))).astype(np.uint8), dim)
    return R.Mx4Rows(torch.from_numpy(pc).cuda(), torch.from_numpy(ps).cuda(), dim), mx4.values(pc, ps, dim)


def check_sums(got, want, terms, length, dt):
    g = got.double().cpu().numpy()
    tol = 2 * (3 * length + 16) * 2.0 ** -24 * terms
    tol = tol + HALF_ULP[dt] * (np.abs(want) + tol) + (2.0 ** -24 if dt == "f16" else 0.0)
    bad = ~(np.abs(g - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:5], g[bad][:5], want[bad][:5], tol[bad][:5])


@pytest.mark.parametrize("m,n,dim", [s for s in SCORE if s[0] > 200])
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_score_sums(R, m, n, dim, dt):
    b, vb = random_rows(R, n, dim, 1)
    x = torch.randn(m, dim, device="cuda").to(DT[dt])
    vx = x.double().cpu().numpy()
    check_sums(R.rslm_mx4_score(x, b), vx @ vb.T, np.abs(vx) @ np.abs(vb).T, dim, "f32")


@pytest.mark.parametrize("m,n,dim", [s for s in BACKWARD if s[0] > 200])
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_gradient_sums(R, m, n, dim, dt):
    b, vb = random_rows(R, n, dim, 2)
    d = (torch.randn(m, n, device="cuda") / 256).to(DT[dt])
    vd = d.double().cpu().numpy()
    got = R.rslm_mx4_score_backward(d, b, dtype=torch.float32)
    check_sums(got, vd @ vb, np.abs(vd) @ np.abs(vb), n, "f32")
    assert torch.equal(got, R.rslm_mx4_score_backward(d, b, dtype=torch.float32))


@pytest.mark.parametrize("m,n,dim,dt", MATMUL)
def test_matmul_of_many_groups(R, m, n, dim, dt):
    """Sums long enough that the loop which loads ahead runs; NaN scales in the first, a middle
    and the last group of a row; stores inside wider rows."""
    a, va = random_rows(R, m, dim, 3)
    b, vb = random_rows(R, n, dim, 4)
    if dt == "f16":
        a = R.Mx4Rows(a.codes, torch.where(a.scales > 0, a.scales - 8, a.scales), dim)
        va = va / 256
    buf = torch.full((m + 2, n + 9), 3.0, device="cuda", dtype=DT[dt])
    out = R.rslm_mx4_matmul(a, b, dtype=DT[dt], out=buf[1:m + 1, 4:4 + n])
    check_sums(out, va @ vb.T, np.abs(va) @ np.abs(vb).T, dim, dt)
    plain = R.rslm_mx4_matmul(a, b, dtype=DT[dt])
    assert torch.equal(plain, out)
    out.fill_(3.0)
    assert (buf == 3).all()
    last = (dim - 1) // 32
    bad_a, bad_b = {0: 0, m // 2: last // 2, m - 1: last}, {1: last, n // 2: last // 2 + 1, n - 1: 0}
    for r, s in bad_a.items():
        a.scales[r, s] = 255
    for r, s in bad_b.items():
        b.scales[r, s] = 255
    got = R.rslm_mx4_matmul(a, b, dtype=DT[dt])
    nan = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    nan[list(bad_a)] = True
    nan[:, list(bad_b)] = True
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], plain[~nan])


@pytest.mark.parametrize("dim", range(1, 16))
def test_rotation_of_few_coordinates(R, dim):
    """Below 16 coordinates a vector is in one or two lanes: the bits of rslm_fwht."""
    rng = np.random.default_rng(dim)
    for passes in (1, 2):
        plan = R.Plan(dim, 4, passes=passes)
        for n in (1, 3, 70, 5000):
            x = torch.from_numpy(rng.standard_normal((n, dim)).astype(np.float32)).cuda()
            c, s = mx4.quantize(R.rslm_fwht(plan, x).double().cpu().numpy())
            pc, ps = mx4.pack(c, s, dim)
            rows = R.rslm_mx4_quantize(x, plan)
            assert np.array_equal(rows.codes.cpu().numpy(), pc) and np.array_equal(rows.scales.cpu().numpy(), ps)
            half = x.half()
            c, s = mx4.quantize(R.rslm_fwht(plan, half.float()).double().cpu().numpy())
            pc, ps = mx4.pack(c, s, dim)
            rows = R.rslm_mx4_quantize(half, plan)
            assert np.array_equal(rows.codes.cpu().numpy(), pc) and np.array_equal(rows.scales.cpu().numpy(), ps)
