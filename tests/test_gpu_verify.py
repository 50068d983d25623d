"""Verification of drafted tokens on the GPU against float64: the tokens and how many
stand are equal (the kernels' weights are within 2^-42, so that a uniform number between
both's borders has a chance below 1e-7 a token here), log probabilities within half a unit of
float32 and 1e-12 of the largest score's distance.
"""

import numpy as np
import pytest

from oracle import mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def make(b, k, n, dt, seed, masked=0.0, draft=True, amp=3.0):
    g = torch.Generator().manual_seed(seed)
    z = amp * torch.randn((b, k + 1, n), generator=g)
    z[torch.rand((b, 1, n), generator=g).expand(b, k + 1, n) < masked] = -float("inf")
    d = z[:, :k] + 0.7 * torch.randn((b, k, n), generator=g)
    z, d = z.to(DT[dt]), d.to(DT[dt])
    noise = -torch.log(-torch.log(torch.rand((b, k, n), generator=g).clamp(1e-6, 1 - 1e-6)))
    tokens = (d.float() + noise).argmax(-1) if k else torch.zeros((b, 0), dtype=torch.int64)
    return z, d if draft else None, tokens, torch.rand((b, k + 1), generator=g)


def check(R, z, d, tokens, uniforms, counts=None, scale=1.0, draft_scale=None, calls=None):
    """The call on these (CPU) tensors, or on `calls` (GPU), against the oracle."""
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    gz, gd = calls if calls else (up(z), up(d))
    r = R.rslm_verify(gz, up(tokens), up(uniforms), draft=gd, counts=up(counts), scale=scale, draft_scale=draft_scale)
    # the calls take scales as float32
    scale = float(np.float32(scale))
    draft_scale = None if draft_scale is None else float(np.float32(draft_scale))
    want = mx8.verify(z.double().numpy(), tokens.numpy(), uniforms.numpy(), None if d is None else d.double().numpy(),
                      None if counts is None else counts.numpy(), scale, draft_scale)
    assert np.array_equal(r.accepted.cpu().numpy(), want[1])
    assert np.array_equal(r.tokens.cpu().numpy(), want[0])
    finite = z.double().numpy()
    finite = np.where(np.isfinite(finite), finite, 0.0)
    far = scale * (finite.max() - finite.min()) + 40
    assert (np.abs(r.logprob.double().cpu().numpy() - want[2]) <= 2.0 ** -24 * np.abs(want[2]) + 1e-12 * far).all()
    return r


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("b,k,n,masked", [(1, 1, 1, 0), (2, 3, 2, 0), (5, 0, 3, 0), (3, 4, 7, 0.3), (1, 4, 1000, 0), (40, 2, 129, 0.9),
                                          (7, 5, 4095, 0), (3, 1, 4096, 0.05), (2, 8, 4097, 0), (30, 4, 9001, 0), (1, 0, 50001, 0.5),
                                          (1, 2, 300001, 0), (64, 1, 20000, 0), (300, 3, 333, 0), (2, 64, 500, 0)])
def test_against_float64(R, dt, draft, b, k, n, masked):
    z, d, tokens, u = make(b, k, n, dt, b + n, masked, draft)
    check(R, z, d, tokens, u, scale=1.25)
    counts = torch.from_numpy(np.random.default_rng(b).integers(-1, k + 2, b).astype(np.int32))
    check(R, z, d, tokens, u, counts, scale=0.6, draft_scale=0.9)


def test_long_rows(R):
    z, d, tokens, u = make(1, 1, 1_000_003, "bf16", 5)
    for seed in range(4):
        check(R, z, d, tokens, torch.rand((1, 2), generator=torch.Generator().manual_seed(seed)))


@pytest.mark.parametrize("n", [5, 300, 5000])
def test_first_last_and_invalid_uniforms(R, n):
    z, d, tokens, _ = make(9, 1, n, "f32", n, masked=0.2)
    z[:, :, 0] = z[:, :, -1] = -float("inf")
    u = torch.tensor([0.0, 2.0 ** -30, 0.5, 1 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan"), float("inf")])
    for first in (0.0, 0.999999):
        r = check(R, z, None, tokens, torch.stack([torch.full((9,), first), u], 1))
        assert (r.tokens.cpu()[:, 0] != 0).all() and (r.tokens.cpu()[:, 0] != n - 1).all()


def test_sharp_and_flat_and_far_scores(R):
    """One score far above all, equal scores, scores that float32 itself cannot take the
    difference of, scales at both ends."""
    b, n = 8, 300
    z = torch.randn((b, 2, n), generator=torch.Generator().manual_seed(1))
    z[0, :, 17] = 1e4
    z[1] = 0.25
    z[2] *= 1e-30
    z[3] = torch.where(torch.arange(n) % 2 == 0, 3e38, -3e38)
    z[4] = torch.where(torch.arange(n) % 3 == 0, 3e38, 2.99e38)
    z[5, :, 4:] = -float("inf")
    z[6] -= 1e6
    tokens = torch.full((b, 1), 3)
    u = torch.rand((b, 2), generator=torch.Generator().manual_seed(2))
    d = z[:, :1].clone()
    for scale in (1.0, 1e-30, 1e30, 2.0 ** 127):
        check(R, z, d, tokens, u, scale=scale)
        check(R, z, None, tokens, u, scale=scale)


def test_the_same_scores_let_drafts_stand(R):
    """p = q: every draft stands for u < 1, whatever it is; and if u is not below 1, p is
    drawn from, as nothing is left of p - q."""
    z, _, _, u = make(6, 3, 700, "bf16", 2)
    tokens = torch.randint(0, 700, (6, 3), generator=torch.Generator().manual_seed(0))
    r = check(R, z, z[:, :3], tokens, u)
    assert (r.accepted == 3).all()
    u[:, 1] = 1.0
    r = check(R, z, z[:, :3], tokens, u)
    assert (r.accepted == 1).all() and (r.tokens[:, 1] >= 0).all() and (r.tokens[:, 2:] == -1).all()


def test_rows_without_probabilities(R):
    inf, nan = float("inf"), float("nan")
    z, d, tokens, u = make(9, 2, 5000, "f32", 7)
    u[:, :2] = 0.0
    z[0, 0] = -inf
    z[1, 1, 4999] = nan
    z[2, 2, 0] = inf
    z[3] = -inf
    d[4, 0] = -inf
    d[5, 1, 77] = nan
    d[6, 0, 4096] = inf
    tokens[7, 1] = -1
    tokens[8, 0] = 5000
    r = check(R, z, d, tokens, u)
    got = r.tokens.cpu()
    assert got[0, 0] == -1 and got[1, 1] == -1 and got[2, 2] == -1 and got[3, 0] == -1
    assert (got[4:, 0] >= 0).all() and list(r.accepted.cpu()) == [0, 1, 2, 0, 0, 1, 0, 1, 0]


def test_drafts_with_no_probability(R):
    z, d, tokens, u = make(4, 1, 50, "f32", 3)
    for i in range(4):
        z[i, :, tokens[i, 0]] = -inf if (inf := float("inf")) else 0
    u[:, 0] = 0.0
    r = check(R, z, d, tokens, u)
    assert (r.accepted == 0).all() and (r.tokens[:, 0].cpu() != tokens[:, 0]).all()


@pytest.mark.parametrize("draft", [True, False])
def test_first_token_has_the_targets_distribution(R, draft):
    """16,384 sequences with one draft each: the first token's counts within 5 standard
    deviations of the target's probabilities (32 counts; a chance of 2e-5 for a wrong alarm,
    and the seed is fixed)."""
    b, n = 16384, 16
    g = torch.Generator().manual_seed(11)
    z, dz = torch.randn((n,), generator=g), torch.randn((n,), generator=g)
    p, q = torch.softmax(z.double(), 0), torch.softmax(dz.double(), 0)
    tokens = torch.multinomial(q, b, replacement=True, generator=g)[:, None] if draft else torch.full((b, 1), int(z.argmax()))
    u = torch.rand((b, 2), generator=g)
    r = R.rslm_verify(z.cuda().expand(b, 2, n), tokens.cuda(), u.cuda(), draft=dz.cuda().expand(b, 1, n) if draft else None)
    for place, on in ((0, torch.ones(b, dtype=torch.bool)), (1, r.accepted.cpu() == 1)):
        count = int(on.sum())
        got = torch.bincount(r.tokens.cpu()[on, place], minlength=n).double()
        assert ((got - count * p).abs() <= 5 * torch.sqrt(count * p * (1 - p)) + 1).all()


def test_strides(R):
    z, d, tokens, u = make(5, 2, 1001, "bf16", 9)
    wide = torch.zeros((3, 5, 1010), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 3:1004] = z.permute(1, 0, 2).cuda()
    drafts = torch.zeros((5, 4, 1001), dtype=torch.bfloat16, device="cuda")
    drafts[:, ::2] = d.cuda()
    check(R, z, d, tokens, u, calls=(wide.permute(1, 0, 2)[:, :, 3:1004], drafts[:, ::2]))
    # rows past a count are not read: NaN there does nothing
    counts = torch.tensor([0, 1, 2, 0, 1], dtype=torch.int32)
    zn, dn = z.clone(), d.clone()
    for i, c in enumerate(counts):
        zn[i, c + 1:] = float("nan")
        dn[i, c:] = float("nan")
    check(R, zn, dn, tokens, u, counts)


def test_no_sequences(R):
    r = R.rslm_verify(torch.empty((0, 3, 50), device="cuda"), torch.empty((0, 2), dtype=torch.int64, device="cuda"),
                      torch.empty((0, 3), device="cuda"))
    assert r.tokens.shape == (0, 3) and r.accepted.shape == (0,)


def test_other_stream_and_captured(R):
    z, d, tokens, u = (t.cuda() for t in make(6, 3, 6000, "f32", 4))
    want = R.rslm_verify(z, tokens, u, draft=d)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    other = R.rslm_verify(z, tokens, u, draft=d, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other.tokens, want.tokens) and torch.equal(other.logprob, want.logprob)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = R.rslm_verify(z, tokens, u, draft=d)
    for seed in range(4):
        u.copy_(torch.rand((6, 4), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        got = [t.clone() for t in (r.tokens, r.accepted, r.logprob)]
        e = R.rslm_verify(z, tokens, u, draft=d)
        R.rslm_verify(z[:1], tokens[:1], u[:1])
        torch.cuda.synchronize()
        assert torch.equal(got[0], e.tokens) and torch.equal(got[1], e.accepted) and torch.equal(got[2], e.logprob)


@pytest.mark.parametrize("b,k,n", [(1, 4, 131072), (24, 3, 40000), (70, 2, 9000)])
def test_calls_one_after_another(R, b, k, n):
    """Two inputs in turn, whose sums are written to the same memory: each call draws from its
    own, whichever workgroup of a sequence comes last."""
    calls = []
    for seed in (1, 2):
        z, d, tokens, u = make(b, k, n, "f32", seed)
        r = check(R, z, d, tokens, u)
        calls.append(([t.cuda() for t in (z, tokens, u)], d.cuda(), r))
    for i in range(60):
        (z, tokens, u), d, want = calls[i % 2]
        r = R.rslm_verify(z, tokens, u, draft=d)
        assert torch.equal(r.tokens, want.tokens) and torch.equal(r.accepted, want.accepted)
        assert torch.equal(r.logprob, want.logprob)
        del r
