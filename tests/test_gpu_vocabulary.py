"""The calls at both ends of a model with a 4-bit vocabulary, one after the other.

Serving: tokens looked up in the 4-bit table, the residual's addition and norm to 8 bits,
the product with the vocabulary's 4-bit rows, and the verification of drafted tokens.
Training: lookup in a float table, norm, scores, log probabilities, and the gradients
back to the table and the norm's weight.
"""

import numpy as np
import pytest

from oracle import mx4, mx8

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def R():
    import paper_2608_30384_amd as R

    return R


def serving(R, dim, vocabulary, b, k, seed, rotated):
    """The state of one step, and the step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    plan = R.Plan(dim, 4) if rotated else None
    rows = R.rslm_mx4_quantize(torch.randn((vocabulary, dim), generator=g, device="cuda"), plan)
    s = dict(rows=rows, weight=1 + 0.2 * torch.randn((dim,), generator=g, device="cuda"),
             residual=torch.randn((b * (k + 1), dim), generator=g, device="cuda").bfloat16(),
             ids=torch.randint(0, vocabulary, (b, k + 1), generator=g, device="cuda"),
             draft=torch.randn((b, k, vocabulary), generator=g, device="cuda").bfloat16(),
             uniforms=torch.rand((b, k + 1), generator=g, device="cuda"))

    def step():
        x = R.rslm_embed(rows, s["ids"].view(-1), scale=0.7, dtype=torch.bfloat16)
        norm = R.rslm_rmsnorm(x, s["weight"], residual=s["residual"], y=False, rows=True)
        scores = R.rslm_mx8_score(norm.rows, rows, dtype=torch.bfloat16).view(b, k + 1, vocabulary)
        # the drafted tokens are those that were looked up, behind the first
        r = R.rslm_verify(scores, s["ids"][:, 1:].contiguous(), s["uniforms"], draft=s["draft"], scale=0.1)
        return x, norm, scores, r

    return s, step


@pytest.mark.parametrize("dim,vocabulary,b,k", [(96, 517, 3, 2), (768, 5000, 8, 4), (256, 131072, 1, 3), (130, 300, 70, 1)])
@pytest.mark.parametrize("rotated", [False, True])
def test_serving(R, dim, vocabulary, b, k, rotated):
    s, step = serving(R, dim, vocabulary, b, k, dim + b, rotated)
    x, norm, scores, r = step()
    table = mx4.values(s["rows"].codes.cpu().numpy(), s["rows"].scales.cpu().numpy(), dim)
    ids = s["ids"].cpu().numpy().reshape(-1)
    want = (torch.from_numpy(table[ids]).float() * 0.7).bfloat16()
    assert torch.equal(x.cpu(), want)
    h = (want.float() + s["residual"].cpu().float()).bfloat16()
    assert torch.equal(norm.h.cpu(), h)
    a = mx8.values(norm.rows.codes.cpu().numpy(), norm.rows.scales.cpu().numpy(), dim)
    y, _ = mx8.rmsnorm(h.double().numpy(), s["weight"].double().cpu().numpy(), 1e-6)
    # half a unit of E4M3, or of its subnormals in a block whose largest is at most 448 units
    top = np.abs(np.pad(y, ((0, 0), (0, -dim % 32)))).reshape(len(y), -1, 32).max(-1).repeat(32, 1)[:, :dim]
    assert (np.abs(a - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * top / 224) * (1 + 1e-4) + 1e-30).all()
    exact, terms = a @ table.T, np.abs(a) @ np.abs(table).T
    got = scores.double().cpu().numpy().reshape(exact.shape)
    tol = (2 * (3 * dim + 16) * 2.0 ** -24 + 7 * 2.0 ** -13) * terms
    assert (np.abs(got - exact) <= tol + 2.0 ** -8 * (np.abs(exact) + tol)).all()
    tokens, accepted, logprob = mx8.verify(scores.double().cpu().numpy(), s["ids"][:, 1:].cpu().numpy(), s["uniforms"].cpu().numpy(),
                                           s["draft"].double().cpu().numpy(), scale=float(np.float32(0.1)))
    assert np.array_equal(r.tokens.cpu().numpy(), tokens) and np.array_equal(r.accepted.cpu().numpy(), accepted)
    assert np.abs(r.logprob.double().cpu().numpy() - logprob).max() <= 2.0 ** -24 * np.abs(logprob).max() + 1e-10


def test_two_captured_steps_in_turn(R):
    """Two graphs of different sizes, replayed in turn with eager steps between them."""
    states = [serving(R, 768, 5000, 8, 4, 1, False), serving(R, 96, 70000, 2, 1, 2, True)]
    graphs = []
    for s, step in states:
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for turn in range(3):
        for s, _ in states:
            s["ids"].copy_(torch.randint(0, s["rows"].n, s["ids"].shape, generator=torch.Generator().manual_seed(turn)))
            s["uniforms"].copy_(torch.rand(s["uniforms"].shape, generator=torch.Generator().manual_seed(turn)))
        for graph, _ in graphs:
            graph.replay()
        for (graph, (x, norm, scores, r)), (s, step) in zip(graphs, states):
            ex, en, es, er = step()
            torch.cuda.synchronize()
            assert torch.equal(x, ex) and torch.equal(norm.rows.codes, en.rows.codes) and torch.equal(scores, es)
            assert torch.equal(r.tokens, er.tokens) and torch.equal(r.logprob, er.logprob)


@pytest.mark.parametrize("n,tokens,dim,vocabulary", [(7, 50, 96, 500), (300, 90, 40, 333)])
def test_training(R, n, tokens, dim, vocabulary):
    """Loss and gradients against float64 autograd.  Each of the calls is off by at most
    e = 2 (3 L + 16) 2^-24 of the sum of its terms' magnitudes, L its longest sum; so the
    gradients of a chain of six are within 6 e, of the same chain taken over magnitudes
    (a row's norm passes an error of its input on with at most three times its size)."""
    g = torch.Generator(device="cuda").manual_seed(n)
    table = torch.randn((tokens, dim), generator=g, device="cuda")
    weight = 1 + 0.2 * torch.randn((dim,), generator=g, device="cuda")
    rows = R.rslm_mx4_quantize(torch.randn((vocabulary, dim), generator=g, device="cuda"))
    ids = torch.randint(-1, tokens, (n,), generator=g, device="cuda")
    target = torch.randint(0, vocabulary, (n,), generator=g, device="cuda")
    scale, eps = 0.2, 1e-3

    x = R.rslm_embed(table, ids, scale=1.5)
    norm = R.rslm_rmsnorm(x, weight, eps=eps)
    scores = R.rslm_mx4_score(norm.y, rows)
    lp = R.rslm_logprob(scores, target, scale=scale)
    dscores = R.rslm_logprob_backward(scores, target, lp, torch.full((n,), -1.0 / n, device="cuda"))
    dx, dweight = R.rslm_rmsnorm_backward(R.rslm_mx4_score_backward(dscores, rows), norm, weight)
    dtable = R.rslm_embed_backward(dx, ids, tokens, scale=1.5)

    t, w = table.double().cpu().requires_grad_(), weight.double().cpu().requires_grad_()
    b = torch.from_numpy(mx4.values(rows.codes.cpu().numpy(), rows.scales.cpu().numpy(), dim))
    on = (ids >= 0).cpu()
    x64 = torch.where(on[:, None], t[ids.clamp(min=0).cpu()] * 1.5, 0.0)
    rstd = 1 / torch.sqrt((x64 * x64).mean(1, keepdim=True) + eps)
    y64 = x64 * rstd * w
    z = (y64 @ b.t()) * float(np.float32(scale))
    logs = torch.log_softmax(z, 1)
    loss = -logs[torch.arange(n), target.cpu()].mean()
    loss.backward()
    assert abs(float(lp.logprob.double().mean()) + float(loss.detach())) < 1e-4
    # magnitudes
    p = logs.exp().detach()
    hit = torch.zeros_like(p)
    hit[torch.arange(n), target.cpu()] = 1
    ds = (p + hit) * scale / n
    # the scores' own error moves p by its size: |dz| <= scale e sum |y b|, of which p and ds follow
    e = 2 * (3 * max(dim, vocabulary, n) + 16) * 2.0 ** -24
    ds = ds * (1 + scale * (y64.abs().detach() @ b.abs().t()).max())
    gy = (ds @ b.abs()) * w.abs().detach()
    u = (x64 * rstd).abs().detach()
    dx_abs = rstd.detach() * (gy + u * (gy * u).mean(1, keepdim=True)) * 3
    dt_abs = torch.zeros((tokens, dim), dtype=torch.float64).index_add_(0, ids.clamp(min=0).cpu(), torch.where(on[:, None], dx_abs, 0.0) * 1.5)
    dw_abs = ((ds @ b.abs()) * u).sum(0) * 3
    assert ((dtable.double().cpu() - t.grad).abs() <= 6 * e * dt_abs + 1e-12).all()
    assert ((dweight.double().cpu() - w.grad).abs() <= 6 * e * dw_abs + 1e-12).all()
    # The bound is one of worst cases: about a tenth of the gradient, as the terms of its sums
    # cancel to a hundredth.  It tells a wrong sign or a lost term; the stages by themselves,
    # each from what the one before gave, are held to their own bounds.
    assert 6 * e * float(dt_abs.norm()) < 0.5 * float(t.grad.norm())
    dy = R.rslm_mx4_score_backward(dscores, rows).double().cpu()
    ds = dscores.double().cpu()
    assert ((dy - ds @ b).abs() <= 2 * (3 * vocabulary + 16) * 2.0 ** -24 * (ds.abs() @ b.abs())).all()
    dx64, dw64 = mx8.rmsnorm_grad(x.double().cpu().numpy(), w.detach().numpy(), eps, dy.numpy(), 0.0)
    gy = dy.abs() * w.abs().detach()
    dx_abs = rstd.detach() * (gy + u * (gy * u).mean(1, keepdim=True))
    assert ((dx.double().cpu() - torch.from_numpy(dx64)).abs() <= (96 + dim) * 2.0 ** -24 * dx_abs + 1e-30).all()
    assert ((dweight.double().cpu() - torch.from_numpy(dw64)).abs() <= (96 + dim + n) * 2.0 ** -24 * (dy.abs() * u).sum(0)).all()
    dt64, terms, count = mx8.embed_grad(dx.double().cpu().numpy(), ids.cpu().numpy(), tokens, 1.5)
    assert (np.abs(dtable.double().cpu().numpy() - dt64) <= (count[:, None] + 2) * 2.0 ** -24 * terms).all()
