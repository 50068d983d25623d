"""The example that runs 4-bit rows and log probabilities together.

Tolerance of the loss and of its gradient (in norm): a score is off by at most
2 (3 dim + 16) 2^-24 of the sum of its terms' magnitudes (below 8 here: |x| up
to about 6, times unit vectors), so z = 20 score by 20 * 8 * 632 * 2^-24 = 6e-3
at dim 100, and p and the gradient by twice that at most relative to themselves."""

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    from examples import collection_softmax

    return collection_softmax


@pytest.mark.parametrize("n,dim,m", [(3001, 100, 37), (5000, 128, 1), (700, 257, 130)])
def test_loss_and_gradient(example, n, dim, m):
    v, distort, g = example.make_collection(n, dim, 3)
    model = example.CollectionSoftmax(v)
    target = torch.randint(0, n, (m,), generator=g, device="cuda")
    x = v[target] @ distort
    loss, dx = model.loss(x, target)
    import paper_2608_30384_amd as R

    rotation = R.rslm_fwht(model.plan, torch.eye(dim, device="cuda")).double()     # rows: the unit vectors'
    values = R.rslm_mx4_dequantize(model.rows).double()
    y = x.double().requires_grad_()
    z = (y @ rotation) @ values.t().contiguous() * model.scale
    want = -(z.gather(1, target[:, None])[:, 0] - torch.logsumexp(z, 1)).mean()
    want.backward()
    tol = 2 * 20 * 8 * 2 * (3 * dim + 16) * 2.0 ** -24
    assert abs(float(loss) - float(want)) <= tol
    assert float((dx.double() - y.grad).norm()) <= tol * float(y.grad.norm())


def test_training_and_answers(example):
    lines = []
    losses, found = example.run(vectors=5003, dim=100, batch=64, steps=30, tell=lines.append)
    assert losses[-1] < 0.1 * losses[0]
    for first, ten in found.values():
        assert first > 0.9 and ten > 0.97
    assert lines[-1].startswith("one query")
