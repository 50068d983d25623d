"""A softmax over a whole 4-bit collection: trains a query adapter, then serves with it.

    python examples/collection_softmax.py [--vectors 100000] [--dim 384] [--batch 256] [--steps 40]

The collection is rotated and kept as 4-bit (MX4) rows.  Queries q are noisy,
linearly distorted vectors of it; the adapter W (dim x dim) is trained so that
q W scores its own vector above all others:

    x = rotate(q W), scores = x b^T, loss = -mean log softmax(scores / T)[target]

with every gradient from the framework: of the log probability to the scores, of
the scores to x, back through the rotation.  No score is left out and no
negatives are drawn: a step normalises over every vector.  Afterwards single
queries are answered (log probability of each answer, entropy), and batches by
the product of 4-bit with 4-bit rows.
"""

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_30384_amd as R  # noqa: E402


def make_collection(n, dim, seed, device="cuda"):
    """Unit vectors, and the distortion of the queries."""
    g = torch.Generator(device=device).manual_seed(seed)
    v = torch.randn(n, dim, generator=g, device=device)
    v /= v.norm(dim=1, keepdim=True)
    distort = torch.eye(dim, device=device) + 4.0 * torch.randn(dim, dim, generator=g, device=device) / dim ** 0.5
    return v, distort, g


class CollectionSoftmax:
    """log softmax over the products with a rotated 4-bit collection."""

    def __init__(self, vectors, temperature=0.05):
        self.plan = R.Plan(vectors.shape[1], 4)
        self.rows = R.rslm_mx4_quantize(vectors, self.plan)
        self.scale = 1.0 / temperature

    def scores(self, x):
        rotated = R.rslm_fwht(self.plan, x)
        return R.rslm_mx4_score(rotated, self.rows)

    def loss(self, x, target):
        """Mean negative log probability of the targets, and its gradient for x."""
        scores = self.scores(x)
        lp = R.rslm_logprob(scores, target, scale=self.scale)
        share = torch.full((x.shape[0],), -1.0 / x.shape[0], device=x.device)
        dscores = R.rslm_logprob_backward(scores, target, lp, share, scale=self.scale, out=scores)
        dx = R.rslm_mx4_score_backward(dscores, self.rows)
        return -lp.logprob.mean(), R.rslm_fwht(self.plan, dx, inverse=True)

    def answer(self, x, k):
        """The k most likely vectors of each query: ids, log probabilities, entropy."""
        lp = R.rslm_logprob(self.scores(x), k=k, scale=self.scale)
        return lp.top_ids, lp.top_logprob, lp.entropy

    def answer_4bit(self, x, k):
        """The same with the queries in 4 bits too."""
        q = R.rslm_mx4_quantize(x, self.plan)
        lp = R.rslm_logprob(R.rslm_mx4_matmul(q, self.rows), k=k, scale=self.scale)
        return lp.top_ids, lp.top_logprob, lp.entropy


def run(vectors=100_000, dim=384, batch=256, steps=40, lr=0.1, seed=0, tell=print):
    v, distort, g = make_collection(vectors, dim, seed)
    model = CollectionSoftmax(v)
    w = torch.eye(dim, device="cuda")

    def queries(m):
        target = torch.randint(0, vectors, (m,), generator=g, device="cuda")
        q = v[target] @ distort
        return q + 0.02 * torch.randn(m, dim, generator=g, device="cuda"), target

    losses = []
    for step in range(steps):
        q, target = queries(batch)
        loss, dx = model.loss(q @ w, target)
        w -= lr * (q.t() @ dx)
        losses.append(loss)
        if step % 10 == 0 or step == steps - 1:
            tell(f"step {step:3d}  loss {float(loss):.3f}")
    q, target = queries(1024)
    found = {}
    for name, call in (("float queries", model.answer), ("4-bit queries", model.answer_4bit)):
        ids, logs, entropy = call(q @ w, 10)
        found[name] = (float((ids[:, 0] == target).float().mean()),
                       float((ids == target[:, None]).any(1).float().mean()))
        tell(f"{name}: right vector first {found[name][0]:.3f}, among ten {found[name][1]:.3f}, "
             f"mean entropy {float(entropy.mean()):.2f}")
    one = (q[:1] @ w).contiguous()
    for _ in range(3):
        model.answer(one, 10)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(100):
        model.answer(one, 10)
    torch.cuda.synchronize()
    tell(f"one query: {(time.perf_counter() - t) * 1e4:.0f} us")
    return [float(x) for x in losses], found


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--vectors", type=int, default=100_000)
    p.add_argument("--dim", type=int, default=384)
    p.add_argument("--batch", type=int, default=256)
    p.add_argument("--steps", type=int, default=40)
    a = p.parse_args()
    run(a.vectors, a.dim, a.batch, a.steps)
