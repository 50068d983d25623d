"""The README's examples from Python run as they stand, and scores of its 8-bit and 4-bit rows
are those of the vectors that were quantised.

E2M1 codes are off by at most a quarter of a value, or of the block's scale, which is at most a
quarter of its largest of 32 (of Gaussian values about 2.1 deviations): 0.25 sqrt(1 + 0.28)
= 0.28 of the vector's length; E4M3's by 2^-4.  Errors of different coordinates are independent
of each other and of the other factor, so scores are off by less than 0.3 of their own size, as
root mean squares over some thousand.  Rows of different bases would be off by sqrt(2).
"""

import os
import re

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_examples():
    import paper_2608_30384_amd as R

    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    assert len(blocks) >= 2
    g = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    dim, vocabulary_size, b, k = 768, 3000, 5, 3
    m = b * (k + 1)
    vectors = normal(vocabulary_size, dim)
    s = dict(R=R, torch=torch, dim=dim, b=b, k=k, vectors=vectors, vocabulary=vectors, x=normal(m, dim),
             target=torch.randint(0, vocabulary_size, (m,), generator=g, device="cuda"), dlogprob=normal(m), dentropy=normal(m),
             table=normal(400, dim), ids=torch.randint(0, 400, (m,), generator=g, device="cuda"), weight=1 + 0.2 * normal(dim),
             drafted=torch.randint(0, vocabulary_size, (b, k), generator=g, device="cuda"),
             uniforms=torch.rand((b, k + 1), generator=g, device="cuda"), draft_scores=normal(b, k, vocabulary_size).bfloat16(),
             dy=normal(m, dim))
    for block in blocks:
        s.update(scores=None, rotated=None)
        exec(block, s)
        left = s["n"].y if "n" in s else s["x"]
        want = left.double() @ vectors.double().t().contiguous()
        for name in ("scores", "rotated"):
            if s[name] is not None:
                assert (s[name].double() - want).square().mean().sqrt() < 0.3 * want.square().mean().sqrt(), name
    assert s["v"].tokens.shape == (b, k + 1) and s["dtable"].shape == s["table"].shape and s["back"].shape == s["x"].shape
