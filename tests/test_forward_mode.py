"""Forward-mode tangents are refused as gradients are: the results would not have them.  No
GPU needed, as the calls look at this first."""

import types

import pytest

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as fw

from paper_2608_30384_amd import api

from .test_written_tensors import I64, DIM, N, ROWS, library, rows_of, t  # noqa: F401

CALLS = {
    "mx4_score": lambda d: api.rslm_mx4_score(d, rows_of(api.Mx4Rows, ROWS, DIM)),
    "mx4_score_backward": lambda d: api.rslm_mx4_score_backward(d, rows_of(api.Mx4Rows, DIM, 40)),
    "rmsnorm": lambda d: api.rslm_rmsnorm(d),
    "rmsnorm_weight": lambda d: api.rslm_rmsnorm(t(N, DIM), d[0]),
    "rmsnorm_residual": lambda d: api.rslm_rmsnorm(t(N, DIM), residual=d),
    "rmsnorm_backward": lambda d: api.rslm_rmsnorm_backward(d, types.SimpleNamespace(h=t(N, DIM), rstd=t(N))),
    "rmsnorm_backward_dh": lambda d: api.rslm_rmsnorm_backward(t(N, DIM), types.SimpleNamespace(h=t(N, DIM), rstd=t(N)), dh=d),
    "embed": lambda d: api.rslm_embed(d, t(N, dtype=I64)),
    "embed_backward": lambda d: api.rslm_embed_backward(d, t(N, dtype=I64), ROWS),
    "logprob": lambda d: api.rslm_logprob(d),
    "logprob_backward": lambda d: api.rslm_logprob_backward(
        t(N, DIM), t(N, dtype=I64), types.SimpleNamespace(scale=1.0, lse=t(N), stats=t(N, 2), entropy=t(N)), d[:, 0].contiguous()),
    "out": lambda d: api.rslm_mx8_dequantize(rows_of(api.Mx8Rows, N, DIM), out=d.as_subclass(type(t(1)))),
    "verify": lambda d: api.rslm_verify(d[:, None], t(N, 0, dtype=I64), t(N, 1)),
}


@pytest.mark.parametrize("name", CALLS)
def test_tangents(name):
    with fw.dual_level():
        primal = torch.zeros(N, DIM)
        d = fw.make_dual(primal, torch.ones(N, DIM))
        with pytest.raises(ValueError, match="tangent"):
            CALLS[name](d)
        with torch.no_grad(), pytest.raises(ValueError, match="tangent"):     # which does not turn forward mode off
            CALLS[name](d)


class Twice(torch.autograd.Function):
    """A call inside a function that gives the derivatives itself."""

    @staticmethod
    def forward(x):
        return api.rslm_rmsnorm(x.as_subclass(type(t(1)))).y

    @staticmethod
    def setup_context(ctx, inputs, output):
        pass

    @staticmethod
    def jvp(ctx, tangent):
        return 2 * tangent


def test_inside_a_function_of_its_own():
    with fw.dual_level():
        assert (fw.unpack_dual(Twice.apply(fw.make_dual(torch.zeros(N, DIM), torch.ones(N, DIM)))).tangent == 2).all()
