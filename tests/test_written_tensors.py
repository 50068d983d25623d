"""What the calls write into a tensor of the caller's counts for autograd as a change in
place.  Without a GPU: the library is replaced by one whose calls do nothing, the tensors say
that they are on a device.
"""

import types

import pytest

torch = pytest.importorskip("torch")

from paper_2608_30384_amd import api

I64 = torch.int64


class OnDevice(torch.Tensor):
    """A tensor of the CPU that passes for one of a device."""

    is_cuda = property(lambda self: True)


def t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


def rows_of(kind, n, dim):
    steps = -(-dim // 128)
    return kind(t(n, kind._bytes * steps, dtype=torch.uint8), t(n, 4 * steps, dtype=torch.uint8), dim)


@pytest.fixture(autouse=True)
def library(monkeypatch):
    class Library:
        def __getattr__(self, name):
            return lambda *a: 0

    monkeypatch.setattr(api.L, "lib", lambda: Library())
    monkeypatch.setattr(api, "_launch_stream", lambda stream, device: 0)
    monkeypatch.setattr(api, "_raw_stream", lambda stream=None, device=None: 0)
    monkeypatch.setattr(api._WS, "get", lambda *a, **k: torch.empty(256, dtype=torch.uint8))


N, DIM, ROWS = 4, 96, 9
PLAN = types.SimpleNamespace(handle=types.SimpleNamespace(value=0), dim=DIM, device=torch.device("cpu"), canon_bytes=48,
                             record_bytes=52, code_bytes=lambda n: 64)
U8, I32 = torch.uint8, torch.int32

# name: (tensors to write to, the call with them)
CALLS = {
    "mx4_quantize": (lambda: rows_of(api.Mx4Rows, N, DIM), lambda r: api.rslm_mx4_quantize(t(N, DIM), rows=r)),
    "mx8_quantize": (lambda: rows_of(api.Mx8Rows, N, DIM), lambda r: api.rslm_mx8_quantize(t(N, DIM), rows=r)),
    "mx4_dequantize": (lambda: t(N, DIM), lambda o: api.rslm_mx4_dequantize(rows_of(api.Mx4Rows, N, DIM), out=o)),
    "mx8_dequantize": (lambda: t(N, DIM), lambda o: api.rslm_mx8_dequantize(rows_of(api.Mx8Rows, N, DIM), out=o)),
    "mx4_matmul": (lambda: t(N, ROWS), lambda o: api.rslm_mx4_matmul(rows_of(api.Mx4Rows, N, DIM), rows_of(api.Mx4Rows, ROWS, DIM), out=o)),
    "mx4_score": (lambda: t(N, ROWS), lambda o: api.rslm_mx4_score(t(N, DIM), rows_of(api.Mx4Rows, ROWS, DIM), out=o)),
    "mx4_score_backward": (lambda: t(N, DIM), lambda o: api.rslm_mx4_score_backward(t(N, ROWS), rows_of(api.Mx4Rows, ROWS, DIM), out=o)),
    "mx8_score": (lambda: t(N, ROWS), lambda o: api.rslm_mx8_score(rows_of(api.Mx8Rows, N, DIM), rows_of(api.Mx4Rows, ROWS, DIM), out=o)),
    "rmsnorm": (lambda: t(N, DIM), lambda o: api.rslm_rmsnorm(t(N, DIM), residual=t(N, DIM), h=o)),
    "rmsnorm_in_place": (lambda: t(N, DIM), lambda o: api.rslm_rmsnorm(o, residual=t(N, DIM), h=o)),
    "rmsnorm_backward": (lambda: t(N, DIM), lambda o: api.rslm_rmsnorm_backward(
        t(N, DIM), types.SimpleNamespace(h=t(N, DIM), rstd=t(N)), out=o)),
    "embed": (lambda: t(N, DIM), lambda o: api.rslm_embed(t(ROWS, DIM), t(N, dtype=I64), out=o)),
    "mx4_embed": (lambda: t(N, DIM), lambda o: api.rslm_embed(rows_of(api.Mx4Rows, ROWS, DIM), t(N, dtype=I64), out=o)),
    "embed_backward": (lambda: t(ROWS, DIM), lambda o: api.rslm_embed_backward(t(N, DIM), t(N, dtype=I64), ROWS, out=o)),
    "logprob_backward": (lambda: t(N, ROWS), lambda o: api.rslm_logprob_backward(
        t(N, ROWS), t(N, dtype=I64), types.SimpleNamespace(scale=1.0, lse=t(N), stats=t(N, 2), entropy=t(N)), t(N), out=o)),
    "fwht": (lambda: t(N, DIM), lambda o: api.rslm_fwht(PLAN, t(N, DIM), o)),
    "encode": (lambda: (t(256, dtype=U8), t(N, dtype=I32), t(N, DIM)),
               lambda o: api.rslm_encode(PLAN, t(N, DIM), o[0], o[1], resid_rot=o[2])),
    "encode_two_stage": (lambda: (t(256, dtype=U8), t(N, dtype=I32), t(256, dtype=U8), t(N, dtype=I32)),
                         lambda o: api.rslm_encode_two_stage(PLAN, PLAN, t(N, DIM), *o)),
    "encode_sq8": (lambda: (t(256, dtype=U8), t(N, dtype=I32), t(N, DIM, dtype=U8)),
                   lambda o: api.rslm_encode_sq8(PLAN, t(N, DIM), o[0], o[1], t(DIM), t(DIM), o[2])),
    "decode": (lambda: t(N, DIM), lambda o: api.rslm_decode(PLAN, t(256, dtype=U8), t(N, dtype=I32), N, out=o)),
    "score": (lambda: t(N, ROWS), lambda o: api.rslm_score(PLAN, t(ROWS, 52, dtype=U8), t(N, DIM), out=o)),
    "assign_probe": (lambda: (t(N, dtype=I32), t(N)), lambda o: api.ivf_assign_probe(t(N, DIM), t(ROWS, DIM), out_ids=o[0], out_scores=o[1])),
    "assign_probe_noalloc": (lambda: (t(N, dtype=I32), t(N)), lambda o: api.ivf_assign_probe_noalloc(t(N, DIM), t(ROWS, DIM), 1, 0, *o)),
    "kmeans_update": (lambda: t(ROWS, DIM), lambda o: api.ivf_kmeans_update(t(N, DIM), t(N, dtype=I32), o)),
    "sq8_fit": (lambda: (t(DIM), t(DIM)), lambda o: api.rslm_sq8_fit(t(N, DIM), *o, accumulate=True)),
    "sq8_encode": (lambda: t(N, DIM, dtype=U8), lambda o: api.rslm_sq8_encode(t(N, DIM), t(DIM), t(DIM), o)),
    "scan_topk": (lambda: (t(N, 3), t(N, 3, dtype=I32)), lambda o: api.rslm_scan_topk(
        PLAN, types.SimpleNamespace(c_struct=lambda: api.L.Index()), t(N, DIM), t(N, 2, dtype=I32), t(N, 2), 3, *o)),
    "rescore": (lambda: (t(N, 3), t(N, 3, dtype=I32)), lambda o: api.rslm_rescore(
        t(ROWS, DIM, dtype=U8), t(DIM), t(DIM), t(N, DIM), t(N, 5), t(N, 5, dtype=I32), 3, *o)),
    "rescore_rslm": (lambda: (t(N, 3), t(N, 3, dtype=I32)), lambda o: api.rslm_rescore_rslm(
        PLAN, t(ROWS, 48, dtype=U8), t(ROWS, dtype=I32), t(N, DIM), t(N, 5), t(N, 5, dtype=I32), 3, *o)),
}


@pytest.mark.parametrize("name", CALLS)
def test_versions(name):
    make, call = CALLS[name]
    o = make()
    written = [o.codes, o.scales] if hasattr(o, "codes") else list(o) if isinstance(o, tuple) else [o]
    before = [w._version for w in written]
    call(o)
    assert all(w._version > b for w, b in zip(written, before))


def test_the_gradient_that_needed_it_raises():
    w, x = torch.ones(N, DIM, requires_grad=True), t(N, DIM)
    loss = (w * x).sum()
    api.rslm_rmsnorm(x, residual=t(N, DIM), h=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_results_with_a_history_are_not_written_over():
    leaf = torch.ones(N, DIM, requires_grad=True)
    with torch.no_grad():
        param = t(N, DIM)
    for out in (2 * leaf, (2 * leaf)[:], (2 * leaf).view(N, DIM)):
        out = out.as_subclass(OnDevice)
        with pytest.raises(ValueError, match="require a gradient"):
            api.rslm_rmsnorm(param, residual=param, h=out)
        with torch.no_grad():
            api.rslm_rmsnorm(param, residual=param, h=out)
        api.rslm_rmsnorm(param, residual=param, h=out.detach())
    # a parameter itself, or a part of it, is loaded so
    api.rslm_mx4_dequantize(rows_of(api.Mx4Rows, N, DIM), out=param.requires_grad_())
    api.rslm_mx4_dequantize(rows_of(api.Mx4Rows, 2, DIM), out=param[:2])


def test_inference_tensors_have_no_version():
    with torch.inference_mode():
        o = t(N, DIM)
        api.rslm_mx4_dequantize(rows_of(api.Mx4Rows, N, DIM), out=o)
    api.rslm_mx4_dequantize(rows_of(api.Mx4Rows, N, DIM), out=o)
