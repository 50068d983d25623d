"""Representative calls of the operators at both ends of a model with a 4-bit
vocabulary, for timing and comparison: tokens looked up in a table and that
table's gradient, the residual's addition with a root-mean-square norm and an
output in 8 bits, products of such 8-bit rows with 4-bit (MX4) rows, and the
verification of drafted tokens against the scores that come of them.

MX8 rows are vectors in microscaled 8-bit floating point: E4M3 codes, one byte a
coordinate, and one E8M0 scale 2^(s - 127) for every 32 coordinates, the least
that keeps them within E4M3's 448.  A row takes 128 bytes of codes and 4 scales
for every 128 coordinates begun; the padding is zero.  MX4 rows have E2M1 codes,
two to a byte with the lower coordinate in the low nibble, and the same scales.

kind "quantize": rows of floats to MX8 rows (as they are, or rotated first) and
back to the values that the codes stand for.  "score": the product of MX8 rows
with MX4 rows.  "norm": h = x + residual and its norm, in 8 bits, or in floats
with the gradients ("grad").  "embed": rows of a float or an MX4 table for given
tokens, with "grad" the table's gradient too.  "verify": how many drafted tokens
of each sequence stand, and the token after them.

Sizes are those of the benchmark's configurations (dimensions 96, 768 and
1,024, batches of 256, 65,536 added vectors), the paper's odd dimension 2,049,
and powers of two.
"""

import functools
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # One query made ready for products with a rotated 4-bit collection.
        dict(name="quantize_one_768", kind="quantize", n=1, dim=768, dtype="f32", rotate=True, extra=0),
        # A bulk of queries or of activations, of the same dimension.
        dict(name="quantize_65536x768", kind="quantize", n=65_536, dim=768, dtype="f32", rotate=True, extra=0),
        # One token's output layer over a vocabulary of 131,072 rows.
        dict(name="score_1x131072x768", kind="score", m=1, n=131_072, dim=768, out="f32"),
        # An odd batch against an odd collection of the sweep's dimension.
        dict(name="score_255x100003x1024", kind="score", m=255, n=100_003, dim=1024, out="f32"),
        # A prompt's worth of rows: bound by the matrix cores.
        dict(name="score_8192x32768x4096", kind="score", m=8192, n=32_768, dim=4096, out="bf16"),
        # The norm in front of a layer for a single token.
        dict(name="norm_one_4096", kind="norm", n=1, dim=4096, dtype="bf16", wtype="bf16", residual=True, grad=False, extra=0),
        # Rows of an odd dimension, inside wider ones.
        dict(name="norm_odd_20001x2049", kind="norm", n=20_001, dim=2049, dtype="f32", wtype="f32", residual=True, grad=False, extra=15),
        # The same norm in a training step, forward and backward.
        dict(name="norm_grad_8192x4096", kind="norm", n=8192, dim=4096, dtype="bf16", wtype="f32", residual=True, grad=True, extra=0),
        # The tokens of a decoding batch looked up in a 4-bit table.
        dict(name="embed_256x768", kind="embed", n=256, rows=131_072, dim=768, dtype="bf16", mx4=True, grad=False),
        # A training step's tokens, most of them frequent ones, and the table's gradient.
        dict(name="embed_grad_65536x768", kind="embed", n=65_536, rows=131_072, dim=768, dtype="bf16", mx4=False, grad=True),
        # One sequence with four drafted tokens.
        dict(name="verify_1x4x131072", kind="verify", b=1, k=4, n=131_072, dtype="f32", draft=True, masked=0.0, ragged=False),
        # A serving batch, with fewer drafts for some sequences.
        dict(name="verify_64x4x131072", kind="verify", b=64, k=4, n=131_072, dtype="bf16", draft=True, masked=0.05, ragged=True),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dim(rng, lo=48, hi=4096):
    if rng.random() < 0.5:
        return rng.choice([64, 96, 100, 128, 200, 256, 300, 384, 512, 768, 960, 1024, 1536, 2048, 4096])
    return _log(rng, lo, hi)


def draw(rng):
    kind = rng.choice(["quantize", "score", "score", "norm", "norm", "embed", "embed", "verify", "verify"])
    if kind == "quantize":
        dim = _dim(rng)
        return dict(kind=kind, n=_log(rng, 1, 50_000_000 // dim), dim=dim, dtype=rng.choice(["f32", "f16", "bf16"]),
                    rotate=rng.random() < 0.5, extra=rng.choice([0, 0, 1, 7, 64]))
    if kind == "score":
        dim, m = _dim(rng), _log(rng, 1, 8192)
        n = _log(rng, 64, min(200_000, 268_000_000 // m, 1_000_000_000_000 // (m * dim)))
        return dict(kind=kind, m=m, n=n, dim=dim, out=rng.choice(["f32", "f16", "bf16"]))
    if kind == "norm":
        dim, dtype, grad = _dim(rng, hi=16384), rng.choice(["f32", "f16", "bf16"]), rng.random() < 0.5
        return dict(kind=kind, n=_log(rng, 1, 32_000_000 // dim), dim=dim, dtype=dtype, wtype=rng.choice(["f32", dtype]),
                    residual=rng.random() < 0.7, grad=grad, extra=rng.choice([0, 0, 1, 7, 64]))
    if kind == "embed":
        dim, mx4 = _dim(rng), rng.random() < 0.3
        rows = _log(rng, 500, min(200_000, 100_000_000 // dim))
        return dict(kind=kind, n=_log(rng, 1, min(200_000, 50_000_000 // dim)), rows=rows, dim=dim,
                    dtype=rng.choice(["f32", "f16", "bf16"]), mx4=mx4, grad=not mx4 and rng.random() < 0.8)
    b, k = _log(rng, 1, 256), rng.choice([0, 1, 2, 3, 4, 5, 8])
    return dict(kind=kind, b=b, k=k, n=_log(rng, 1000, min(262_144, 75_000_000 // (b * (2 * k + 1)))),
                dtype=rng.choice(["f32", "f16", "bf16"]), draft=k > 0 and rng.random() < 0.7,
                masked=rng.choice([0.0, 0.0, 0.05, 0.9]), ragged=k > 0 and rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _steps(dim):
    return -(-dim // 128)


def _normal(g, shape, dtype="f32"):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(_TYPES[dtype])


def _uniform(g, shape):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


def _scales(g, r, n, dim):
    """Scales of n rows of unit-norm vectors, a few octaves wide."""
    of = torch.from_numpy((127 - round(math.log2(dim) / 2) + r.integers(-2, 2, 512)).astype(np.uint8)).cuda()
    scales = of.index_select(0, torch.randint(0, 512, (n * 4 * _steps(dim),), generator=g, device="cuda", dtype=torch.int32)).view(n, -1)
    scales[:, -(-dim // 32):] = 0
    return scales


def _rows4(g, seed, n, dim):
    """Codes and scales of n MX4 rows: bytes of close to Gaussian coordinates."""
    r = np.random.default_rng(seed)
    c = np.searchsorted([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], 2.2 * np.abs(r.standard_normal((8192, 2)))) + 8 * r.integers(0, 2, (8192, 2))
    of = torch.from_numpy((c[:, 0] | (c[:, 1] << 4)).astype(np.uint8)).cuda()
    codes = of.index_select(0, torch.randint(0, 8192, (n * 64 * _steps(dim),), generator=g, device="cuda", dtype=torch.int32)).view(n, -1)
    codes[:, (dim + 1) // 2:] = 0
    if dim % 2:
        codes[:, dim // 2] &= 15
    return codes, _scales(g, r, n, dim)


def _rows8(g, seed, n, dim):
    """Codes and scales of n MX8 rows, their coordinates close to Gaussian."""
    r = np.random.default_rng(seed)
    v = np.clip(128 * r.standard_normal(8192), -448, 448)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.abs(v))), -6) - 3)
    e = np.rint(np.abs(v) / step) * step
    x = np.maximum(np.floor(np.log2(np.maximum(e, 2.0 ** -9))), -6)
    c = np.where(e < 2.0 ** -6, e * 512, (x + 7) * 8 + (e / 2.0 ** x - 1) * 8) + 128 * (v < 0)
    of = torch.from_numpy(c.astype(np.uint8)).cuda()
    codes = of.index_select(0, torch.randint(0, 8192, (n * 128 * _steps(dim),), generator=g, device="cuda", dtype=torch.int32)).view(n, -1)
    codes[:, dim:] = 0
    scales = _scales(g, r, n, dim)
    scales[:, : -(-dim // 32)] -= 6
    return codes, scales


def _spread(g, n, dim, extra, dtype):
    """Rows with a power-law variance spectrum and norms that vary, inside rows `extra` wider."""
    wide = _normal(g, (n, dim + extra))
    wide *= torch.arange(1, dim + extra + 1, device="cuda") ** -0.25
    wide *= torch.exp(0.5 * _normal(g, (n, 1)))
    return wide.to(_TYPES[dtype])[:, :dim]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    kind = case["kind"]
    if kind == "quantize":
        s["x"] = _spread(g, case["n"], case["dim"], case["extra"], case["dtype"])
        if case["rotate"]:
            r = np.random.default_rng(seed)
            signs, perm = 1 - 2 * r.integers(0, 2, 256), r.permutation(128)
            s["tables"] = _tables(case["dim"], signs, perm)
            if own:  # the codec plan that holds the rotation
                import paper_2608_30384_amd as R

                s["plan"] = R.Plan(case["dim"], 4, passes=2, signs=signs, perm=perm)
    elif kind == "score":
        s["a"] = _rows8(g, seed + 1, case["m"], case["dim"])
        s["b"] = _rows4(g, seed, case["n"], case["dim"])
    elif kind == "norm":
        n, dim, extra, dtype = case["n"], case["dim"], case["extra"], case["dtype"]
        s["x"] = _spread(g, n, dim, extra, dtype)
        s["residual"] = 3 * _spread(g, n, dim, extra, dtype) if case["residual"] else None
        s["weight"] = (1 + 0.2 * _normal(g, (dim,))).to(_TYPES[case["wtype"]])
        if case["grad"]:
            s["dy"], s["dh"] = 0.01 * _normal(g, (n, dim), dtype), 0.01 * _normal(g, (n, dim), dtype)
    elif kind == "embed":
        n, rows, dim = case["n"], case["rows"], case["dim"]
        s["table"] = _rows4(g, seed, rows, dim) if case["mx4"] else _normal(g, (rows, dim), case["dtype"])
        # frequencies that fall as one over the rank, and a few places that hold no token
        ids = (torch.exp(_uniform(g, (n,)) * math.log(rows)) - 1).to(torch.int64).clamp(max=rows - 1)
        ids = torch.randperm(rows, generator=g, device="cuda")[ids]
        s["ids"] = torch.where(_uniform(g, (n,)) < 0.03, -1, ids)
        s["scale"] = math.sqrt(dim)
        if case["grad"]:
            s["dout"] = 0.01 * _normal(g, (n, dim), case["dtype"])
    else:
        b, k, n = case["b"], case["k"], case["n"]
        z = 3 * _normal(g, (b, k + 1, n))
        if case["masked"]:
            z.masked_fill_(_uniform(g, (b, 1, n)) < case["masked"], -math.inf)
        d = z[:, :k] + 0.7 * _normal(g, (b, k, n))
        s["target"], s["draft"] = z.to(_TYPES[case["dtype"]]), d.to(_TYPES[case["dtype"]])
        s["scale"] = 1.25
        noise = -torch.log(-torch.log(_uniform(g, (b, k, n)).clamp(1e-7, 1 - 1e-7)))
        s["tokens"] = (s["draft"] * s["scale"] + noise).argmax(-1) if k else torch.zeros((b, 0), dtype=torch.int64, device="cuda")
        s["uniforms"] = _uniform(g, (b, k + 1))
        s["counts"] = torch.randint(0, k + 1, (b,), generator=g, device="cuda", dtype=torch.int32) if case["ragged"] else None
        if not case["draft"]:
            s["draft"] = None
    return s


# ------------------------------------------------------------------ plain forms
def _power(e):
    """2^(e - 127) for whole numbers 0 <= e < 255 (e = 0 is subnormal)."""
    e = e.to(torch.int32)
    return torch.where(e > 0, (e << 23).view(torch.float32), 2.0 ** -127)


def _tables(dim, signs, perm):
    """The rotation's tables: sign vectors of both passes and the source of each
    coordinate of the permutation and transpose between them."""
    block = min(128, 1 << (dim.bit_length() - 1))
    bits = block.bit_length() - 1
    inner = perm if block == 128 else np.array([int(format(i, "0%db" % bits)[::-1] or "0", 2) if bits else 0 for i in range(block)])
    m = dim // block
    source = np.arange(dim)
    source[: m * block] = (np.arange(m)[None, :] * block + inner[:, None]).reshape(-1)
    i = np.arange(dim)
    return dict(block=block, source=torch.from_numpy(source).cuda(),
                s1=torch.from_numpy(signs[i % 256].astype(np.float32)).cuda(),
                s2=torch.from_numpy(signs[(i + 127) % 256].astype(np.float32)).cuda())


def _butterfly(x, h):
    y = x.view(*x.shape[:-1], -1, 2, h)
    return torch.stack((y[..., 0, :] + y[..., 1, :], y[..., 0, :] - y[..., 1, :]), -2).view(x.shape)


def _hadamard(x, block):
    """Walsh-Hadamard transform of every whole block, then of the block that ends at the last coordinate."""
    stages = [1 << i for i in range(block.bit_length() - 1)]
    unit = torch.tensor(1.0 / math.sqrt(block), dtype=torch.float32, device=x.device)
    whole = x.shape[1] // block * block
    y = x.clone()
    y[:, :whole] = (functools.reduce(_butterfly, stages, x[:, :whole].reshape(-1, block)) * unit).view(-1, whole)
    if whole < x.shape[1]:
        y[:, -block:] = functools.reduce(_butterfly, stages, y[:, -block:].contiguous()) * unit
    return y


def _quantized(x):
    """The values of the MX8 rows of float32 rows x, in bfloat16, which holds them exactly."""
    n, dim = x.shape
    y = torch.nn.functional.pad(x, (0, -dim % 32)).view(n, -1, 32)
    top = y.abs().amax(-1, keepdim=True).view(torch.int32)
    e = ((top >> 23) - 8 + ((top & 0x7FFFFF) > 0x600000)).clamp_(0, 253)
    v = y * ((254 - e) << 23).view(torch.float32)
    # a unit in the last of E4M3's 3 places: 2^-9 at least
    unit = ((((v.view(torch.int32) >> 23) & 255).clamp_(min=121) - 3) << 23).view(torch.float32)
    v = torch.round(v / unit) * unit * _power(e)
    return torch.where(top < 0x7F800000, v, math.nan).view(n, -1)[:, :dim].to(torch.bfloat16)


def _values4(rows, dim):
    """float32 values of MX4 rows."""
    codes, scales = rows
    n = codes.shape[0]
    c = torch.stack((codes & 15, codes >> 4), -1).view(n, -1, 32).to(torch.int32)
    # E2M1's exponent and mantissa at the low end of float32's, then 2^126 for
    # the difference of the exponents' biases: exact, 0.5 (a subnormal) too
    v = (((c & 7) << 22) | ((c & 8) << 28)).view(torch.float32) * 2.0 ** 126
    return (v * _power(scales)[..., None]).view(n, -1)[:, :dim]


def _values8(rows, dim):
    """float32 values of MX8 rows (E4M3's exponent bias is 7, float32's 127)."""
    codes, scales = rows
    c = codes.view(codes.shape[0], -1, 32).to(torch.int32)
    v = (((c & 127) << 20) | ((c & 128) << 24)).view(torch.float32) * 2.0 ** 120
    return (v * _power(scales)[..., None]).view(codes.shape[0], -1)[:, :dim]


def _plain_norm(s):
    dtype = _TYPES[s["dtype"]]
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dtype)
    hf, w = h.float(), s["weight"].float()
    rstd = torch.rsqrt((hf * hf).mean(1, keepdim=True) + EPS)
    y = hf * rstd * w
    out = {} if s["residual"] is None else dict(h=h)
    if not s["grad"]:
        return dict(out, values=_quantized(y))
    dy, xh = s["dy"].float(), hf * rstd
    g = dy * w
    dx = rstd * (g - xh * (g * xh).mean(1, keepdim=True)) + s["dh"].float()
    return dict(out, y=y.to(dtype), dx=dx.to(dtype), dweight=(dy * xh).sum(0).to(s["weight"].dtype))


def _plain_embed(s):
    dtype, ids, scale = _TYPES[s["dtype"]], s["ids"], s["scale"]
    on, at = (ids >= 0)[:, None], ids.clamp(min=0)
    rows = _values4((s["table"][0][at], s["table"][1][at]), s["dim"]) if s["mx4"] else s["table"][at].float()
    out = dict(out=torch.where(on, rows * scale, 0.0).to(dtype))
    if s["grad"]:
        d = torch.zeros((s["rows"], s["dim"]), dtype=torch.float32, device=ids.device)
        d.index_add_(0, at, torch.where(on, s["dout"].float(), 0.0))
        out["dtable"] = (d * scale).to(dtype)
    return out


def _probabilities(scores, scale):
    """Probabilities and their logarithms, in 64 bits: a sampled token is a value next to a border."""
    z = scores.double() * scale
    top = z.amax(-1, keepdim=True)
    logs = z - top - (z - top).exp().sum(-1, keepdim=True).log()
    return logs.exp(), logs


def _plain_verify(s):
    b, k, n, tokens, u = s["b"], s["k"], s["n"], s["tokens"], s["uniforms"].double()
    p, logs = _probabilities(s["target"], s["scale"])
    count = torch.full((b,), k, device=u.device) if s["counts"] is None else s["counts"].long()
    px = p[:, :k].gather(2, tokens[..., None])[..., 0]
    if s["draft"] is None:
        stands = u[:, :k] < px
    else:
        q = _probabilities(s["draft"], s["scale"])[0]
        stands = u[:, :k] * q.gather(2, tokens[..., None])[..., 0] < px
    place = torch.arange(k + 1, device=u.device)
    stands &= place[:k] < count[:, None]
    accepted = stands.long().cumprod(1).sum(1)
    # the token after those that stand: from p, or from what p has over q
    seq = torch.arange(b, device=u.device)
    r = p[seq, accepted]
    if k:
        at = accepted.clamp(max=k - 1)
        hit = torch.arange(n, device=u.device) == tokens[seq, at][:, None]
        over = torch.where(hit, 0.0, r) if s["draft"] is None else (r - q[seq, at]).clamp(min=0)
        drafted = (accepted < count) & (over.sum(1) > 0)
        r = torch.where(drafted[:, None], over, r)
    c = r.cumsum(1)
    next_one = (c > u[:, k:] * c[:, -1:]).to(torch.int8).argmax(1)
    out = torch.where(place < accepted[:, None], torch.nn.functional.pad(tokens, (0, 1)), -1)
    out[seq, accepted] = next_one
    logprob = torch.where(out < 0, 0.0, logs.gather(2, out.clamp(min=0)[..., None])[..., 0]).float()
    return dict(tokens=out, accepted=accepted.to(torch.int32), logprob=logprob)


def _plain(s):
    kind = s["kind"]
    if kind == "quantize":
        x = s["x"].float()
        if s["rotate"]:
            t = s["tables"]
            x = _hadamard((_hadamard(x * t["s1"], t["block"]))[:, t["source"]] * t["s2"], t["block"])
        return _quantized(x)
    if kind == "score":
        return torch.mm(_values8(s["a"], s["dim"]), _values4(s["b"], s["dim"]).t()).to(_TYPES[s["out"]])
    return {"norm": _plain_norm, "embed": _plain_embed, "verify": _plain_verify}[kind](s)


# ------------------------------------------------------------------ one pass
def run(s):
    if not own:
        return _plain(s)
    import paper_2608_30384_amd as R

    kind = s["kind"]
    if kind == "quantize":
        return R.rslm_mx8_dequantize(R.rslm_mx8_quantize(s["x"], plan=s.get("plan")), dtype=torch.bfloat16)
    if kind == "score":
        return R.rslm_mx8_score(R.Mx8Rows(*s["a"], s["dim"]), R.Mx4Rows(*s["b"], s["dim"]), dtype=_TYPES[s["out"]])
    if kind == "norm":
        r = R.rslm_rmsnorm(s["x"], s["weight"], residual=s["residual"], eps=EPS, y=s["grad"], rows=not s["grad"])
        out = {} if s["residual"] is None else dict(h=r.h)
        if not s["grad"]:
            return dict(out, values=R.rslm_mx8_dequantize(r.rows, dtype=torch.bfloat16))
        dx, dweight = R.rslm_rmsnorm_backward(s["dy"], r, s["weight"], dh=s["dh"])
        return dict(out, y=r.y, dx=dx, dweight=dweight)
    if kind == "embed":
        table = R.Mx4Rows(*s["table"], s["dim"]) if s["mx4"] else s["table"]
        out = dict(out=R.rslm_embed(table, s["ids"], scale=s["scale"], dtype=_TYPES[s["dtype"]]))
        if s["grad"]:
            out["dtable"] = R.rslm_embed_backward(s["dout"], s["ids"], s["rows"], scale=s["scale"])
        return out
    r = R.rslm_verify(s["target"], s["tokens"], s["uniforms"], draft=s["draft"], counts=s["counts"], scale=s["scale"])
    return dict(tokens=r.tokens, accepted=r.accepted, logprob=r.logprob)


# ------------------------------------------------------------------ 64 bits
def _level4():
    level = np.array([0, 1, 2, 3, 4, 6, 8, 12], dtype=np.float64) / 2
    level = np.concatenate([level, -level])
    byte = np.arange(256)
    return torch.from_numpy(np.stack([level[byte & 15], level[byte >> 4]], 1)).cuda()


def _level8():
    byte = np.arange(256)
    e, m = (byte >> 3) & 15, byte & 7
    v = np.where(e == 0, np.ldexp(m / 8.0, -6), np.ldexp(1 + m / 8.0, e - 7))
    return torch.from_numpy(np.where(byte & 128, -v, v)).cuda()


def _values64(rows, dim, level):
    power = torch.from_numpy(np.ldexp(1.0, np.arange(256) - 127)).cuda()

    def some(codes, scales):
        v = level[codes.long()].reshape(codes.shape[0], -1, 32) * power[scales.long()].unsqueeze(-1)
        return v.reshape(codes.shape[0], -1)[:, :dim]

    return torch.cat([some(c, s) for c, s in zip(rows[0].split(4096), rows[1].split(4096))])


def _quantized64(x):
    out = torch.empty_like(x)
    for o in range(0, x.shape[1], 32):
        y = x[:, o:o + 32]
        m, e = torch.frexp(y.abs().amax(1, keepdim=True))  # top = m 2^e, m of [1/2, 1)
        unit = torch.exp2((e - 9 + (m > 0.875)).clamp(min=-127).double())
        v = y / unit
        step = torch.exp2((torch.frexp(v).exponent - 1).clamp(min=-6).double() - 3)
        out[:, o:o + 32] = torch.round(v / step) * step * unit
    return out


def _rotation64(dim, block, s1, source, s2):
    """The rotation as a dense matrix."""
    h = functools.reduce(np.kron, [np.array([[1.0, 1.0], [1.0, -1.0]])] * (block.bit_length() - 1), np.ones((1, 1))) / math.sqrt(block)
    whole = dim // block * block
    blocks = np.eye(dim)
    blocks[:whole, :whole] = np.kron(np.eye(dim // block), h)
    if whole < dim:
        last = np.eye(dim)
        last[-block:, -block:] = h
        blocks = last @ blocks
    return blocks @ (s2[:, None] * (blocks @ np.diag(s1))[source])


def _exact_norm(case, s):
    x = s["x"].double()
    total = x if s["residual"] is None else x + s["residual"].double()
    h = total if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()
    w = s["weight"].double()
    size = torch.sqrt(h.square().mean(1, keepdim=True) + EPS)
    unit = h / size
    out = {} if s["residual"] is None else dict(h=total)
    if not case["grad"]:
        return dict(out, values=_quantized64(unit * w))
    g = s["dy"].double() * w
    along = (g * unit).sum(1, keepdim=True) / case["dim"]
    return dict(out, y=unit * w, dx=(g - along * unit) / size + s["dh"].double(), dweight=(s["dy"].double() * unit).sum(0))


def _exact_embed(case, s):
    ids, on = s["ids"], s["ids"] >= 0
    out = torch.zeros((case["n"], case["dim"]), dtype=torch.float64, device="cuda")
    if case["mx4"]:
        out[on] = _values64((s["table"][0][ids[on]], s["table"][1][ids[on]]), case["dim"], _level4()) * s["scale"]
    else:
        out[on] = s["table"][ids[on]].double() * s["scale"]
    out = dict(out=out)
    if case["grad"]:
        d = torch.zeros((case["rows"], case["dim"]), dtype=torch.float64, device="cuda")
        out["dtable"] = d.index_put_((ids[on],), s["dout"][on].double() * s["scale"], accumulate=True)
    return out


def _exact_verify(case, s):
    k, tokens, accepted, logprob = case["k"], [], [], []
    drafts, uniforms = s["tokens"].tolist(), s["uniforms"].double().tolist()
    counts = [k] * case["b"] if s["counts"] is None else s["counts"].tolist()
    for b in range(case["b"]):
        logs = torch.log_softmax(s["target"][b].double() * s["scale"], -1)
        q = None if s["draft"] is None else torch.softmax(s["draft"][b].double() * s["scale"], -1)
        i = 0
        while i < counts[b]:
            t = drafts[b][i]
            if not uniforms[b][i] * (1.0 if q is None else float(q[i, t])) < float(logs[i, t].exp()):
                break
            i += 1
        r = logs[i].exp()
        if i < counts[b]:
            over = r.clone()
            if q is None:
                over[drafts[b][i]] = 0
            else:
                over = torch.relu(r - q[i])
            r = over if float(over.sum()) > 0 else r
        c = r.cumsum(0)
        chosen = int(torch.searchsorted(c, uniforms[b][k] * c[-1:], right=True)[0])
        row = drafts[b][:i] + [chosen]
        tokens.append(row + [-1] * (k + 1 - len(row)))
        accepted.append(i)
        logprob.append([float(logs[j, t]) for j, t in enumerate(row)] + [0.0] * (k + 1 - len(row)))
    return dict(tokens=torch.tensor(tokens, device="cuda"), accepted=torch.tensor(accepted, dtype=torch.int32, device="cuda"),
                logprob=torch.tensor(logprob, dtype=torch.float64, device="cuda"))


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        if case["dim"] > 2100 and case["rotate"]:
            return None
        x = s["x"].double()
        if case["rotate"]:
            t = {k: v.cpu().numpy() if k != "block" else v for k, v in s["tables"].items()}
            r = _rotation64(case["dim"], t["block"], t["s1"].astype(np.float64), t["source"], t["s2"].astype(np.float64))
            x = torch.mm(x, torch.from_numpy(r).cuda().t().contiguous())
        return _quantized64(x)
    if kind == "score":
        return torch.mm(_values64(s["a"], case["dim"], _level8()), _values64(s["b"], case["dim"], _level4()).t())
    return {"norm": _exact_norm, "embed": _exact_embed, "verify": _exact_verify}[kind](case, s)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n, dim = case["n"], case["dim"]
        # rows read, codes and scales written and read again, values written
        return dict(bytes=n * ((_BYTES[case["dtype"]] + 2) * dim + 2 * (dim + dim / 32)),
                    flops=n * dim * (2 + (2 * 8 if case["rotate"] else 0)))
    if kind == "score":
        m, n, dim = case["m"], case["n"], case["dim"]
        return dict(bytes=n * (dim / 2 + dim / 32) + m * (dim + dim / 32) + m * n * _BYTES[case["out"]], flops=2 * m * n * dim)
    if kind == "norm":
        n, dim, e = case["n"], case["dim"], _BYTES[case["dtype"]]
        parts = 3 if case["residual"] else 1  # x, the residual and h
        w = dim * _BYTES[case["wtype"]]
        if not case["grad"]:  # codes and scales written and read again, values written
            return dict(bytes=n * dim * (parts * e + 2 * (1 + 1 / 32) + 2) + w, flops=8 * n * dim)
        # y; then h, dy, dh and dx
        return dict(bytes=n * dim * e * (parts + 1 + 4) + 3 * w, flops=16 * n * dim)
    if kind == "embed":
        n, dim, e = case["n"], case["dim"], _BYTES[case["dtype"]]
        read = min(n, case["rows"]) * (dim / 2 + dim / 32 if case["mx4"] else dim * e)
        back = (n + case["rows"]) * dim * e + 8 * n if case["grad"] else 0
        return dict(bytes=read + n * dim * e + 8 * n + back, flops=(2 if case["grad"] else 1) * n * dim)
    b, k, n = case["b"], case["k"], case["n"]
    rows = b * (k + 1 + (k if case["draft"] else 0))
    return dict(bytes=rows * n * _BYTES[case["dtype"]] + b * (k + 1) * 24, flops=4 * rows * n)
