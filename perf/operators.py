"""Representative calls of the 4-bit (MX4) operators and of the log
probabilities over scores, for timing and comparison.

MX4 rows are vectors in microscaled 4-bit floating point: E2M1 codes (0, 0.5,
1, 1.5, 2, 3, 4, 6 and their negatives), two to a byte with the lower
coordinate in the low nibble, and one E8M0 scale 2^(s - 127) for every 32
coordinates.  A row takes 64 bytes of codes and 4 scales for every 128
coordinates begun; the padding is zero.

kind "quantize": rows of floats to MX4 rows (as they are, or rotated first) and
back to the values that the codes stand for.  "matmul": the product of two sets
of MX4 rows.  "score": the product of float rows with MX4 rows.  "backward":
the gradient of that product with respect to the float rows.  "logprob": log
probability of a given entry, log-sum-exp, entropy and the most likely entries
of each row of scores, and with "grad" the gradient of the first and third with
respect to the scores.

Sizes are those of the benchmark's configurations (dimensions 96, 768 and
1,024, batches of 256 queries, 4,096 lists, 65,536 added vectors, 1,000,000
records), the paper's odd dimension 2,049, and powers of two.
"""

import functools
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def listed():
    return [
        # One query made ready for a 4-bit collection: launches and latency.
        dict(name="quantize_one_768", kind="quantize", n=1, dim=768, dtype="f32", rotate=True, extra=0),
        # The vectors that one benchmark step adds to a collection.
        dict(name="quantize_add_768", kind="quantize", n=65_536, dim=768, dtype="f32", rotate=True, extra=0),
        # A weight matrix or collection in 16 bits, of an odd dimension, inside
        # wider rows (the compression microbenchmark's dimension).
        dict(name="quantize_odd_2049", kind="quantize", n=40_001, dim=2049, dtype="bf16", rotate=False, extra=15),
        # A batch of 4-bit queries against 4,096 centres.
        dict(name="matmul_256x4096x768", kind="matmul", m=256, n=4096, dim=768, out="f32"),
        # An odd batch against an odd collection of the low-dimensional configuration.
        dict(name="matmul_37x100003x96", kind="matmul", m=37, n=100_003, dim=96, out="f32"),
        # Bulk products: all pairs of two large sets, bound by the matrix cores.
        dict(name="matmul_8192x32768x4096", kind="matmul", m=8192, n=32_768, dim=4096, out="bf16"),
        # One query, or one token's activations, against a million rows: bound
        # by reading them.
        dict(name="score_1x1000000x768", kind="score", m=1, n=1_000_000, dim=768, dtype="bf16", out="f32"),
        # A batch of float32 queries against a collection of the sweep's dimension.
        dict(name="score_256x131072x1024", kind="score", m=256, n=131_072, dim=1024, dtype="f32", out="f32"),
        # Gradients of a few rows' scores over an odd collection.
        dict(name="backward_4x10007x96", kind="backward", m=4, n=10_007, dim=96, dtype="f32"),
        # Gradients of a batch of queries over a large collection.
        dict(name="backward_256x131072x768", kind="backward", m=256, n=131_072, dim=768, dtype="bf16"),
        # One row of scores, as each step of a served model or one query has it.
        dict(name="logprob_1x131072", kind="logprob", m=1, n=131_072, dtype="f32", k=20, masked=0.05, grad=False),
        # A training step's batch of rows, forward and backward.
        dict(name="logprob_4096x32768_grad", kind="logprob", m=4096, n=32_768, dtype="bf16", k=10, masked=0.0, grad=True),
    ]


# ------------------------------------------------------------------ drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dim(rng, lo=48, hi=4096):
    if rng.random() < 0.5:
        return rng.choice([64, 96, 100, 128, 200, 256, 300, 384, 512, 768, 960, 1024, 1536, 2048, 4096])
    return _log(rng, lo, hi)


def draw(rng):
    kind = rng.choice(["quantize", "matmul", "score", "score", "backward", "logprob", "logprob"])
    if kind == "quantize":
        dim = _dim(rng)
        return dict(kind=kind, n=_log(rng, 1, 80_000_000 // dim), dim=dim, dtype=rng.choice(["f32", "f16", "bf16"]),
                    rotate=rng.random() < 0.5, extra=rng.choice([0, 0, 1, 7, 64]))
    if kind == "matmul":
        dim, m = _dim(rng), _log(rng, 1, 8192)
        n = _log(rng, 64, min(200_000, 268_000_000 // m, 1_000_000_000_000 // (m * dim)))
        return dict(kind=kind, m=m, n=n, dim=dim, out=rng.choice(["f32", "f16", "bf16"]))
    if kind in ("score", "backward"):
        dim = _dim(rng)
        m = _log(rng, 1, 16) if rng.random() < 0.5 else _log(rng, 16, 512)
        n = _log(rng, 64, min(1_000_000, 700_000_000 // dim, 30_000_000_000 // (m * dim)))
        c = dict(kind=kind, m=m, n=n, dim=dim, dtype=rng.choice(["f32", "f16", "bf16"]))
        return dict(c, out=rng.choice(["f32", c["dtype"]])) if kind == "score" else c
    m = _log(rng, 1, 4096)
    return dict(kind=kind, m=m, n=_log(rng, 500, min(1_000_000, 130_000_000 // m)), dtype=rng.choice(["f32", "f16", "bf16"]),
                k=rng.choice([0, 1, 5, 20, 100]), masked=rng.choice([0.0, 0.0, 0.05, 0.9]), grad=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
def _steps(dim):
    return -(-dim // 128)


def _normal(g, shape, dtype="f32"):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(_TYPES[dtype])


def _rows(g, seed, n, dim):
    """Codes and scales of n MX4 rows: rotated unit-norm vectors, whose
    coordinates are close to Gaussian, drawn from a table of such bytes."""
    r = np.random.default_rng(seed)
    z = r.standard_normal((512, 32))
    e = np.floor(np.log2(np.abs(z).max(1)))
    v = np.abs(z) / 2.0 ** (e - 2)[:, None]
    c = np.searchsorted([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], v) + 8 * (z < 0)
    codes_of = torch.from_numpy((c[:, 0::2] | (c[:, 1::2] << 4)).astype(np.uint8).reshape(-1)).cuda()
    scales_of = torch.from_numpy((e - 2 + 127 - round(math.log2(dim) / 2) + r.integers(-1, 2, 512)).astype(np.uint8)).cuda()
    codes = codes_of.index_select(0, torch.randint(0, codes_of.numel(), (n * 64 * _steps(dim),), generator=g, device="cuda", dtype=torch.int32)).view(n, -1)
    scales = scales_of.index_select(0, torch.randint(0, scales_of.numel(), (n * 4 * _steps(dim),), generator=g, device="cuda", dtype=torch.int32)).view(n, -1)
    codes[:, (dim + 1) // 2:] = 0
    if dim % 2:
        codes[:, dim // 2] &= 15
    scales[:, -(-dim // 32):] = 0
    return codes, scales


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    kind = case["kind"]
    if kind == "quantize":
        # a power-law variance spectrum and norms that vary from row to row
        wide = _normal(g, (case["n"], case["dim"] + case["extra"]))
        wide *= torch.arange(1, case["dim"] + case["extra"] + 1, device="cuda") ** -0.5
        wide *= torch.exp(0.5 * _normal(g, (case["n"], 1)))
        s["x"] = wide.to(_TYPES[case["dtype"]])[:, : case["dim"]]
        if case["rotate"]:
            r = np.random.default_rng(seed)
            signs, perm = 1 - 2 * r.integers(0, 2, 256), r.permutation(128)
            s["tables"] = _tables(case["dim"], signs, perm)
            if own:  # the codec plan that holds the rotation
                import paper_2608_30384_amd as R

                s["plan"] = R.Plan(case["dim"], 4, passes=2, signs=signs, perm=perm)
        return s
    if kind == "logprob":
        s["scores"] = (3.0 * _normal(g, (case["m"], case["n"]))).to(_TYPES[case["dtype"]])
        if case["masked"]:
            s["scores"][torch.rand((case["m"], case["n"]), generator=g, device="cuda") < case["masked"]] = -math.inf
        s["scale"] = 1.25
        s["target"] = torch.randint(-1, case["n"], (case["m"],), generator=g, device="cuda")
        s["grads"] = (_normal(g, (case["m"],)), 0.1 * _normal(g, (case["m"],)))
        return s
    s["b"] = _rows(g, seed, case["n"], case["dim"])
    if kind == "matmul":
        s["a"] = _rows(g, seed + 1, case["m"], case["dim"])
    elif kind == "score":
        s["x"] = _normal(g, (case["m"], case["dim"]), case["dtype"])
    else:
        # the gradient that a softmax over the scores sends back: mostly small
        s["dout"] = (0.01 * _normal(g, (case["m"], case["n"])) * torch.exp(_normal(g, (case["m"], case["n"])))).to(_TYPES[case["dtype"]])
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


def _plain_quantize(s):
    x = s["x"].float()
    if s["rotate"]:
        t = s["tables"]
        x = _hadamard((_hadamard(x * t["s1"], t["block"]))[:, t["source"]] * t["s2"], t["block"])
    n, dim = x.shape
    y = torch.nn.functional.pad(x, (0, -dim % 32)).view(n, -1, 32)
    top = y.abs().amax(-1, keepdim=True)
    e = (((top.view(torch.int32) >> 23) & 255) - 2).clamp_(min=0)
    v = (y * ((254 - e) << 23).view(torch.float32)).abs()
    c = (v > 0.25).to(torch.int32) + (v >= 0.75) + (v > 1.25) + (v >= 1.75) + (v > 2.5) + (v >= 3.5) + (v > 5.0)
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=x.device)[c]
    v = torch.where(y < 0, -v, v) * _power(e)
    v = torch.where(torch.isfinite(top), v, math.nan)
    return v.view(n, -1)[:, :dim].to(s["x"].dtype)


def _values(rows, dim):
    """float32 values of MX4 rows."""
    codes, scales = rows
    n = codes.shape[0]
    c = torch.stack((codes & 15, codes >> 4), -1).view(n, -1, 32).to(torch.int32)
    # E2M1's exponent and mantissa at the low end of float32's, then 2^126 for
    # the difference of the exponents' biases: exact, 0.5 (a subnormal) too
    v = (((c & 7) << 22) | ((c & 8) << 28)).view(torch.float32) * 2.0 ** 126
    return (v * _power(scales)[..., None]).view(n, -1)[:, :dim]


def _plain_logprob(s):
    x, n, t = s["scores"].float(), s["n"], s["target"]
    z = x * s["scale"]
    dead = z == -math.inf
    top = z.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    lse = (z - top).exp().sum(1, keepdim=True).log() + top
    logs = torch.where(dead, -math.inf, z - lse)
    p = logs.exp()
    entropy = -torch.where(dead, 0.0, p * logs).sum(1, keepdim=True)
    one = t.clamp(min=0)[:, None]
    logprob = torch.where(t < 0, 0.0, logs.gather(1, one)[:, 0])
    # the k largest, the lower index first among equals
    bits = (x + 0.0).view(torch.int32).to(torch.int64)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 32) + ((1 << 31) - 1 - torch.arange(n, device=x.device))
    ids = key.topk(s["k"], 1).indices
    best = logs.gather(1, ids)
    out = dict(logprob=logprob, lse=lse[:, 0], entropy=entropy[:, 0], top=best,
               ids=torch.where(best == -math.inf, -1, ids).to(torch.int32))
    if s["grad"]:
        dl, dh = (v[:, None] for v in s["grads"])
        hit = (torch.arange(n, device=x.device) == t[:, None]).float()
        d = torch.where(t[:, None] < 0, 0.0, dl) * (hit - p) - dh * p * (logs + entropy)
        out["dscores"] = torch.where(dead, 0.0, d * s["scale"]).to(s["scores"].dtype)
    return out


def _plain(s):
    kind = s["kind"]
    if kind == "quantize":
        return _plain_quantize(s)
    if kind == "logprob":
        return _plain_logprob(s)
    b = _values(s["b"], s["dim"])
    if kind == "matmul":
        return torch.mm(_values(s["a"], s["dim"]), b.t()).to(_TYPES[s["out"]])
    if kind == "score":
        return torch.mm(s["x"].float(), b.t()).to(_TYPES[s["out"]])
    return torch.mm(s["dout"].float(), b).to(s["dout"].dtype)


# ------------------------------------------------------------------ one pass
def run(s):
    if not own:
        return _plain(s)
    import paper_2608_30384_amd as R

    kind = s["kind"]
    if kind == "quantize":
        return R.rslm_mx4_dequantize(R.rslm_mx4_quantize(s["x"], plan=s.get("plan")), dtype=s["x"].dtype)
    if kind == "logprob":
        r = R.rslm_logprob(s["scores"], s["target"], s["k"], scale=s["scale"])
        out = dict(logprob=r.logprob, lse=r.lse, entropy=r.entropy, top=r.top_logprob, ids=r.top_ids)
        if s["grad"]:
            out["dscores"] = R.rslm_logprob_backward(s["scores"], s["target"], r, s["grads"][0], s["grads"][1], scale=s["scale"])
        return out
    b = R.Mx4Rows(*s["b"], s["dim"])
    if kind == "matmul":
        return R.rslm_mx4_matmul(R.Mx4Rows(*s["a"], s["dim"]), b, dtype=_TYPES[s["out"]])
    if kind == "score":
        return R.rslm_mx4_score(s["x"], b, dtype=_TYPES[s["out"]])
    return R.rslm_mx4_score_backward(s["dout"], b)


# ------------------------------------------------------------------ 64 bits
def _values64(rows, dim):
    level = np.array([0, 1, 2, 3, 4, 6, 8, 12], dtype=np.float64) / 2
    level = np.concatenate([level, -level])
    byte = np.arange(256)
    pair = torch.from_numpy(np.stack([level[byte & 15], level[byte >> 4]], 1)).cuda()
    power = torch.from_numpy(np.ldexp(1.0, byte - 127)).cuda()

    def some(codes, scales):
        v = pair[codes.long()].reshape(codes.shape[0], -1, 32) * power[scales.long()].unsqueeze(-1)
        return v.reshape(codes.shape[0], -1)[:, :dim]

    return torch.cat([some(c, s) for c, s in zip(rows[0].split(4096), rows[1].split(4096))])


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
        level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
        between = (level[1:] + level[:-1]) / 2
        out = torch.empty_like(x)
        for o in range(0, case["dim"], 32):
            y = x[:, o:o + 32]
            e = (torch.frexp(y.abs().amax(1, keepdim=True)).exponent - 3).clamp(min=-127)
            unit = ((e.long() + 1023) << 52).view(torch.float64)  # 2^e
            v = y.abs() / unit
            lower, upper = torch.bucketize(v, between), torch.bucketize(v, between, right=True)
            out[:, o:o + 32] = torch.copysign(level[torch.where(lower % 2 == 0, lower, upper)], y) * unit
        return out
    if kind == "logprob":
        z = s["scores"].double() * s["scale"]
        live = z > -math.inf
        lse = torch.logsumexp(z, 1)
        logs = torch.log_softmax(z, 1).masked_fill(~live, -math.inf)
        p = logs.exp()
        plogs = (p * logs).masked_fill(~live, 0.0)
        entropy = -plogs.sum(1)
        rows = torch.arange(case["m"], device="cuda")
        on = s["target"] >= 0
        out = dict(logprob=torch.where(on, logs[rows, s["target"].clamp(min=0)], 0.0), lse=lse, entropy=entropy,
                   top=z.topk(case["k"], 1).values - lse[:, None], ids=None)
        if case["grad"]:
            dl = s["grads"][0].double() * on
            dh = s["grads"][1].double()
            d = -p * dl[:, None] - dh[:, None] * (plogs + p * entropy[:, None])
            d[rows[on], s["target"][on]] += dl[on]
            out["dscores"] = (d * s["scale"]).masked_fill(~live, 0.0)
        return out
    b = _values64(s["b"], case["dim"])
    if kind == "matmul":
        return torch.mm(_values64(s["a"], case["dim"]), b.t())
    if kind == "score":
        return torch.mm(s["x"].double(), b.t())
    return torch.mm(s["dout"].double(), b)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n, dim = case["n"], case["dim"]
        # rows read, codes and scales written and read again, values written
        return dict(bytes=n * (2 * dim * _BYTES[case["dtype"]] + 2 * (dim / 2 + dim / 32)),
                    flops=n * dim * (2 + (2 * 8 if case["rotate"] else 0)))
    m, n = case["m"], case["n"]
    if kind == "logprob":
        e = _BYTES[case["dtype"]]
        passes = 3 if case["grad"] else 1  # scores read; read again and their gradient written
        return dict(bytes=passes * m * n * e + m * (8 * case["k"] + 28), flops=(12 if case["grad"] else 6) * m * n)
    rows = n * (case["dim"] / 2 + case["dim"] / 32)
    flops = 2 * m * n * case["dim"]
    if kind == "matmul":
        return dict(bytes=rows * (1 + m / n) + m * n * _BYTES[case["out"]], flops=flops)
    if kind == "score":
        return dict(bytes=rows + m * case["dim"] * _BYTES[case["dtype"]] + m * n * _BYTES[case["out"]], flops=flops)
    return dict(bytes=rows + m * (n + case["dim"]) * _BYTES[case["dtype"]], flops=flops)
