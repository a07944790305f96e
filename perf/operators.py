"""What the layer operators are measured on: group norm with an activation, dropout, and 8-bit matrix products.

Every case names its operator in ``op``:

``norm``         y = act(gamma * (x - mean) * rstd + beta) over the channel groups of x [n, spatial, channels]
``norm_grad``    the gradients of that: dx, dgamma, dbeta
``dropout``      y = residual + keep * x / (1 - p), the mask drawn from a counter and never stored
``quantize``     x as e4m3 values with a scale for each block of 128 (rows, or 128 x 128 tiles), with its transpose if asked
``matmul``       act(a b^T + bias) of two such operands
``linear``       quantize and matmul: an activation against kept 8-bit weights
``linear_grad``  the two products of its backward pass: dx = dy w, dw = dy^T x

With ``own`` false ``run`` computes them in elementary torch operations in 32 bits; with ``own`` true it calls the library.
"""

import math

import numpy as np
import torch

own = False

BLOCK = 128          # contraction indices that share a scale
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}
STREAM_DROPOUT = 7   # stream of the counter-based generator that dropout draws from
GAMMA, MIX1, MIX2 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB


# ------------------------------------------------------------------ cases
def listed():
    return [
        # a batch of 64 pairs through a 500-wide layer: the smallest training step, latency alone
        dict(name="norm_rows_small", op="norm", n=128, spatial=1, channels=500, groups=10, act="relu", dtype="bf16", pad=4),
        # feature maps of 64 x 64, channels last, larger than L2
        dict(name="norm_images", op="norm", n=32, spatial=4096, channels=512, groups=32, act="silu", dtype="bf16", pad=0),
        # the backward pass of an exact-precision 2000-wide layer, 1024 pairs, groups of an odd width
        dict(name="norm_grad_rows", op="norm_grad", n=2048, spatial=1, channels=2000, groups=16, act="relu", dtype="fp32", pad=0),
        # the backward pass on feature maps of 56 x 56
        dict(name="norm_grad_images", op="norm_grad", n=32, spatial=3136, channels=320, groups=32, act="silu", dtype="bf16", pad=0),
        # one small exact-precision batch
        dict(name="dropout_small", op="dropout", rows=128, cols=500, p=0.5, residual=False, dtype="fp32"),
        # a residual stream of a large net, far larger than L2
        dict(name="dropout_residual", op="dropout", rows=16384, cols=8192, p=0.1, residual=True, dtype="bf16"),
        # the fp32 master weights of a 784-2000 layer, both ways round, as after an optimizer step
        dict(name="quantize_weights", op="quantize", rows=2000, cols=784, tile=True, both=True, dtype="fp32"),
        # an activation of the large net, both ways round, as a training step needs it
        dict(name="quantize_train", op="quantize", rows=4096, cols=8192, tile=False, both=True, dtype="bf16"),
        # one sample through a 2000-2000 layer: serving, the weights read once
        dict(name="matmul_single", op="matmul", m=1, n=2000, k=2000, tile=True, bias=True, relu=True, out="bf16"),
        # a ragged batch, no size a multiple of anything
        dict(name="matmul_ragged", op="matmul", m=333, n=1999, k=1337, tile=True, bias=True, relu=False, out="fp32"),
        # the 8192-8192 layer of the large net at 4096 rows
        dict(name="linear_large", op="linear", m=4096, n=8192, k=8192, relu=False, bias=True, dtype="bf16", out="bf16"),
        # the backward pass of a 2000-2000 layer, 1024 pairs
        dict(name="linear_grad", op="linear_grad", m=2048, n=2000, k=2000, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "dropout", "quantize", "matmul", "matmul", "linear", "linear_grad"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op in ("norm", "norm_grad"):
        spatial = 1 if rng.random() < 0.4 else _log(rng, 2, 16384)
        groups = rng.choice([1, 2, 4, 8, 16, 32])
        width = _log(rng, 2, 256)
        if rng.random() < 0.5:
            width = -(-width // 8) * 8
        most = max(1, (1 << 25) // (spatial * groups * width))
        return dict(op=op, n=_log(rng, 1, min(most, 8192)), spatial=spatial, channels=groups * width, groups=groups,
                    act=rng.choice(["none", "relu", "silu"]), dtype=dtype, pad=rng.choice([0, 0, 0, 8, 3]))
    if op == "dropout":
        cols = _log(rng, 1, 16384)
        return dict(op=op, rows=_log(rng, 1, min(16384, (1 << 27) // cols)), cols=cols, p=rng.choice([0.05, 0.1, 0.3, 0.5]),
                    residual=rng.random() < 0.5, dtype=dtype)
    if op == "quantize":
        return dict(op=op, rows=_log(rng, 1, 8192), cols=_log(rng, 1, 8192), tile=rng.random() < 0.4, both=rng.random() < 0.5, dtype=dtype)
    m, n, k = _log(rng, 1, 4096), _log(rng, 16, 8192), _log(rng, 16, 8192)
    if op == "matmul":
        return dict(op=op, m=m, n=n, k=k, tile=rng.random() < 0.7, bias=rng.random() < 0.5, relu=rng.random() < 0.5,
                    out=rng.choice(["bf16", "fp32"]))
    if op == "linear":
        return dict(op=op, m=m, n=n, k=k, relu=rng.random() < 0.5, bias=rng.random() < 0.5, dtype=dtype, out=rng.choice(["bf16", "fp32"]))
    return dict(op=op, m=m, n=_log(rng, 16, 4096), k=_log(rng, 16, 4096), dtype=dtype)


def _blocks(size):
    return -(-size // BLOCK)


def _padded(size):
    return -(-size // 16) * 16


def work(case):
    c, op = case, case["op"]
    if op in ("norm", "norm_grad"):
        count, b = c["n"] * c["spatial"] * c["channels"], BYTES[c["dtype"]]
        small = 2 * c["n"] * c["groups"] * 4 + 2 * c["channels"] * 4  # mean and rstd, gamma and beta
        if op == "norm":
            return {"bytes": 2 * count * b + small, "flops": 8 * count}
        return {"bytes": 3 * count * b + small + 2 * c["channels"] * 4, "flops": 16 * count}
    if op == "dropout":
        count = c["rows"] * c["cols"]
        return {"bytes": count * BYTES[c["dtype"]] * (3 if c["residual"] else 2), "flops": 2 * count}
    if op == "quantize":
        r, k = c["rows"], c["cols"]
        scales = _blocks(r) * _blocks(k) if c["tile"] else r * _blocks(k)
        moved = r * k * BYTES[c["dtype"]] + r * k + 4 * scales
        if c["both"]:
            moved += r * k + 4 * (_blocks(r) * _blocks(k) if c["tile"] else k * _blocks(r))
        return {"bytes": moved, "flops": 2 * r * k}
    m, n, k = c["m"], c["n"], c["k"]
    if op == "linear_grad":
        scales = 4 * (_blocks(n) * _blocks(k) + _blocks(m) * k)
        return {"bytes": m * n * BYTES[c["dtype"]] + n * k + m * k + scales + m * k * BYTES["bf16"] + n * k * 4, "flops": 4 * m * n * k}
    moved = n * k + m * n * BYTES[c["out"]] + (4 * n if c["bias"] else 0)
    if op == "linear":
        return {"bytes": moved + m * k * BYTES[c["dtype"]] + 4 * _blocks(n) * _blocks(k), "flops": 2 * m * n * k}
    scales = 4 * (m * _blocks(k) + (_blocks(n) if c["tile"] else n) * _blocks(k))
    return {"bytes": moved + m * k + scales, "flops": 2 * m * n * k}


# ----------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _activity(gen, rows, cols):
    """A layer's activity: rectified, rows of differing size."""
    return torch.relu(_randn(gen, rows, cols)) * torch.exp(0.5 * _randn(gen, rows, 1))


def prepare(case, seed):
    c, op = case, case["op"]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": dict(c)}
    if op in ("norm", "norm_grad"):
        n, spatial, ch, dt = c["n"], c["spatial"], c["channels"], DTYPES[c["dtype"]]
        shape = (n, ch) if spatial == 1 else (n, spatial, ch)
        buf = torch.zeros(*shape[:-1], ch + c["pad"], device="cuda", dtype=dt)
        buf[..., :ch] = 2.0 * _randn(gen, *shape) + _randn(gen, ch)
        s["x"] = buf[..., :ch]
        s["gamma"], s["beta"] = 1.0 + 0.2 * _randn(gen, ch), 0.2 * _randn(gen, ch)
        if op == "norm_grad":  # what the forward pass kept
            s["dy"] = _randn(gen, *shape).to(dt)
            g = s["x"].float().reshape(n, spatial, c["groups"], -1)
            mean = g.mean((1, 3), keepdim=True)
            s["mean"] = mean.view(n, -1).contiguous()
            s["rstd"] = torch.rsqrt((g - mean).square().mean((1, 3)) + 1e-5)
        return s
    if op == "dropout":
        s["x"] = _randn(gen, c["rows"], c["cols"]).to(DTYPES[c["dtype"]])
        s["residual"] = _randn(gen, c["rows"], c["cols"]).to(DTYPES[c["dtype"]]) if c["residual"] else None
        s["seed"], s["offset"] = int(seed) & ((1 << 56) - 1), 1000 + 7 * (int(seed) & 0xFFFF)
        return s
    if op == "quantize":
        x = 0.03 * _randn(gen, c["rows"], c["cols"]) if c["tile"] else _activity(gen, c["rows"], c["cols"])
        s["x"] = x.to(DTYPES[c["dtype"]])
        return s
    m, n, k = c["m"], c["n"], c["k"]
    w = _randn(gen, n, k) / math.sqrt(k)
    if op == "linear_grad":
        s["dy"] = (_randn(gen, m, n) * torch.exp(0.5 * _randn(gen, m, 1)) / m).to(DTYPES[c["dtype"]])
        s["wt"], s["wt_scale"] = _quantize(w.t(), True)
        s["xt"], s["xt_scale"] = _quantize(_activity(gen, m, k).t(), False)
        return s
    s["w"], s["w_scale"] = _quantize(w, c.get("tile", True))
    s["bias"] = 0.1 * _randn(gen, n) if c["bias"] else None
    if op == "linear":
        s["x"] = _activity(gen, m, k).to(DTYPES[c["dtype"]])
    else:
        s["a"], s["a_scale"] = _quantize(_activity(gen, m, k), False)
    return s


# ------------------------------------------------------------ plain forms
def _act(u, act):
    return torch.relu(u) if act == "relu" else u * torch.sigmoid(u) if act == "silu" else u


def _act_slope(u, act):
    if act == "relu":
        return (u > 0).float()
    if act == "silu":
        p = torch.sigmoid(u)
        return p * (1 + u * (1 - p))
    return torch.ones_like(u)


def _norm(s):
    c, x = s["case"], s["x"]
    n, spatial, groups, ch = c["n"], c["spatial"], c["groups"], c["channels"]
    g = x.float().reshape(n, spatial, groups, ch // groups)
    mean = g.mean((1, 3), keepdim=True)
    d = g - mean
    rstd = torch.rsqrt(d.square().mean((1, 3), keepdim=True) + 1e-5)
    u = (d * rstd).view(n, spatial, ch) * s["gamma"] + s["beta"]
    return _act(u, c["act"]).view(x.shape).to(x.dtype), mean.view(n, groups), rstd.view(n, groups)


def _norm_grad(s):
    c, x = s["case"], s["x"]
    n, spatial, groups, ch = c["n"], c["spatial"], c["groups"], c["channels"]
    mean, rstd = s["mean"].view(n, 1, groups, 1), s["rstd"].view(n, 1, groups, 1)
    h = ((x.float().reshape(n, spatial, groups, -1) - mean) * rstd).view(n, spatial, ch)
    u = h * s["gamma"] + s["beta"]
    du = s["dy"].float().view(n, spatial, ch) * _act_slope(u, c["act"])
    dgamma, dbeta = (du * h).sum((0, 1)), du.sum((0, 1))
    dh = (du * s["gamma"]).view(n, spatial, groups, -1)
    h = h.view(n, spatial, groups, -1)
    dx = rstd * (dh - dh.mean((1, 3), keepdim=True) - h * (dh * h).mean((1, 3), keepdim=True))
    return dx.view(x.shape).to(x.dtype), dgamma, dbeta


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _shift(z, by):
    """Logical right shift of 64-bit words."""
    return (z >> by) & ((1 << (64 - by)) - 1)


def _mix(z):
    z = (z ^ _shift(z, 30)) * _signed(MIX1)
    z = (z ^ _shift(z, 27)) * _signed(MIX2)
    return z ^ _shift(z, 31)


def _keep(seed, offset, rows, cols, p):
    """The mask: 16 bits of word offset + r * ceil(cols / 4) + j / 4 for element (r, j)."""
    state = _mix(torch.tensor([_signed((seed << 8) | STREAM_DROPOUT)], device="cuda"))
    words = -(-cols // 4)
    i = torch.arange(rows * words, device="cuda") + _signed(offset + 1)
    z = _mix(state + i * _signed(GAMMA))
    bits = (z[:, None] >> torch.arange(0, 64, 16, device="cuda")) & 0xFFFF
    return bits.view(rows, words * 4)[:, :cols] >= round(p * 65536)


def _dropout(s):
    c, x = s["case"], s["x"]
    keep = _keep(s["seed"], s["offset"], c["rows"], c["cols"], c["p"])
    y = torch.where(keep, x.float() * (65536.0 / (65536 - round(c["p"] * 65536))), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


def _quantize(x, tile):
    """x [rows, k] as e4m3 [rows, k padded to 16] and scales [ceil(k / 128), rows or ceil(rows / 128)]."""
    rows, k = x.shape
    kb, rb = _blocks(k), _blocks(rows)
    full = x.new_zeros(rb * BLOCK if tile else rows, kb * BLOCK, dtype=torch.float32)
    full[:rows, :k] = x.float()
    v = full.view(rb, BLOCK, kb, BLOCK) if tile else full.view(rows, 1, kb, BLOCK)
    amax = v.abs().amax((1, 3), keepdim=True)
    scale = torch.clamp(amax / torch.full_like(amax, E4M3_MAX), min=SCALE_MIN)  # a quotient of tensors: rounded once
    q = torch.clamp(v * (1.0 / scale), -E4M3_MAX, E4M3_MAX).view(-1, kb * BLOCK)
    return q[:rows, :_padded(k)].to(torch.float8_e4m3fn).contiguous(), scale.view(-1, kb).t().contiguous()


def _values(q, scale, rows, k, tile):
    """The matrix [rows, k] that (q, scale) stand for."""
    per = scale.t().repeat_interleave(BLOCK, 1)[:, :k]
    if tile:
        per = per.repeat_interleave(BLOCK, 0)[:rows]
    return q[:, :k].float() * per


def _matmul(s, a, a_scale, w, w_scale, tile):
    c = s["case"]
    y = _values(a, a_scale, c["m"], c["k"], False) @ _values(w, w_scale, c["n"], c["k"], tile).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    if c["relu"]:
        y = torch.relu(y)
    return y.to(DTYPES[c["out"]])


def _linear_grad(s):
    c = s["case"]
    m, n, k = c["m"], c["n"], c["k"]
    dy, dy_scale = _quantize(s["dy"], False)
    dyt, dyt_scale = _quantize(s["dy"].t(), False)
    dx = _values(dy, dy_scale, m, n, False) @ _values(s["wt"], s["wt_scale"], k, n, True).t()
    dw = _values(dyt, dyt_scale, n, m, False) @ _values(s["xt"], s["xt_scale"], k, m, False).t()
    return dx.to(torch.bfloat16), dw


def _run_plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        return _norm(s)
    if op == "norm_grad":
        return _norm_grad(s)
    if op == "dropout":
        return _dropout(s)
    if op == "quantize":
        one = _quantize(s["x"], c["tile"])
        return one + _quantize(s["x"].t(), c["tile"]) if c["both"] else one
    if op == "matmul":
        return _matmul(s, s["a"], s["a_scale"], s["w"], s["w_scale"], c["tile"])
    if op == "linear":
        return _matmul(s, *_quantize(s["x"], False), s["w"], s["w_scale"], True)
    return _linear_grad(s)


# ------------------------------------------------------- the library's calls
def _run_own(s):
    from paper_2404_08573_gb300 import ff

    c, op = s["case"], s["case"]["op"]
    if op == "norm":
        return ff.group_norm_act(s["x"], s["gamma"], s["beta"], c["groups"], act=c["act"], eps=1e-5)
    if op == "norm_grad":
        return ff.group_norm_act_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["beta"], c["groups"], act=c["act"])
    if op == "dropout":
        return ff.dropout(s["x"], c["p"], s["seed"], s["offset"], residual=s["residual"])
    if op == "quantize":
        if c["both"]:
            a, t = ff.fp8_quantize_both(s["x"], tile=c["tile"])
            return a.q, a.scale, t.q, t.scale
        a = ff.fp8_quantize(s["x"], tile=c["tile"])
        return a.q, a.scale
    if op == "linear_grad":
        dy, dyt = ff.fp8_quantize_both(s["dy"])
        dx = ff.fp8_matmul(dy, ff.Fp8Matrix(s["wt"], s["wt_scale"], c["k"], c["n"], tile=True))
        dw = ff.fp8_matmul(dyt, ff.Fp8Matrix(s["xt"], s["xt_scale"], c["k"], c["m"]), out_dtype=torch.float32)
        return dx, dw
    if op == "linear":
        a, tile = ff.fp8_quantize(s["x"]), True
    else:
        a, tile = ff.Fp8Matrix(s["a"], s["a_scale"], c["m"], c["k"]), c["tile"]
    w = ff.Fp8Matrix(s["w"], s["w_scale"], c["n"], c["k"], tile=tile)
    return ff.fp8_matmul(a, w, bias=s["bias"], relu=c["relu"], out_dtype=DTYPES[c["out"]])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------- the definitions in 64 bits
def _e4m3_exact(v):
    """Nearest e4m3 value, ties to even: 3 fraction bits, least exponent -6."""
    e = torch.clamp(torch.frexp(v)[1] - 1, min=-6)
    step = ((e.long() - 3 + 1023) << 52).view(torch.float64)  # 2 ** (e - 3), by its bits
    return torch.clamp(torch.round(v / step) * step, -E4M3_MAX, E4M3_MAX)


def _quantize_exact(x, tile):
    """Values, padded values and scales. A scale is a 32-bit number by definition, and so are its reciprocal and their product."""
    rows, k = x.shape
    x = x.double()
    rb, kb = _blocks(rows), _blocks(k)
    row_of = torch.arange(rows, device="cuda") // (BLOCK if tile else 1)
    col_of = torch.arange(k, device="cuda") // BLOCK
    index = (row_of[:, None] * kb + col_of).view(-1)
    amax = torch.zeros((rb if tile else rows) * kb, device="cuda", dtype=torch.float64)
    amax.scatter_reduce_(0, index, x.abs().reshape(-1), "amax")
    scale = (amax / torch.full_like(amax, E4M3_MAX)).float().clamp(min=SCALE_MIN)
    inverse = (1.0 / scale.double()).float()
    q = _e4m3_exact((x * inverse.double()[index].view(rows, k)).float().double())
    padded = torch.nn.functional.pad(q, (0, _padded(k) - k))
    return q * scale.double()[index].view(rows, k), padded, scale.double().view(-1, kb).t()


def _values_exact(q, scale, rows, k, tile):
    row_of = torch.arange(rows, device="cuda") // (BLOCK if tile else 1)
    return q.float().double()[:, :k] * scale.double()[torch.arange(k, device="cuda") // BLOCK][:, row_of].t()


def _norm_exact(s):
    c, x = s["case"], s["x"]
    x64 = x.double().reshape(c["n"], c["spatial"], c["groups"], -1).transpose(1, 2).flatten(2)  # [n, group, all of it]
    var, mean = torch.var_mean(x64, 2, unbiased=False)
    rstd = (var + 1e-5) ** -0.5
    u = ((x64 - mean[..., None]) * rstd[..., None]).view(c["n"], c["groups"], c["spatial"], -1).transpose(1, 2).flatten(2)
    u = u * s["gamma"].double() + s["beta"].double()
    y = u.clamp(min=0) if c["act"] == "relu" else u / (1 + torch.exp(-u)) if c["act"] == "silu" else u
    return y.view(x.shape), mean, rstd


def _norm_grad_exact(s):
    """By the chain rule, one channel group at a time as a vector of its own."""
    c, x = s["case"], s["x"]
    n, spatial, groups, ch = c["n"], c["spatial"], c["groups"], c["channels"]
    per = ch // groups

    def grouped(t):
        return t.double().reshape(n, spatial, groups, per).transpose(1, 2)  # [n, group, spatial, per]

    rstd = s["rstd"].double()[:, :, None, None]
    gamma, beta = s["gamma"].double().view(groups, 1, per), s["beta"].double().view(groups, 1, per)
    h = (grouped(x) - s["mean"].double()[:, :, None, None]) * rstd
    u = gamma * h + beta
    if c["act"] == "relu":
        slope = torch.where(u > 0, 1.0, 0.0).double()
    elif c["act"] == "silu":
        e = torch.exp(-u)
        slope = (1 + e + u * e) / (1 + e) ** 2
    else:
        slope = torch.ones_like(u)
    du = grouped(s["dy"]) * slope
    dgamma, dbeta = torch.einsum("ngsc,ngsc->gc", du, h).reshape(-1), torch.einsum("ngsc->gc", du).reshape(-1)
    dh = du * gamma
    count = spatial * per
    along = torch.einsum("ngsc,ngsc->ng", dh, h)[:, :, None, None] / count
    across = torch.einsum("ngsc->ng", dh)[:, :, None, None] / count
    dx = rstd * (dh - across - h * along)
    return dx.transpose(1, 2).reshape(x.shape), dgamma, dbeta


def _mix_exact(z):
    z = (z ^ (z >> np.uint64(30))) * np.uint64(MIX1)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(MIX2)
    return z ^ (z >> np.uint64(31))


def _dropout_exact(s):
    c, x = s["case"], s["x"]
    rows, cols = c["rows"], c["cols"]
    words = -(-cols // 4)
    state = _mix_exact(np.array([(s["seed"] << 8) | STREAM_DROPOUT], dtype=np.uint64))
    i = np.arange(1, rows * words + 1, dtype=np.uint64) + np.uint64(s["offset"])
    bits = _mix_exact(state + i * np.uint64(GAMMA)).astype("<u8").view("<u2").reshape(rows, words * 4)[:, :cols]
    drop = round(c["p"] * 65536)
    keep = torch.from_numpy(bits >= drop).cuda()
    y = torch.where(keep, x.double() * 65536 / (65536 - drop), 0.0)
    return y if s["residual"] is None else y + s["residual"].double()


def exact(case, seed):
    s = prepare(case, seed)
    c, op = s["case"], case["op"]
    if op == "norm":
        return _norm_exact(s)
    if op == "norm_grad":
        return _norm_grad_exact(s)
    if op == "dropout":
        return _dropout_exact(s)
    if op == "quantize":
        one = _quantize_exact(s["x"], c["tile"])[1:]
        return one + _quantize_exact(s["x"].t(), c["tile"])[1:] if c["both"] else one
    m, n, k = c["m"], c["n"], c["k"]
    if op == "linear_grad":
        dx = _quantize_exact(s["dy"], False)[0] @ _values_exact(s["wt"], s["wt_scale"], k, n, True).t()
        dw = _quantize_exact(s["dy"].t(), False)[0] @ _values_exact(s["xt"], s["xt_scale"], k, m, False).t()
        return dx, dw
    a = _quantize_exact(s["x"], False)[0] if op == "linear" else _values_exact(s["a"], s["a_scale"], m, k, False)
    y = a @ _values_exact(s["w"], s["w_scale"], n, k, c.get("tile", True)).t()
    if s["bias"] is not None:
        y = y + s["bias"].double()
    return torch.where(y > 0, y, 0.0) if c["relu"] else y
