"""What the operators of a deep head are measured on: RMS norm, label log-probabilities, gradient clipping, 4-bit products.

Every case names its operator in ``op``:

``rms``            h = x + residual, y = gamma * h / sqrt(mean h^2 + eps), y in the input's type or as e4m3 with a scale per 128
``rms_grad``       its gradients: dx (with what the residual stream hands back added) and dgamma
``logprobs``       per row of logits: the label's log-probability, the entropy, the ``top`` likeliest classes, max and log sum
``logprobs_grad``  the gradient of the label's log-probability and of the entropy
``clip``           the 2-norm over many gradients, and copies of them scaled to at most ``max_norm``
``fp4_quantize``   x as e2m1 values with a power-of-two scale per 32 (and its transpose), and the values these stand for
``fp4_matmul``     act(a b^T + bias) of two such operands
``fp4_linear``     quantize and matmul: an activation against kept 4-bit weights

With ``own`` false ``run`` computes them in elementary torch operations; with ``own`` true it calls the library.
"""

import math

import torch

own = False

EPS = 1e-5
E4M3_MAX, E4M3_BLOCK, SCALE_MIN = 448.0, 128, 2.0 ** -126
FP4_BLOCK = 32       # contraction indices that share a power-of-two scale
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}


# ------------------------------------------------------------------ cases
def listed():
    return [
        # serving one sample through a 2000-wide block in 8 bits: latency alone
        dict(name="rms_single", op="rms", rows=1, cols=2000, residual=True, fp8=True, dtype="bf16", pad=0),
        # the residual stream of a large net, far larger than L2, on its way into an 8-bit product
        dict(name="rms_large", op="rms", rows=16384, cols=8192, residual=True, fp8=True, dtype="bf16", pad=0),
        # the backward pass of a large net's training step, the residual stream's gradient joined in
        dict(name="rms_grad", op="rms_grad", rows=4096, cols=8192, dh=True, dtype="bf16", pad=0),
        # serving one answer out of many classes, with alternatives
        dict(name="logprobs_single", op="logprobs", rows=1, classes=131072, top=8, masked=0.0, dtype="bf16"),
        # scoring a batch against labels, an odd number of classes, a tenth of them barred
        dict(name="logprobs_score", op="logprobs", rows=2048, classes=49999, top=4, masked=0.1, dtype="fp32"),
        # the loss gradient of a training step with an entropy bonus
        dict(name="logprobs_grad", op="logprobs_grad", rows=4096, classes=65536, entropy=True, masked=0.0, dtype="bf16"),
        # the gradients of a 10-class head on 2000 features with its norm: latency alone
        dict(name="clip_head", op="clip", tensors=4, total=24010, matrix=0.83, dtype="fp32"),
        # the gradients of a net of four 8192 x 8192 layers
        dict(name="clip_large", op="clip", tensors=12, total=4 * 8192 * 8194, matrix=0.24, dtype="fp32"),
        # the fp32 master weights of a 784-2000 layer, both ways round, as after an optimizer step
        dict(name="fp4_quantize_weights", op="fp4_quantize", rows=2000, cols=784, both=True, dtype="fp32"),
        # an activation of the large net, both ways round, as a training step needs it
        dict(name="fp4_quantize_train", op="fp4_quantize", rows=4096, cols=8192, both=True, dtype="bf16"),
        # one sample through an 8192-8192 layer: serving, the weights read once
        dict(name="fp4_single", op="fp4_matmul", m=1, n=8192, k=8192, bias=True, relu=True, out="bf16"),
        # the 8192-8192 layer of the large net at 4096 rows
        dict(name="fp4_linear_large", op="fp4_linear", m=4096, n=8192, k=8192, bias=True, relu=False, dtype="bf16", out="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rms", "rms", "rms_grad", "logprobs", "logprobs", "logprobs_grad", "clip", "fp4_quantize", "fp4_matmul", "fp4_matmul", "fp4_linear"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op in ("rms", "rms_grad"):
        cols = _log(rng, 16, 32768)
        if rng.random() < 0.5:
            cols = -(-cols // 8) * 8
        rows, pad = _log(rng, 1, min(16384, (1 << 26) // cols)), rng.choice([0, 0, 0, 8, 3])
        if op == "rms":
            return dict(op=op, rows=rows, cols=cols, residual=rng.random() < 0.6, fp8=rng.random() < 0.5, dtype=dtype, pad=pad)
        return dict(op=op, rows=rows, cols=cols, dh=rng.random() < 0.6, dtype=dtype, pad=pad)
    if op in ("logprobs", "logprobs_grad"):
        classes = _log(rng, 2, 200000)
        if rng.random() < 0.5:
            classes = -(-classes // 8) * 8
        rows, masked = _log(rng, 1, min(16384, max(1, (1 << 27) // classes))), rng.choice([0.0, 0.0, 0.2])
        if op == "logprobs":
            return dict(op=op, rows=rows, classes=classes, top=min(classes, rng.choice([0, 1, 5, 8, 20, 32])), masked=masked, dtype=dtype)
        return dict(op=op, rows=rows, classes=classes, entropy=rng.random() < 0.5, masked=masked, dtype=dtype)
    if op == "clip":
        tensors = _log(rng, 1, 60)
        return dict(op=op, tensors=tensors, total=_log(rng, 8 * tensors, 1 << 27), matrix=rng.uniform(0.05, 0.9), dtype=dtype)
    if op == "fp4_quantize":
        return dict(op=op, rows=_log(rng, 1, 8192), cols=_log(rng, 1, 8192), both=rng.random() < 0.5, dtype=dtype)
    m, n, k = _log(rng, 1, 4096), _log(rng, 16, 8192), _log(rng, 16, 8192)
    if op == "fp4_matmul":
        return dict(op=op, m=m, n=n, k=k, bias=rng.random() < 0.5, relu=rng.random() < 0.5, out=rng.choice(["bf16", "fp32"]))
    return dict(op=op, m=m, n=n, k=k, bias=rng.random() < 0.5, relu=rng.random() < 0.5, dtype=dtype, out=rng.choice(["bf16", "fp32"]))


def _cdiv(a, b):
    return -(-a // b)


def _sizes(c):
    """Values of each gradient: the even ones matrices that share most of the total by halves, the others short vectors."""
    left, sizes = c["total"], []
    for i in range(c["tensors"] - 1):
        part = max(1, int(left * (c["matrix"] if i % 2 == 0 else 0.001)))
        part = min(part, left - (c["tensors"] - 1 - i))
        sizes.append(part)
        left -= part
    return sizes + [left]


def work(case):
    c, op = case, case["op"]
    if op in ("rms", "rms_grad"):
        count, b = c["rows"] * c["cols"], BYTES[c["dtype"]]
        small = 4 * c["rows"] + 4 * c["cols"]  # rstd, gamma
        if op == "rms":
            moved = count * b * (3 if c["residual"] else 1) + small
            moved += count + 4 * c["rows"] * _cdiv(c["cols"], E4M3_BLOCK) if c["fp8"] else count * b
            return {"bytes": moved, "flops": 5 * count}
        return {"bytes": count * b * (4 if c["dh"] else 3) + small + 4 * c["cols"], "flops": 9 * count}
    if op in ("logprobs", "logprobs_grad"):
        count, b = c["rows"] * c["classes"], BYTES[c["dtype"]]
        if op == "logprobs":
            return {"bytes": count * b + c["rows"] * (20 + 8 * c["top"]), "flops": 6 * count}
        return {"bytes": 2 * count * b + c["rows"] * (16 + (8 if c["entropy"] else 0)), "flops": 6 * count}
    if op == "clip":
        return {"bytes": 2 * c["total"] * BYTES[c["dtype"]] + 4, "flops": 3 * c["total"]}
    if op == "fp4_quantize":
        r, k = c["rows"], c["cols"]
        one = r * k * (BYTES["bf16"] + 0.5)
        scales = r * _cdiv(k, FP4_BLOCK) + (k * _cdiv(r, FP4_BLOCK) if c["both"] else 0)
        return {"bytes": r * k * BYTES[c["dtype"]] + one * (2 if c["both"] else 1) + scales, "flops": 2 * r * k}
    m, n, k = c["m"], c["n"], c["k"]
    moved = n * k / 2 + n * _cdiv(k, FP4_BLOCK) + m * n * BYTES[c["out"]] + (4 * n if c["bias"] else 0)
    moved += m * k * BYTES[c["dtype"]] if op == "fp4_linear" else m * k / 2 + m * _cdiv(k, FP4_BLOCK)
    return {"bytes": moved, "flops": 2 * m * n * k}


# ----------------------------------------------------------------- inputs
def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _rand(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda")


def _padded_rows(t, pad, dt):
    """t in rows that lie pad elements apart."""
    buf = torch.zeros(t.shape[0], t.shape[1] + pad, device="cuda", dtype=dt)
    buf[:, : t.shape[1]] = t
    return buf[:, : t.shape[1]]


def prepare(case, seed):
    c, op = case, case["op"]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"case": dict(c)}
    if op in ("rms", "rms_grad"):
        rows, cols, dt = c["rows"], c["cols"], DTYPES[c["dtype"]]
        spread = torch.exp(0.5 * _randn(gen, rows, 1))
        s["gamma"] = 1.0 + 0.2 * _randn(gen, cols)
        x = _padded_rows(_randn(gen, rows, cols) * spread, c["pad"], dt)
        if op == "rms":
            s["x"] = x
            s["residual"] = _padded_rows(2.0 * _randn(gen, rows, cols) * spread, c["pad"], dt) if c["residual"] else None
            return s
        s["h"] = x  # what the forward pass kept
        s["rstd"] = torch.rsqrt(x.float().square().mean(1) + EPS)
        s["dy"] = _randn(gen, rows, cols).to(dt)
        s["dh"] = _randn(gen, rows, cols).to(dt) if c["dh"] else None
        return s
    if op in ("logprobs", "logprobs_grad"):
        rows, classes, dt = c["rows"], c["classes"], DTYPES[c["dtype"]]
        x = _randn(gen, rows, classes)
        x = (x * (1.0 + 3.0 * _rand(gen, rows, 1)) + 5.0).to(dt)
        labels = (_rand(gen, rows) * classes).long().clamp(max=classes - 1)
        if c["masked"]:  # classes that are barred in every row, never a row's label
            barred = _rand(gen, classes) < c["masked"]
            x.masked_fill_(barred[None, :], float("-inf"))
            x[torch.arange(rows, device="cuda"), labels] = 6.0
        if rows > 4:
            labels[3] = -1  # a row without a label
        s["logits"], s["labels"] = x, labels.int()
        if op == "logprobs_grad":  # what the forward pass kept, and what comes from above
            logp, entropy, _, _, stats = _logprobs(x, s["labels"], 0)
            s["stats"], s["dlogp"] = stats, -(0.5 + _rand(gen, rows)) / rows
            s["entropy"], s["dentropy"] = (entropy, -0.01 * (0.5 + _rand(gen, rows)) / rows) if c["entropy"] else (None, None)
        return s
    if op == "clip":
        dt = DTYPES[c["dtype"]]
        s["grads"] = [(_randn(gen, n) * math.exp(-(i % 5))).to(dt) for i, n in enumerate(_sizes(c))]
        s["out"] = [torch.empty_like(g) for g in s["grads"]]  # where the optimizer reads them
        s["max_norm"] = 1.0
        return s
    if op == "fp4_quantize":
        x = _randn(gen, c["rows"], c["cols"]) * torch.exp(0.5 * _randn(gen, c["rows"], 1))
        s["x"] = x.to(DTYPES[c["dtype"]])
        return s
    m, n, k = c["m"], c["n"], c["k"]
    s["w"], s["w_scale"] = _fp4_packed(_randn(gen, n, k) / math.sqrt(k))
    s["bias"] = 0.1 * _randn(gen, n) if c["bias"] else None
    x = torch.relu(_randn(gen, m, k)) * torch.exp(0.5 * _randn(gen, m, 1))  # a layer's activity
    if op == "fp4_linear":
        s["x"] = x.to(DTYPES[c["dtype"]])
    else:
        s["a"], s["a_scale"] = _fp4_packed(x)
    return s


# ------------------------------------------------------------ plain forms
def _fp8(y):
    """y [rows, k] in 32 bits as e4m3 [rows, k padded to 16] and scales [ceil(k / 128), rows]."""
    rows, k = y.shape
    kb = _cdiv(k, E4M3_BLOCK)
    v = torch.nn.functional.pad(y, (0, kb * E4M3_BLOCK - k)).view(rows, kb, E4M3_BLOCK)
    amax = v.abs().amax(2, keepdim=True)
    scale = torch.clamp(amax / torch.full_like(amax, E4M3_MAX), min=SCALE_MIN)
    q = torch.clamp(v * (1.0 / scale), -E4M3_MAX, E4M3_MAX).view(rows, -1)
    return q[:, : _cdiv(k, 16) * 16].to(torch.float8_e4m3fn).contiguous(), scale.view(rows, kb).t().contiguous()


def _rms(s):
    c, x = s["case"], s["x"]
    h = x if s["residual"] is None else (x.float() + s["residual"].float()).to(x.dtype)
    v = h.float()
    rstd = torch.rsqrt(v.square().mean(1) + EPS)
    y = v * rstd[:, None] * s["gamma"]
    kept = (rstd,) if s["residual"] is None else (h, rstd)
    return (_fp8(y) if c["fp8"] else (y.to(x.dtype),)) + kept


def _rms_grad(s):
    h, dy = s["h"], s["dy"].float()
    n = h.float() * s["rstd"][:, None]
    du = dy * s["gamma"]
    dx = s["rstd"][:, None] * (du - n * (du * n).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return dx.to(h.dtype), (dy * n).sum(0)


def _logprobs(logits, labels, top):
    """Label's log-probability (0 without a label), entropy, the top classes' log-probabilities and indices, [max, log sum]."""
    x = logits.float()
    most = x.amax(1)
    d = x - most[:, None]
    e = torch.exp(d)
    total = e.sum(1)
    ln = torch.log(total)
    has = labels >= 0
    logp = torch.where(has, d.gather(1, labels.clamp(min=0).long()[:, None])[:, 0] - ln, 0.0)
    entropy = ln - torch.where(e > 0, e * d, 0.0).sum(1) / total
    bits = (x + 0.0).view(torch.int32).long()  # as whole numbers in the floats' order, then the lowest index first
    key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) + (x.shape[1] - 1 - torch.arange(x.shape[1], device=x.device))
    index = x.shape[1] - 1 - (key.topk(top, 1).values & 0xFFFFFFFF)
    return logp, entropy, d.gather(1, index) - ln[:, None], index.int(), torch.stack((most, ln), 1)


def _logprobs_grad(s):
    x, labels = s["logits"].float(), s["labels"]
    logp = x - s["stats"][:, :1] - s["stats"][:, 1:]
    p = torch.exp(logp)
    g = torch.where(labels >= 0, s["dlogp"], 0.0)
    grad = -p * g[:, None]
    if s["dentropy"] is not None:
        grad = grad - s["dentropy"][:, None] * torch.where(p > 0, p * (logp + s["entropy"][:, None]), 0.0)
    grad.scatter_add_(1, labels.clamp(min=0).long()[:, None], g[:, None])
    return grad.to(s["logits"].dtype)


def _clip(s):
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt().float()
    by = torch.clamp(s["max_norm"] / norm, max=1.0)
    return norm.view(1), [(g.float() * by).to(g.dtype) for g in s["grads"]]


def _power(e):
    """2 ** e in 32 bits, by its bits (-126 <= e <= 127)."""
    return ((e + 127) << 23).int().view(torch.float32)


def _fp4_values(x):
    """Of x [rows, k]: e2m1 values [rows, blocks, 32] and the exponents [rows, blocks, 1] of their power-of-two scales."""
    rows, k = x.shape
    kb = _cdiv(k, FP4_BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, kb * FP4_BLOCK - k)).view(rows, kb, FP4_BLOCK)
    amax = v.abs().amax(2, keepdim=True)
    e = torch.where(amax > 0, torch.frexp(amax)[1].long() - 3, -127).clamp(min=-127)  # floor(log2 amax) less e2m1's largest, 2
    a = v * _power(-e)  # a power of two that 32 bits hold: no rounding
    step = torch.where(a.abs() < 2, 0.5, torch.where(a.abs() < 4, 1.0, 2.0))
    return torch.clamp(torch.round(a / step) * step, -6.0, 6.0), e


def _fp4_stands_for(x):
    q, e = _fp4_values(x)
    half = torch.div(e, 2, rounding_mode="floor")  # 2 ** -127 is below the least power that has all its bits
    return (q * _power(half) * _power(e - half)).view(x.shape[0], -1)[:, : x.shape[1]].to(torch.bfloat16)


def _fp4_packed(x):
    """x as bytes of two e2m1 codes, the even index low [rows, 16 * blocks], and scale codes in tiles of 128 rows and four
    blocks [ceil(rows / 128), ceil(blocks / 4), 32, 4, 4]: row 32 i + j of a tile, block b at [j, i, b]."""
    q, e = _fp4_values(x)
    rows, kb = e.shape[:2]
    a = q.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    code = code.view(rows, -1)
    rb, cb = _cdiv(rows, 128), _cdiv(kb, 4)
    scale = torch.zeros(rb * 128, cb * 4, dtype=torch.uint8, device=x.device)
    scale[:rows, :kb] = (e[:, :, 0] + 127).to(torch.uint8)
    return code[:, ::2] | code[:, 1::2] << 4, scale.view(rb, 4, 32, cb, 4).permute(0, 3, 2, 1, 4).contiguous()


def _fp4_unpacked(q, scale, rows, k, dt):
    """The matrix [rows, k] that the bytes stand for."""
    levels = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=q.device, dtype=dt)
    code = torch.stack((q & 15, q >> 4), 2).view(rows, -1).long()
    v = levels[code & 7] * (1 - 2 * (code >> 3)).to(dt)
    e = scale.permute(0, 3, 2, 1, 4).reshape(scale.shape[0] * 128, -1)[:rows, : _cdiv(k, FP4_BLOCK)].long() - 127
    two = torch.full((), 2.0, device=q.device, dtype=torch.float64)
    return (v * torch.pow(two, e).to(dt).repeat_interleave(FP4_BLOCK, 1))[:, :k]


def _fp4_product(s, a):
    c = s["case"]
    y = a @ _fp4_unpacked(s["w"], s["w_scale"], c["n"], c["k"], torch.float32).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return (torch.relu(y) if c["relu"] else y).to(DTYPES[c["out"]])


def _run_plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "rms":
        return _rms(s)
    if op == "rms_grad":
        return _rms_grad(s)
    if op == "logprobs":
        return _logprobs(s["logits"], s["labels"], c["top"])
    if op == "logprobs_grad":
        return _logprobs_grad(s)
    if op == "clip":
        return _clip(s)
    if op == "fp4_quantize":
        one = (_fp4_stands_for(s["x"]),)
        return one + (_fp4_stands_for(s["x"].t()),) if c["both"] else one
    if op == "fp4_matmul":
        return _fp4_product(s, _fp4_unpacked(s["a"], s["a_scale"], c["m"], c["k"], torch.float32))
    return _fp4_product(s, _fp4_stands_for(s["x"]).float())


# ------------------------------------------------------- the library's calls
def _run_own(s):
    from paper_2404_08573_gb300 import ff

    c, op = s["case"], s["case"]["op"]
    if op == "rms":
        if c["fp8"]:
            a, h, rstd = ff.rms_norm_fp8(s["x"], s["gamma"], residual=s["residual"], eps=EPS)
            y = (a.q, a.scale)
        else:
            y, h, rstd = ff.rms_norm(s["x"], s["gamma"], residual=s["residual"], eps=EPS)
            y = (y,)
        return y + ((rstd,) if s["residual"] is None else (h, rstd))
    if op == "rms_grad":
        return ff.rms_norm_backward(s["dy"], s["h"], s["rstd"], s["gamma"], dh=s["dh"])
    if op == "logprobs":
        r = ff.label_logprobs(s["logits"], s["labels"], top=c["top"])
        return r.logp, r.entropy, r.top_logp, r.top_index, r.stats
    if op == "logprobs_grad":
        return ff.label_logprobs_backward(s["logits"], s["labels"], s["stats"], s["dlogp"], entropy=s["entropy"], dentropy=s["dentropy"])
    if op == "clip":
        return ff.clip_grad_norm(s["grads"], s["max_norm"], out=s["out"]), s["out"]
    if op == "fp4_quantize":
        if c["both"]:
            a, t = ff.fp4_quantize_both(s["x"])
            return ff.fp4_dequantize(a), ff.fp4_dequantize(t)
        return (ff.fp4_dequantize(ff.fp4_quantize(s["x"])),)
    a = ff.fp4_quantize(s["x"]) if op == "fp4_linear" else ff.Fp4Matrix(s["a"], s["a_scale"], c["m"], c["k"])
    w = ff.Fp4Matrix(s["w"], s["w_scale"], c["n"], c["k"])
    return ff.fp4_matmul(a, w, bias=s["bias"], relu=c["relu"], out_dtype=DTYPES[c["out"]])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------- the definitions in 64 bits
def _to_grid(a, fraction, least, most):
    """Nearest floating value with so many fraction bits, ties to even: least exponent ``least``, largest value ``most``."""
    e = torch.clamp(torch.frexp(a)[1].double() - 1, min=least)
    step = torch.exp2(e - fraction)
    return torch.clamp(torch.round(a / step) * step, -most, most)


def _rms_exact(s):
    c, x = s["case"], s["x"]
    h = x.double() if s["residual"] is None else (x.double() + s["residual"].double()).to(x.dtype).double()
    rstd = (torch.linalg.vector_norm(h, dim=1) ** 2 / c["cols"] + EPS) ** -0.5
    y = torch.einsum("rc,r,c->rc", h, rstd, s["gamma"].double())
    kept = (rstd,) if s["residual"] is None else (h, rstd)
    if not c["fp8"]:
        return (y,) + kept
    block = torch.arange(c["cols"], device="cuda") // E4M3_BLOCK
    kb = _cdiv(c["cols"], E4M3_BLOCK)
    scale = torch.zeros(c["rows"], kb, device="cuda", dtype=torch.float64)
    scale.scatter_reduce_(1, block.expand(c["rows"], -1), y.abs(), "amax")
    scale = (scale / E4M3_MAX).clamp(min=SCALE_MIN)
    q = torch.zeros(c["rows"], _cdiv(c["cols"], 16) * 16, device="cuda", dtype=torch.float64)
    q[:, : c["cols"]] = _to_grid(y / scale[:, block], 3, -6, E4M3_MAX)
    return (q, scale.t()) + kept


def _rms_grad_exact(s):
    """By the chain rule through the mean square."""
    c, h, dy = s["case"], s["h"].double(), s["dy"].double()
    rstd, gamma = s["rstd"].double(), s["gamma"].double()
    along = torch.einsum("rc,rc,c->r", dy, h, gamma)  # d sum(dy y) / d rstd
    dx = torch.einsum("rc,c,r->rc", dy, gamma, rstd) - torch.einsum("r,r,rc->rc", along, rstd ** 3, h) / c["cols"]
    if s["dh"] is not None:
        dx = dx + s["dh"].double()
    return dx, torch.einsum("rc,rc,r->c", dy, h, rstd)


def _logprobs_exact(s):
    x, labels, top = s["logits"].double(), s["labels"].long(), s["case"]["top"]
    most = x.max(1).values
    z = torch.logsumexp(x, 1)
    logp = torch.zeros_like(z)
    rows = torch.nonzero(labels >= 0)[:, 0]
    logp[rows] = x[rows, labels[rows]] - z[rows]
    every = x - z[:, None]
    entropy = -torch.where(torch.isinf(every), 0.0, torch.exp(every) * every).sum(1)
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    return logp, entropy, value[:, :top] - z[:, None], index[:, :top].int(), torch.stack((most, z - most), 1)


def _logprobs_grad_exact(s):
    x, labels = s["logits"].double(), s["labels"].long()
    z = s["stats"].double().sum(1)
    grad = torch.exp(x - z[:, None])
    p = grad.clone()
    rows = torch.nonzero(labels >= 0)[:, 0]
    g = torch.zeros_like(z)
    g[rows] = s["dlogp"].double()[rows]
    grad *= -g[:, None]
    grad[rows, labels[rows]] += g[rows]
    if s["dentropy"] is not None:
        inner = torch.where(p > 0, x - z[:, None] + s["entropy"].double()[:, None], 0.0)
        grad -= s["dentropy"].double()[:, None] * p * inner
    return grad


def _clip_exact(s):
    norm = math.sqrt(math.fsum(torch.linalg.vector_norm(g.double()).item() ** 2 for g in s["grads"]))
    by = min(1.0, s["max_norm"] / norm)
    return torch.tensor([norm], dtype=torch.float64, device="cuda"), [g.double() * by for g in s["grads"]]


def _fp4_exact(x):
    """The values that x's 4-bit form stands for: a block's scale is 2 to the floor of log2 of its largest magnitude, less 2."""
    rows, k = x.shape
    x = x.double()
    block = torch.arange(k, device="cuda") // FP4_BLOCK
    amax = torch.zeros(rows, _cdiv(k, FP4_BLOCK), device="cuda", dtype=torch.float64)
    amax.scatter_reduce_(1, block.expand(rows, -1), x.abs(), "amax")
    scale = torch.exp2(torch.clamp(torch.frexp(amax)[1].double() - 3, min=-127))
    scale = torch.where(amax > 0, scale, 2.0 ** -127)[:, block]
    return _to_grid(x / scale, 1, 0, 6.0) * scale


def exact(case, seed):
    s = prepare(case, seed)
    c, op = s["case"], case["op"]
    if op == "rms":
        return _rms_exact(s)
    if op == "rms_grad":
        return _rms_grad_exact(s)
    if op == "logprobs":
        return _logprobs_exact(s)
    if op == "logprobs_grad":
        return _logprobs_grad_exact(s)
    if op == "clip":
        return _clip_exact(s)
    if op == "fp4_quantize":
        one = (_fp4_exact(s["x"]),)
        return one + (_fp4_exact(s["x"].t()),) if c["both"] else one
    m, n, k = c["m"], c["n"], c["k"]
    a = _fp4_exact(s["x"]) if op == "fp4_linear" else _fp4_unpacked(s["a"], s["a_scale"], m, k, torch.float64)
    y = a @ _fp4_unpacked(s["w"], s["w_scale"], n, k, torch.float64).t()
    if s["bias"] is not None:
        y = y + s["bias"].double()
    return torch.where(y > 0, y, 0.0) if c["relu"] else y
