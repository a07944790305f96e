"""The 8-bit quantizer, bit for bit against its definition, and the 8-bit
matrix product against the exact product of what its operands stand for.

Product tolerance: e4m3 products are exact in fp32; a k-block sums 128 of them
on the tensor cores (each addition within 2^-23, truncating adders included),
each block is scaled by one rounded product of scales and added with one more
rounding.  So |err| <= 2^-23 (128 + blocks + 4) * sum |a b| element by
element, plus half a unit of the output type.
"""

import numpy as np
import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu


def e4m3_round(v):
    """fp32 values in [-448, 448] to the nearest e4m3 value, ties to even, in 64 bits."""
    v = np.asarray(v, np.float64)
    _, e = np.frexp(v)
    step = 2.0 ** (np.maximum(e - 1, -6) - 3)
    return np.clip(np.round(v / step) * step, -448.0, 448.0)  # np.round: half to even


def quantize_ref(x, tile):
    """Values [rows, ceil16(k)] and scales [k blocks, rows or row blocks] of finite fp32 x."""
    x = np.asarray(x, np.float32)
    rows, k = x.shape
    kb, rb = -(-k // 128), -(-rows // 128)
    full = np.zeros((rb * 128, kb * 128), np.float32)
    full[:rows, :k] = x
    blocks = np.abs(full.reshape(rb, 128, kb, 128))
    amax = blocks.max(axis=(1, 3)) if tile else blocks.max(axis=3).reshape(rb * 128, kb)[:rows]
    scale = np.maximum((amax / np.float32(448.0)).astype(np.float32), np.float32(2.0 ** -126))
    inv = (np.float32(1.0) / scale).astype(np.float32)
    per = np.repeat(np.repeat(inv, 128, axis=0)[:rows] if tile else inv, 128, axis=1)
    q = e4m3_round((full[:rows] * per).astype(np.float32))
    return q[:, :-(-k // 16) * 16], scale.T


def strided(torch, t, pad, lead):
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + lead,), float("nan"), dtype=t.dtype, device="cuda")
    view = buf[lead:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


def values(m):
    """What an Fp8Matrix stands for, in 64 bits."""
    q = m.q.float().double().cpu().numpy()[:, :m.k]
    s = np.repeat(m.scale.double().cpu().numpy().T, 128, axis=1)[:, :m.k]
    return q * (np.repeat(s, 128, axis=0)[:m.rows] if m.tile else s)


QSIZES = [(1, 1), (1, 128), (1, 2000), (128, 128), (129, 127), (3, 16), (127, 130), (300, 77), (2000, 784), (65, 1337)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("size", QSIZES)
def test_quantize_bit_for_bit(size, tile, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    rows, k = size
    n = QSIZES.index(size)
    gen = torch.Generator().manual_seed(n)
    x = torch.randn(rows, k, generator=gen) * torch.exp(3 * torch.randn(rows, 1, generator=gen))
    x[:, ::7] = 0
    if n % 3 == 0:
        x[: rows // 2] = 0  # blocks of zeros only
    if n % 4 == 1:
        x *= 1e-38  # scales at the floor, subnormal inputs
    if n % 4 == 2:
        x *= 1e30
    x = x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    xg = strided(torch, x, *((0, 0), (8, 0), (3, 1))[n % 3])
    straight, transposed = ff.fp8_quantize_both(xg, tile=tile)
    one, other = ff.fp8_quantize(xg, tile=tile), ff.fp8_quantize(xg, tile=tile, transpose=True)
    for got, again, ref in ((straight, one, x.float().numpy()), (transposed, other, x.float().numpy().T)):
        q, scale = quantize_ref(ref, tile)
        assert got.q.shape == q.shape and got.scale.shape == scale.shape
        assert np.array_equal(got.scale.cpu().numpy(), scale)
        assert np.array_equal(got.q.float().cpu().numpy(), q)
        assert torch.equal(got.q.view(torch.uint8), again.q.view(torch.uint8)) and torch.equal(got.scale, again.scale)


def test_quantize_ties_and_extremes():
    """Every e4m3 midpoint rounds to even; the largest of a block is 448 exactly."""
    torch = torch_cuda()
    ff = lib_ready()
    grid = np.unique(np.abs(e4m3_round(np.concatenate([np.linspace(0, 448, 20001), np.linspace(0, 0.1, 20001)]))))
    mid = (grid[1:] + grid[:-1]) / 2  # exact in fp32
    rows = -(-mid.size // 127)
    x = np.zeros((rows, 128), np.float32)
    flat = np.zeros(rows * 127, np.float32)
    flat[:mid.size] = mid
    x[:, 0], x[:, 1:] = 448.0, flat.reshape(rows, 127)
    x[1::2] *= -1
    got = ff.fp8_quantize(torch.from_numpy(x).cuda())
    assert np.array_equal(got.scale.cpu().numpy(), np.ones((1, rows), np.float32))
    assert np.array_equal(got.q.float().cpu().numpy(), e4m3_round(x))


def test_quantize_marks_non_finite_blocks():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(4, 300, device="cuda")
    clean = ff.fp8_quantize(x)
    x[1, 5], x[2, 290] = float("nan"), -float("inf")
    a = ff.fp8_quantize(x)
    s = a.scale.cpu().numpy()
    assert np.isnan(s[0, 1]) and np.isinf(s[2, 2])
    hit = np.zeros((3, 4), bool)
    hit[0, 1] = hit[2, 2] = True
    assert np.array_equal(s[~hit], clean.scale.cpu().numpy()[~hit])
    w = ff.fp8_quantize(torch.randn(40, 300, device="cuda"), tile=True)
    for relu in (False, True):
        y = ff.fp8_matmul(a, w, relu=relu)
        assert torch.isnan(y[1:3]).all() and torch.isfinite(y[[0, 3]]).all()
    bad = torch.randn(200, 300, device="cuda")
    bad[150, 10] = float("inf")
    y = ff.fp8_matmul(clean, ff.fp8_quantize(bad, tile=True))
    assert torch.isfinite(y[:, :128]).all() and torch.isnan(y[:, 128:]).all()


def operands(torch, ff, m, n, k, tile, seed):
    gen = torch.Generator().manual_seed(seed)
    a = torch.randn(m, k, generator=gen) * torch.exp(torch.randn(m, 1, generator=gen))
    b = torch.randn(n, k, generator=gen) * torch.exp(torch.randn(n, 1, generator=gen)) * 0.1
    a[:, : k // 3] *= 50  # scales that differ from block to block
    return ff.fp8_quantize(a.cuda()), ff.fp8_quantize(b.cuda(), tile=tile), gen


def check_product(got, a, b, bias, relu):
    A, B = values(a), values(b)
    ref, mag = A @ B.T, np.abs(A) @ np.abs(B).T
    blocks = -(-a.k // 128)
    tol = 2.0 ** -23 * (128 + blocks + 4) * mag + 1e-37
    if bias is not None:
        bias = bias.double().cpu().numpy()
        ref, tol = ref + bias, tol + 2.0 ** -23 * np.abs(bias)
    if relu:
        ref = np.maximum(ref, 0)
    g = got.double().cpu().numpy()
    assert g.shape == ref.shape
    half = 2.0 ** -8 if str(got.dtype) == "torch.bfloat16" else 2.0 ** -23
    bad = ~(np.abs(g - ref) <= tol + half * np.abs(ref))
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), g[bad][:4], ref[bad][:4])


MATMULS = [
    (1, 1, 1), (1, 16, 128), (1, 2000, 2000), (2, 130, 129), (3, 1999, 1337), (16, 257, 300), (17, 64, 127), (31, 500, 784),
    (64, 129, 2000), (65, 100, 1000), (127, 128, 16), (128, 256, 256), (129, 255, 513), (200, 2000, 784), (256, 256, 128),
    (257, 511, 640), (333, 1999, 1337), (512, 10, 2000), (640, 1024, 384), (1000, 3, 130), (2048, 2000, 784), (1500, 777, 257),
]


@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("size", MATMULS)
def test_matmul(size, tile):
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = size
    i = MATMULS.index(size)
    a, b, gen = operands(torch, ff, m, n, k, tile, seed=i)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for out_dtype, relu, with_bias in ((torch.bfloat16, i % 2 == 0, True), (torch.float32, i % 2 == 1, i % 3 == 0)):
        bias = torch.randn(n, generator=gen).cuda() if with_bias else None
        got = ff.fp8_matmul(a, b, bias=bias, relu=relu, out_dtype=out_dtype, status=status)
        check_product(got, a, b, bias, relu)
        again = ff.fp8_matmul(a, b, bias=bias, relu=relu, out_dtype=out_dtype)
        assert torch.equal(got, again)
    assert int(status) == 0


@pytest.mark.parametrize("size", [(1, 300, 500), (40, 131, 257), (300, 515, 400)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_matmul_writes_only_its_matrix(size, dtype):
    """Rows of an odd stride, an odd start: the gaps keep what they held."""
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = size
    a, b, _ = operands(torch, ff, m, n, k, True, seed=77)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    want = ff.fp8_matmul(a, b, out_dtype=dt)
    for pad, lead in ((5, 3), (8, 8), (1, 0)):
        buf = torch.full((lead + m * (n + pad) + 16,), 7.0, dtype=dt, device="cuda")
        out = buf[lead:lead + m * (n + pad)].view(m, n + pad)[:, :n]
        assert ff.fp8_matmul(a, b, out=out) is out
        assert torch.equal(out, want)
        out.fill_(7.0)
        assert bool((buf == 7.0).all())


def test_layer_products():
    """The forward product and both products of the backward pass, against the exact products of the quantized operands;
    and the whole against the unquantized layer, within the quantizer's error (each operand within 2^-4 of itself or,
    near zero, 2^-10 scales): the relative error of the norms stays below 2 * 2^-4."""
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = 300, 500, 784
    gen = torch.Generator().manual_seed(5)
    x, w, dy = (torch.randn(*s, generator=gen).cuda() for s in ((m, k), (n, k), (m, n)))
    xq, xt = ff.fp8_quantize_both(x)
    wq, wt = ff.fp8_quantize_both(w, tile=True)
    dq, dt = ff.fp8_quantize_both(dy)
    for a, b, exact in ((xq, wq, x.double() @ w.double().t()), (dq, wt, dy.double() @ w.double()),
                        (dt, xt, dy.double().t() @ x.double())):
        got = ff.fp8_matmul(a, b, out_dtype=torch.float32)
        check_product(got, a, b, None, False)
        assert float((got.double() - exact).norm() / exact.norm()) < 2 * 2.0 ** -4


def test_offsets_past_32_bits():
    """An operand and an output of more than 2^31 bytes and elements: the last rows, against the same rows alone."""
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = 34000, 65600, 65600  # a: 2.2 GB, c: 2.2e9 elements
    aq = torch.zeros(m, k, dtype=torch.uint8, device="cuda")
    aq[-300:] = torch.randint(0, 0x77, (300, k), dtype=torch.uint8, device="cuda")  # finite, non-negative
    sa = torch.rand(-(-k // 128), m, device="cuda") + 0.5
    bq = torch.randint(0, 0x77, (n, 16), dtype=torch.uint8, device="cuda")
    a16 = ff.Fp8Matrix(aq[:, :16].contiguous().view(torch.float8_e4m3fn), sa[:1].contiguous(), m, 16)
    b16 = ff.Fp8Matrix(bq.view(torch.float8_e4m3fn), torch.rand(1, -(-n // 128), device="cuda") + 0.5, n, 16, tile=True)
    c = ff.fp8_matmul(a16, b16)  # an output past 2^31 elements
    tail = ff.Fp8Matrix(a16.q[-300:].contiguous(), sa[:1, -300:].contiguous(), 300, 16)
    assert torch.equal(c[-300:], ff.fp8_matmul(tail, b16))
    del c
    big = ff.Fp8Matrix(aq.view(torch.float8_e4m3fn), sa, m, k)  # an operand past 2^31 bytes
    w = ff.Fp8Matrix(torch.randint(0, 0x77, (40, k), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
                     torch.rand(-(-k // 128), 1, device="cuda") + 0.5, 40, k, tile=True)
    tail = ff.Fp8Matrix(aq[-300:].contiguous().view(torch.float8_e4m3fn), sa[:, -300:].contiguous(), 300, k)
    y, z = ff.fp8_matmul(big, w, out_dtype=torch.float32)[-300:], ff.fp8_matmul(tail, w, out_dtype=torch.float32)
    # the two sizes may sum in other orders: k/128 + 128 roundings of positive sums at most
    assert float(((y - z).abs() / z).max()) <= 2 * 2.0 ** -23 * (128 + k / 128 + 4)
    del big, aq
    x = torch.zeros(34000, 65600, dtype=torch.bfloat16, device="cuda")  # 2.2e9 elements
    x[-1] = torch.randn(65600, device="cuda")
    q, one = ff.fp8_quantize(x), ff.fp8_quantize(x[-1:])
    assert torch.equal(q.q[-1].view(torch.uint8), one.q[0].view(torch.uint8)) and torch.equal(q.scale[:, -1], one.scale[:, 0])


def test_streams_and_a_captured_graph():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(100, 900, device="cuda")
    w = ff.fp8_quantize(torch.randn(700, 900, device="cuda"), tile=True)
    want = ff.fp8_matmul(ff.fp8_quantize(x), w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ff.fp8_matmul(ff.fp8_quantize(x, stream=side), w, stream=side)
    for _ in range(20):
        torch.full((1 << 16,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    static = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = ff.fp8_matmul(ff.fp8_quantize(static), w)
    for k in range(3):
        static.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ff.fp8_matmul(ff.fp8_quantize(static), w))


def test_empty_and_refused():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(6, 40, device="cuda")
    a, w = ff.fp8_quantize(x), ff.fp8_quantize(torch.randn(9, 40, device="cuda"), tile=True)
    none = ff.fp8_quantize(x[:0])
    assert ff.fp8_matmul(none, w).shape == (0, 9)
    for bad in (x.cpu(), x.half(), x.t(), x[0], x[:, :0], x[:1].expand(6, 40)):
        with pytest.raises((TypeError, ValueError)):
            ff.fp8_quantize(bad)
    with pytest.raises(ValueError):
        ff.fp8_quantize_both(x[:0])
    other = ff.fp8_quantize(torch.randn(9, 41, device="cuda"), tile=True)
    for args, kw in (((a, other), {}), ((w, w), {}), ((a, w), dict(out_dtype=torch.float16)),
                     ((a, w), dict(bias=torch.ones(8, device="cuda"))), ((a, w), dict(out=torch.empty(6, 8, device="cuda"))),
                     ((a, w), dict(status=torch.zeros(1, device="cuda"))), ((a, w), dict(out=torch.empty(9, 6, device="cuda").t()))):
        with pytest.raises((TypeError, ValueError)):
            ff.fp8_matmul(*args, **kw)
    for q, s, rows, k, tile in ((a.q[:5], a.scale, 6, 40, False), (a.q, a.scale, 6, 60, False), (a.q, a.scale, 6, 40, True),
                                (a.q.float(), a.scale, 6, 40, False), (a.q, a.scale.double(), 6, 40, False)):
        with pytest.raises(ValueError):
            ff.Fp8Matrix(q, s, rows, k, tile=tile)
