"""4-bit matrices: the quantizer and its inverse bit for bit against their
definition, and the product against the exact product of what its operands
stand for.

Product tolerance: e2m1 products times two powers of two are exact in fp32, and
the tensor cores add them up in fp32 (each addition within 2^-23, truncating
adders included), partial sums of up to 8 slices of the contraction once more:
|err| <= 2^-23 (k + 12) * sum |a b| element by element, then the bias, and the
half step of the output type.
"""

import numpy as np
import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def quantize_ref(x):
    """Of fp32 x [rows, k]: values on the grid [rows, 32 * blocks], exponents [rows, blocks] (-127 .. 125), in 64 bits."""
    x = np.asarray(x, np.float64)
    rows, k = x.shape
    kb = -(-k // 32)
    full = np.zeros((rows, kb, 32))
    full.reshape(rows, -1)[:, :k] = x
    amax = np.abs(full).max(axis=2)
    e = np.where(amax > 0, np.frexp(amax)[1] - 3, -127)
    e = np.maximum(e, -127)
    v = full * 2.0 ** -e[:, :, None]
    _, f = np.frexp(v)
    step = 2.0 ** (np.maximum(f - 1, 0) - 1)  # e2m1: one fraction bit, least exponent 0
    return np.clip(np.round(v / step) * step, -6, 6).reshape(rows, -1), e


def pack_ref(v, e):
    """Codes [rows, 16 * blocks] and scale tiles of values and exponents."""
    a = np.abs(v)
    code = np.where(a < 2, a * 2, np.where(a < 4, a + 2, a / 2 + 4)).astype(np.uint8) | (np.signbit(v).astype(np.uint8) << 3)
    rows, kb = e.shape
    scale = np.zeros((-(-rows // 128) * 128, -(-kb // 4) * 4), np.uint8)
    scale[:rows, :kb] = e + 127
    tiles = scale.reshape(-(-rows // 128), 4, 32, -(-kb // 4), 4).transpose(0, 3, 2, 1, 4)
    return code[:, ::2] | code[:, 1::2] << 4, tiles


def strided(torch, t, pad, lead):
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + lead,), float("nan"), dtype=t.dtype, device="cuda")
    view = buf[lead:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


QSIZES = [(1, 1), (1, 32), (1, 33), (31, 2), (32, 64), (33, 31), (128, 128), (129, 127), (3, 16), (127, 130), (300, 77), (2000, 784),
          (65, 1337), (1, 8192)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", QSIZES)
def test_quantize_bit_for_bit(size, dtype):
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
    xg = strided(torch, x, *((0, 0), (8, 0), (3, 1), (2, 2))[n % 4])
    straight, transposed = ff.fp4_quantize_both(xg)
    one, other = ff.fp4_quantize(xg), ff.fp4_quantize(xg, transpose=True)
    for got, again, ref in ((straight, one, x.float().numpy()), (transposed, other, x.float().numpy().T)):
        v, e = quantize_ref(ref)
        q, scale = pack_ref(v, e)
        assert got.q.shape == q.shape and got.scale.shape == scale.shape
        assert np.array_equal(got.scale.cpu().numpy(), scale)
        assert np.array_equal(got.q.cpu().numpy(), q)
        assert torch.equal(got.q, again.q) and torch.equal(got.scale, again.scale)
        want = (v * np.repeat(2.0 ** e, 32, axis=1))[:, :ref.shape[1]]
        assert np.array_equal(ff.fp4_dequantize(got, out_dtype=torch.float32).double().cpu().numpy(), want)
        assert np.array_equal(ff.fp4_dequantize(got).double().cpu().numpy(), want)  # exact in bf16 too
        for pad, lead in ((3, 1), (8, 8)):
            buf = torch.full((lead + ref.shape[0] * (ref.shape[1] + pad) + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
            view = buf[lead:lead + ref.shape[0] * (ref.shape[1] + pad)].view(ref.shape[0], -1)[:, :ref.shape[1]]
            assert ff.fp4_dequantize(got, out=view) is view and np.array_equal(view.double().cpu().numpy(), want)
            view.fill_(7.0)
            assert bool((buf == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(5, 641), (33, 2049), (130, 1337), (257, 300), (300, 78), (640, 37), (1030, 1021),
                                  (40000, 37), (9001, 130)])
def test_rows_of_every_alignment(size, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    rows, k = size
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn(rows, k, generator=torch.Generator().manual_seed(rows)).to(dt)
    refs = [pack_ref(*quantize_ref(r)) for r in (x.float().numpy(), x.float().numpy().T)]
    v, e = quantize_ref(x.float().numpy())
    want = torch.from_numpy((v * np.repeat(2.0 ** e, 32, axis=1))[:, :k]).cuda()
    for pad, lead in ((0, 0), (1, 0), (2, 2), (3, 1), (4, 4), (8, 8)):
        xg = strided(torch, x, pad, lead)
        both = ff.fp4_quantize_both(xg)
        for got, (q, scale) in ((both[0], refs[0]), (both[1], refs[1]), (ff.fp4_quantize(xg), refs[0])):
            assert np.array_equal(got.scale.cpu().numpy(), scale) and np.array_equal(got.q.cpu().numpy(), q)
        for out_dt in (torch.bfloat16, torch.float32):
            buf = torch.full((lead + rows * (k + pad) + 64,), 7.0, dtype=out_dt, device="cuda")
            view = buf[lead:lead + rows * (k + pad)].view(rows, -1)[:, :k]
            ff.fp4_dequantize(both[0], out=view)
            assert torch.equal(view.double(), want)  # both types hold every value
            view.fill_(7.0)
            assert bool((buf == 7.0).all())


def test_every_code_and_midpoint():
    torch = torch_cuda()
    ff = lib_ready()
    grid = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
    points = np.concatenate((grid, (grid[1:] + grid[:-1]) / 2, [6.5, 7, 7.75], np.nextafter(np.float32(2.5), 3)[None]))
    x = np.zeros((2 * points.size, 32), np.float32)
    x[:, 0] = 4.0  # scale 1
    x[:, 5] = np.concatenate((points, -points))
    got = ff.fp4_quantize(torch.from_numpy(x).cuda())
    assert np.array_equal(ff.fp4_dequantize(got, out_dtype=torch.float32).double().cpu().numpy(), quantize_ref(x)[0])


def test_blocks_that_are_not_finite():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(70, 100, device="cuda")
    clean = ff.fp4_dequantize(ff.fp4_quantize(x))
    x[1, 5], x[2, 70] = float("nan"), -float("inf")
    for a, back in ((ff.fp4_quantize(x), ff.fp4_dequantize(ff.fp4_quantize(x))),):
        hit = torch.zeros(70, 100, dtype=torch.bool, device="cuda")
        hit[1, :32] = hit[2, 64:96] = True
        assert bool(back[hit].isnan().all()) and torch.equal(back[~hit], clean[~hit])
    w = ff.fp4_quantize(torch.randn(40, 100, device="cuda"))
    for relu in (False, True):
        c = ff.fp4_matmul(a, w, relu=relu)
        assert bool(c[1:3].isnan().all()) and bool(torch.isfinite(c[[0, 3, 69]]).all())


SIZES = [(1, 1, 1), (1, 16, 32), (1, 2000, 784), (3, 10, 2000), (16, 128, 256), (17, 129, 300), (32, 500, 64), (33, 70, 65),
         (64, 300, 1000), (100, 2000, 784), (128, 128, 8192), (130, 260, 520), (333, 1999, 1337), (256, 4000, 96), (500, 500, 500),
         (1, 8192, 8192), (2048, 2000, 784), (1000, 3001, 2000), (4096, 1030, 513)]


def exact(ff, torch, a, b):
    return (ff.fp4_dequantize(a, out_dtype=torch.float32).double(), ff.fp4_dequantize(b, out_dtype=torch.float32).double())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES)
def test_matmul(size, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = size
    i = SIZES.index(size)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(i)
    x = torch.randn(m, k, generator=gen) * torch.exp(2 * torch.randn(m, 1, generator=gen))
    w = torch.randn(n, k, generator=gen) * torch.exp(torch.randn(n, -(-k // 32), generator=gen)).repeat_interleave(32, 1)[:, :k]
    a, b = ff.fp4_quantize(x.cuda()), ff.fp4_quantize(w.cuda())
    av, bv = exact(ff, torch, a, b)
    bias = torch.randn(n, generator=gen).cuda() if i % 2 else None
    want = av @ bv.t()
    size_of = av.abs() @ bv.abs().t()
    for relu in (False, True):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        c = ff.fp4_matmul(a, b, bias=bias, relu=relu, out_dtype=dt, status=status)
        v = want if bias is None else want + bias.double()
        tol = 2 * U * (k + 12) * size_of + (0 if bias is None else 2 * U * (want.abs() + bias.double().abs()))
        tol = tol + v.abs() * (torch.finfo(dt).eps / 2) + 2.0 ** -120
        if relu:
            v = v.clamp(min=0)
        assert c.shape == (m, n) and c.dtype == dt and int(status) == 0
        assert bool(((c.double() - v).abs() <= tol).all())
        assert torch.equal(c, ff.fp4_matmul(a, b, bias=bias, relu=relu, out_dtype=dt))
    for pad, lead in ((0, 0), (5, 3), (8, 8), (-n % 8, 8)):
        buf = torch.full((lead + m * (n + pad) + 64,), 7.0, dtype=dt, device="cuda")
        view = buf[lead:lead + m * (n + pad)].view(m, n + pad)[:, :n]
        assert ff.fp4_matmul(a, b, bias=bias, relu=True, out=view) is view
        assert torch.equal(view, c)
        view.fill_(7.0)
        assert bool((buf == 7.0).all())
    ff.fp8_check()


def test_three_products_of_a_layer():
    """y = x w^T, dx = dy w and dw = dy^T x from one quantization of each, both ways round."""
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = 200, 300, 150
    x, w, dy = (torch.randn(*s, device="cuda") for s in ((m, k), (n, k), (m, n)))
    (xs, xt), (ws, wt), (ds, dt) = (ff.fp4_quantize_both(t) for t in (x, w, dy))
    for a, b in ((xs, ws), (ds, wt), (dt, xt)):
        av, bv = exact(ff, torch, a, b)
        got = ff.fp4_matmul(a, b, out_dtype=torch.float32).double()
        assert got.shape == (a.rows, b.rows)
        assert bool(((got - av @ bv.t()).abs() <= 2 * U * (a.k + 12) * (av.abs() @ bv.abs().t())).all())


def test_extreme_scales():
    """Products of blocks at the ends of the scale's range, inside fp32's."""
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(20, 256, device="cuda").abs() + 0.5
    for up, down in ((2.0 ** 100, 2.0 ** -100), (2.0 ** -120, 2.0 ** 100), (2.0 ** -60, 2.0 ** -50)):
        a, b = ff.fp4_quantize(x * up), ff.fp4_quantize(x * down)
        av, bv = exact(ff, torch, a, b)
        want = av @ bv.t()
        got = ff.fp4_matmul(a, b, out_dtype=torch.float32).double()
        assert bool(((got - want).abs() <= 2 * U * 268 * want).all())


def test_graph_and_streams():
    torch = torch_cuda()
    ff = lib_ready()
    x, w = torch.randn(70, 784, device="cuda"), ff.fp4_quantize(torch.randn(500, 784, device="cuda"))

    def step(stream=None):
        return ff.fp4_matmul(ff.fp4_quantize(x, stream=stream), w, relu=True, stream=stream)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    x.normal_()
    graph.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = step(side)
    torch.cuda.synchronize()
    assert torch.equal(held, step()) and torch.equal(held, other)


def test_empty_and_refusals():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(8, 64, device="cuda")
    a, b = ff.fp4_quantize(x), ff.fp4_quantize(torch.randn(5, 64, device="cuda"))
    none = ff.fp4_quantize(x[:0])
    assert none.q.shape == (0, 32) and ff.fp4_matmul(none, b).shape == (0, 5) and ff.fp4_matmul(b, none).shape == (5, 0)
    assert ff.fp4_dequantize(none).shape == (0, 64)
    other = ff.fp4_quantize(torch.randn(5, 65, device="cuda"))
    for bad, call in ((TypeError, lambda: ff.fp4_quantize(x.half())), (ValueError, lambda: ff.fp4_quantize(x[0])),
                      (ValueError, lambda: ff.fp4_quantize(x.t())), (ValueError, lambda: ff.fp4_quantize(x.cpu())),
                      (ValueError, lambda: ff.fp4_quantize(x[:0], transpose=True)), (TypeError, lambda: ff.fp4_matmul(a, x)),
                      (TypeError, lambda: ff.fp4_matmul(x, a)), (ValueError, lambda: ff.fp4_matmul(a, other)),
                      (ValueError, lambda: ff.fp4_matmul(a, b, bias=torch.zeros(4, device="cuda"))),
                      (ValueError, lambda: ff.fp4_matmul(a, b, out=x)), (TypeError, lambda: ff.fp4_matmul(a, b, out_dtype=torch.half)),
                      (TypeError, lambda: ff.fp4_dequantize(x)), (ValueError, lambda: ff.fp4_dequantize(a, out=x[:2])),
                      (ValueError, lambda: ff.Fp4Matrix(a.q, b.scale, 8, 96)), (ValueError, lambda: ff.Fp4Matrix(a.q[:, :16], a.scale, 8, 64)),
                      (TypeError, lambda: ff.fp4_matmul(ff.fp8_quantize(x), b))):
        with pytest.raises(bad):
            call()
