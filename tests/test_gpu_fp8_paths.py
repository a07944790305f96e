"""The 8-bit product's kernels at sizes that reach all of each: CTA pairs that
take several tiles of several k-blocks, with every kind of scale and of C, and
split products of 128 columns.  Against 64 bits on the GPU; tolerances as in
test_gpu_fp8.py."""

import ctypes

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu


def launched(ff, call):
    """call()'s result and its kernels: kind -> launches."""
    L = ff.lib()
    L.ff_profile_read.restype = ctypes.c_int
    names, counts = (ctypes.c_char_p * 64)(), (ctypes.c_longlong * 64)()
    ms, work = (ctypes.c_double * 64)(), (ctypes.c_double * 64)()
    L.ff_profile_enable(1)
    try:
        out = call()
        n = L.ff_profile_read(64, names, counts, ms, work)
    finally:
        L.ff_profile_enable(0)
    return out, {names[i].decode(): counts[i] for i in range(n)}


def operands(torch, ff, m, n, k, tile, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    a = torch.randn(m, k, generator=gen, device="cuda") * torch.exp(torch.randn(m, 1, generator=gen, device="cuda"))
    b = 0.1 * torch.randn(n, k, generator=gen, device="cuda") * torch.exp(torch.randn(n, 1, generator=gen, device="cuda"))
    a[:, : k // 3] *= 50  # scales that differ from block to block
    return ff.fp8_quantize(a), ff.fp8_quantize(b, tile=tile), torch.randn(n, generator=gen, device="cuda")


def values(m):
    s = m.scale.double().t().repeat_interleave(128, 1)[:, :m.k]
    return m.q.float().double()[:, :m.k] * (s.repeat_interleave(128, 0)[:m.rows] if m.tile else s)


def check(torch, got, a, b, bias, relu):
    A, B = values(a), values(b).t()
    ref = A @ B + bias.double()
    tol = 2.0 ** -23 * ((128 + -(-a.k // 128) + 4) * (A.abs() @ B.abs()) + bias.double().abs()) + 1e-37
    if relu:
        ref = ref.clamp(min=0)
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -23
    bad = ~((got.double() - ref).abs() <= tol + half * ref.abs())
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())


PAIR = "fp8_gemm_pair_tc"


@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(2501, 4303, 700), (2504, 4304, 700)])
def test_pairs_with_several_tiles(size, dtype, tile):
    """10 x 17 tiles of 256 x 256: two or three for each pair of SMs, six k-blocks each, the last one and the last tiles
    ragged.  Rows of C that are not 16-byte aligned, and rows that are."""
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = size
    a, b, bias = operands(torch, ff, m, n, k, tile, seed=n)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    got, kinds = launched(ff, lambda: ff.fp8_matmul(a, b, bias=bias, relu=tile, out_dtype=dt))
    assert kinds == {PAIR: 1}
    check(torch, got, a, b, bias, tile)
    ff.fp8_check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tile", [False, True])
def test_pairs_write_only_their_matrix(tile, dtype):
    """C within larger buffers, at odd strides and starts: the gaps keep what they held."""
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = 2055, 2001, 784
    a, b, bias = operands(torch, ff, m, n, k, tile, seed=3)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    want, kinds = launched(ff, lambda: ff.fp8_matmul(a, b, bias=bias, out_dtype=dt))
    assert kinds == {PAIR: 1}
    check(torch, want, a, b, bias, False)
    for pad, lead in ((5, 3), (7, 8), (15, 16), (1, 0)):
        buf = torch.full((lead + m * (n + pad) + 64,), 7.0, dtype=dt, device="cuda")
        out = buf[lead:lead + m * (n + pad)].view(m, n + pad)[:, :n]
        assert ff.fp8_matmul(a, b, bias=bias, out=out) is out
        assert torch.equal(out, want)
        out.fill_(7.0)
        assert bool((buf == 7.0).all())


@pytest.mark.parametrize("tile", [False, True])
def test_the_large_layer(tile):
    torch = torch_cuda()
    ff = lib_ready()
    a, b, bias = operands(torch, ff, 4096, 8192, 8192, tile, seed=8)
    got, kinds = launched(ff, lambda: ff.fp8_matmul(a, b, bias=bias))
    assert kinds == {PAIR: 1}
    check(torch, got, a, b, bias, False)


# 128 columns: A's rows on them with the contraction split over 4 and 2 CTAs or whole, and B's rows on them
@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("size", [(106, 4584, 4903), (200, 4000, 4000), (890, 1284, 7515), (700, 700, 8000), (65, 8000, 3000)])
def test_split_products_of_128_columns(size, tile):
    torch = torch_cuda()
    ff = lib_ready()
    a, b, bias = operands(torch, ff, *size, tile, seed=size[0])
    for dt, relu in ((torch.float32, False), (torch.bfloat16, True)):
        got, kinds = launched(ff, lambda: ff.fp8_matmul(a, b, bias=bias, relu=relu, out_dtype=dt))
        assert kinds == {"fp8_gemm_tc": 1}
        check(torch, got, a, b, bias, relu)
