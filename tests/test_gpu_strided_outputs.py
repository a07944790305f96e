"""Outputs inside larger buffers, at odd strides and starts: what lies between and around their rows keeps what it held."""

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
GAPS = ((0, 0), (5, 3), (8, 8), (1, 0), (4, 4))  # elements between rows, elements before the first


def inside(torch, shape, dtype, pad, lead):
    """A buffer of sevens and a view of the shape in it."""
    rows, cols = 1, shape[-1]
    for d in shape[:-1]:
        rows *= d
    buf = torch.full((lead + rows * (cols + pad) + 64,), 7.0, dtype=dtype, device="cuda")
    return buf, buf[lead:lead + rows * (cols + pad)].view(*shape[:-1], cols + pad)[..., :cols]


def untouched(buf, view):
    view.fill_(7.0)
    return bool((buf == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(70, 1, 500, 10), (30, 1, 6000, 1), (40, 49, 256, 32), (512, 196, 64, 4), (20, 9, 125, 5),
                                   (3, 5000, 130, 2), (2, 7001, 24, 3)])
def test_group_norm(shape, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.randn(n, S, C, device="cuda").to(dt)
    y, m, r = ff.group_norm_act(x, None, None, G)
    dx, _, _ = ff.group_norm_act_backward(x, x, m, r, None, None, G)
    near = lambda a, b: torch.allclose(a.float(), b.float(), rtol=2.0 ** -7 if dtype == "bf16" else 1e-5, atol=1e-4)
    for pad, lead in GAPS:
        buf, out = inside(torch, (n, S, C), dt, pad, lead)
        assert ff.group_norm_act(x, None, None, G, out=out)[0] is out
        assert near(out, y) and untouched(buf, out)
        assert ff.group_norm_act_backward(x, x, m, r, None, None, G, out=out)[0] is out
        assert near(out, dx) and untouched(buf, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(1, 1), (3, 5), (128, 500), (64, 2048), (4001, 31), (7, 1999), (300, 777)])
def test_dropout(size, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, res = torch.randn(*size, device="cuda").to(dt), torch.randn(*size, device="cuda").to(dt)
    for r in (None, res):
        want = ff.dropout(x, 0.4, 9, 17, residual=r)
        for pad, lead in GAPS:
            buf, out = inside(torch, size, dt, pad, lead)
            assert ff.dropout(x, 0.4, 9, 17, residual=r, out=out) is out
            assert torch.equal(out, want) and untouched(buf, out)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(1, 2000, 784), (20, 1999, 500), (100, 3001, 2000), (700, 701, 8000), (2055, 2001, 300),
                                  (2048, 2004, 300), (2500, 4302, 200)])
def test_matmul(size, dtype):
    """Few rows and many: rows that end inside a 16-byte unit, at strides that are whole units and not."""
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = size
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    a, b = ff.fp8_quantize(torch.randn(m, k, device="cuda")), ff.fp8_quantize(torch.randn(n, k, device="cuda"), tile=True)
    want = ff.fp8_matmul(a, b, out_dtype=dt)
    for pad, lead in GAPS + ((-n % 8, 8), (8 + -n % 8, 0), (-n % 4, 4)):
        buf, out = inside(torch, (m, n), dt, pad, lead)
        assert ff.fp8_matmul(a, b, out=out) is out
        assert torch.equal(out, want) and untouched(buf, out)
