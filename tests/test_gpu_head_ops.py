"""The operators of a deep head: calls on other streams, without autograd, past
2^31 elements, at sizes that reach every kernel, and both outputs of a norm."""

import ctypes
import warnings

import pytest

from .gpu_common import lib_ready, torch_cuda
from .test_gpu_fp8_paths import launched
from .test_gpu_streams import check, inputs

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def test_streams():
    torch = torch_cuda()
    ff = lib_ready()
    for rows, cols in ((700, 500), (300, 20000)):
        x, r, g = inputs(torch, rows, cols), inputs(torch, rows, cols, seed=1), inputs(torch, cols, seed=2)
        y, h, rstd = ff.rms_norm(x, g, residual=r)
        need = ff.lib().ff_rms_norm_workspace(rows, cols)
        check(lambda s: ff.rms_norm(x, g, residual=r, stream=s))
        check(lambda s: ff.rms_norm_fp8(x, g, stream=s)[::2])
        check(lambda s: ff.rms_norm_backward(y, h, rstd, g, dh=x, stream=s), [need])
    labels = torch.zeros(300, dtype=torch.int32, device="cuda")
    logits = inputs(torch, 300, 5000)
    p = ff.label_logprobs(logits, labels, top=4)
    check(lambda s: [getattr(ff.label_logprobs(logits, labels, top=4, stream=s), n) for n in ff.LabelLogprobs.__slots__])
    check(lambda s: ff.label_logprobs_backward(logits, labels, p.stats, p.logp, stream=s))
    grads = [inputs(torch, 700, 500), inputs(torch, 3_000_000, seed=1)]
    into = [torch.empty_like(g) for g in grads]
    need = ff.lib().ff_clip_grad_norm_workspace(2)
    check(lambda s: ff.clip_grad_norm(grads, 1.0, out=into, stream=s), [need])
    x = inputs(torch, 500, 784)
    a, b = ff.fp4_quantize(x), ff.fp4_quantize(inputs(torch, 300, 784, seed=1))
    check(lambda s: ff.fp4_quantize_both(x, stream=s))
    check(lambda s: ff.fp4_dequantize(a, stream=s))
    check(lambda s: ff.fp4_matmul(a, b, out_dtype=torch.float32, stream=s))


def test_a_lost_gradient_is_not_silent():
    torch = torch_cuda()
    ff = lib_ready()
    x, g = torch.randn(8, 32, device="cuda"), torch.ones(32, device="cuda", requires_grad=True)
    p, bias = x.clone().requires_grad_(), torch.zeros(8, device="cuda", requires_grad=True)
    a = ff.fp4_quantize(x)
    calls = [lambda: ff.rms_norm(p, None)[0], lambda: ff.rms_norm(x, g)[0], lambda: ff.rms_norm(x, None, residual=p)[0],
             lambda: ff.rms_norm_fp8(p, None)[0].scale, lambda: ff.label_logprobs(p, None).entropy, lambda: ff.fp4_quantize(p).q,
             lambda: ff.fp4_quantize_both(p)[0].q, lambda: ff.fp4_matmul(a, a, bias=bias)]
    for call in calls:
        with pytest.warns(UserWarning, match="not recorded by autograd") as seen:
            first = call()
        assert "test_gpu_head_ops" in seen[0].filename
        with torch.no_grad(), warnings.catch_warnings():
            warnings.simplefilter("error")
            assert torch.equal(call(), first)


def values(ff, m):
    import torch
    return ff.fp4_dequantize(m, out_dtype=torch.float32).double()


KINDS = {"fp4_gemm_tc", "fp4_gemm_pair_tc"}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size,kind", [((2501, 4303, 700), "fp4_gemm_pair_tc"), ((2504, 8304, 700), "fp4_gemm_pair_tc"),
                                       ((1846, 1127, 2259), "fp4_gemm_pair_tc"), ((1848, 1128, 2304), "fp4_gemm_pair_tc"),
                                       ((4000, 10, 2000), "fp4_gemm_tc"), ((3000, 30, 800), "fp4_gemm_tc"), ((5, 3000, 5000), "fp4_gemm_tc"),
                                       ((30, 700, 5000), "fp4_gemm_tc"), ((60, 900, 5000), "fp4_gemm_tc")])
def test_product_kernels_with_several_tiles(size, kind, dtype):
    """Pairs that take several tiles of several stages, both tile widths, both ways of storing, and split products each
    way round; the tolerance is test_gpu_fp4.py's."""
    torch = torch_cuda()
    ff = lib_ready()
    m, n, k = size
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    a, b = ff.fp4_quantize(inputs(torch, m, k)), ff.fp4_quantize(inputs(torch, n, k, seed=1))
    bias = inputs(torch, n, seed=2)
    c, kinds = launched(ff, lambda: ff.fp4_matmul(a, b, bias=bias, out_dtype=dt))
    assert {v for v in kinds if v in KINDS} == {kind}
    A, B = values(ff, a), values(ff, b).t()
    want = A @ B + bias.double()
    tol = 2 * U * ((k + 12) * (A.abs() @ B.abs()) + want.abs() + bias.double().abs()) + want.abs() * torch.finfo(dt).eps / 2
    assert bool(((c.double() - want).abs() <= tol).all())


def test_a_norm_with_both_outputs():
    """The C entry gives y and its 8-bit blocks from one call, the same as one by one."""
    torch = torch_cuda()
    ff = lib_ready()
    for cols in (300, 33000):
        x, g = inputs(torch, 9, cols).bfloat16(), inputs(torch, cols, seed=1)
        y, _, rstd = ff.rms_norm(x, g)
        a, _, _ = ff.rms_norm_fp8(x, g)
        y2, r2, q2, s2 = torch.empty_like(y), torch.empty_like(rstd), torch.empty_like(a.q), torch.empty_like(a.scale)
        assert ff.lib().ff_rms_norm(x.data_ptr(), cols, None, 0, 9, cols, g.data_ptr(), 1e-5, 1, None, 0, y2.data_ptr(), cols,
                                    q2.data_ptr(), s2.data_ptr(), r2.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(y, y2) and torch.equal(rstd, r2) and torch.equal(a.q.view(torch.uint8), q2.view(torch.uint8))
        assert torch.equal(a.scale, s2)


def test_gradients_without_one_of_their_outputs():
    torch = torch_cuda()
    ff = lib_ready()
    L = ff.lib()
    for rows, cols in ((50, 300), (700, 600), (20, 20000)):
        h, dy = inputs(torch, rows, cols), inputs(torch, rows, cols, seed=1)
        _, _, rstd = ff.rms_norm(h, None)
        dx, dgamma = ff.rms_norm_backward(dy, h, rstd, None)
        need = L.ff_rms_norm_workspace(rows, cols)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        s = torch.cuda.current_stream().cuda_stream
        one, two = torch.empty_like(dx), torch.empty_like(dgamma)
        args = (dy.data_ptr(), cols, h.data_ptr(), cols, rows, cols, rstd.data_ptr(), None, None, 0, 0)
        assert L.ff_rms_norm_backward(*args, one.data_ptr(), cols, None, ws.data_ptr(), need, s) == 0
        assert L.ff_rms_norm_backward(*args, None, 0, two.data_ptr(), ws.data_ptr(), need, s) == 0
        assert torch.equal(one, dx) and torch.equal(two, dgamma)


def big(torch, rows, cols, seed):
    return torch.randn(rows, cols, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", dtype=torch.bfloat16)


def test_past_2_31_elements():
    """Rows from beyond the 2^31st element, against the same rows alone (whose kernels may add in another order)."""
    torch = torch_cuda()
    ff = lib_ready()
    rows, cols = 270000, 8192  # 2.2e9 values
    x = big(torch, rows, cols, 1)
    some = torch.tensor([0, 1, 131072, 262143, 262144, 262145, rows - 1], device="cuda")
    part = x[some].contiguous()
    near = lambda a, b: torch.allclose(a.float(), b.float(), rtol=2.0 ** -7, atol=1e-5)
    y, _, rstd = ff.rms_norm(x, None, residual=x)
    y2, _, rstd2 = ff.rms_norm(part, None, residual=part)
    assert near(y[some], y2) and near(rstd[some], rstd2)
    del y
    a, _, _ = ff.rms_norm_fp8(x, None)
    b, _, _ = ff.rms_norm_fp8(part, None)
    assert near(a.scale[:, some], b.scale) and bool(((a.q[some].float() - b.q.float()).abs() <= 32).all())
    del a
    _, _, rstd = ff.rms_norm(x, None)
    dx, dgamma = ff.rms_norm_backward(x, x, rstd, None)
    dx2, _ = ff.rms_norm_backward(part, part, rstd[some].contiguous(), None)
    assert near(dx[some], dx2)
    # dgamma = sum dy n = rstd sum x^2, all terms positive: 128 in a row, then partial sums
    want = torch.zeros(cols, dtype=torch.float64, device="cuda")
    for i in range(0, rows, 30000):
        want += (x[i:i + 30000].double().square() * rstd[i:i + 30000].double()[:, None]).sum(0)
    assert bool(((dgamma.double() - want).abs() <= (128 + rows // 4096 + 35) * U * want).all())
    del dx
    labels = torch.randint(0, cols, (rows,), dtype=torch.int32, device="cuda")
    r, r2 = ff.label_logprobs(x, labels, top=3), ff.label_logprobs(part, labels[some].contiguous(), top=3)
    assert torch.equal(r.top_index[some], r2.top_index) and torch.allclose(r.logp[some], r2.logp, rtol=1e-5)
    d = ff.label_logprobs_backward(x, labels, r.stats, r.logp)
    d2 = ff.label_logprobs_backward(part, labels[some].contiguous(), r2.stats, r2.logp)
    assert torch.allclose(d[some].float(), d2.float(), rtol=2.0 ** -7, atol=1e-6)
    del d
    q, qt = ff.fp4_quantize_both(x)
    p = ff.fp4_quantize(part)
    assert torch.equal(q.q[some], p.q) and torch.equal(ff.fp4_dequantize(q)[some], ff.fp4_dequantize(p))
    last = x[rows - rows % 32 - 32:].contiguous()  # whole blocks of 32 rows at the end, transposed
    end = ff.fp4_quantize(last, transpose=True)
    assert torch.equal(qt.q[:, -end.q.shape[1]:], end.q)
    w = ff.fp4_quantize(big(torch, 8192, cols, 2))
    c = ff.fp4_matmul(q, w)  # 2.2e9 results
    c2 = ff.fp4_matmul(p, w)
    assert torch.allclose(c[some].float(), c2.float(), rtol=2.0 ** -7, atol=0.05)
    del c, q, qt
    flat, exact = x.view(-1), 0.0
    for i in range(0, flat.numel(), 1 << 28):
        exact += float(flat[i:i + (1 << 28)].double().square().sum())
    ends = [flat[:1000].double(), flat[-1000:].double()]
    norm = ff.clip_grad_norm([flat], 1.0)
    assert abs(float(norm) - exact ** 0.5) <= 20 * U * exact ** 0.5
    for got, was in zip((flat[:1000], flat[-1000:]), ends):
        want = was / exact ** 0.5
        assert bool(((got.double() - want).abs() <= want.abs() * (2.0 ** -8 + 22 * U)).all())
