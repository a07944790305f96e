"""The layer operators are outside autograd, and say so where it would record a call."""

import warnings

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu


def test_a_lost_gradient_is_not_silent():
    torch = torch_cuda()
    ff = lib_ready()
    x, w = torch.randn(8, 32, device="cuda"), torch.randn(16, 32, device="cuda")
    p = x.clone().requires_grad_()
    g, bias = torch.ones(32, device="cuda", requires_grad=True), torch.zeros(16, device="cuda", requires_grad=True)
    a, b = ff.fp8_quantize(x), ff.fp8_quantize(w, tile=True)
    calls = [lambda: ff.group_norm_act(p, None, None, 4)[0], lambda: ff.group_norm_act(x, g, None, 4)[0],
             lambda: ff.dropout(p, 0.5, 1), lambda: ff.dropout(x, 0.5, 1, residual=p), lambda: ff.fp8_quantize(p).scale,
             lambda: ff.fp8_quantize_both(p)[0].scale, lambda: ff.fp8_matmul(a, b, bias=bias)]
    for call in calls:
        with pytest.warns(UserWarning, match="not recorded by autograd") as seen:
            first = call()
        assert seen[0].filename == __file__ or "test_gpu_autograd" in seen[0].filename
        with torch.no_grad(), warnings.catch_warnings():
            warnings.simplefilter("error")
            assert torch.equal(call(), first)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        ff.group_norm_act(x, g.detach(), None, 4)
        ff.fp8_matmul(a, b)
