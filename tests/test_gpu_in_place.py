"""Operator calls that write a caller's tensors: what they return, and what
autograd knows of it."""

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu


def test_a_norm_over_its_own_input_hands_back_no_input():
    """Its gradient needs the input, which the output has replaced: it is not returned as if it were still there."""
    torch = torch_cuda()
    ff = lib_ready()
    for shape in ((6, 300), (2, 3, 300), (1, 33000)):
        x = torch.randn(*shape, device="cuda")
        want, h, rstd = ff.rms_norm(x, None)
        assert h is x
        buf = x.clone()
        y, h, again = ff.rms_norm(buf, None, out=buf)
        assert y is buf and h is None and torch.equal(y, want) and torch.equal(again, rstd)
        with pytest.raises(ValueError, match="h must match"):
            ff.rms_norm_backward(y, h, again, None)
        view = x.clone()
        y, h, _ = ff.rms_norm(view, None, out=view.view(shape))
        assert h is None and torch.equal(y, want)
        empty = torch.empty(0, shape[-1], device="cuda")
        assert ff.rms_norm(empty, None, out=torch.empty_like(empty))[1] is empty
        # with a residual h has a buffer of its own, whatever out is
        r = torch.randn(*shape, device="cuda")
        want, kept, _ = ff.rms_norm(x, None, residual=r)
        buf = x.clone()
        y, h, _ = ff.rms_norm(buf, None, residual=r, out=buf)
        assert torch.equal(y, want) and torch.equal(h, kept)


def test_a_backward_pass_over_overwritten_values_is_refused():
    """Autograd saves x for the gradient of w; a call that then writes x is not to go unnoticed."""
    torch = torch_cuda()
    ff = lib_ready()
    gen = torch.Generator().manual_seed(0)
    x, r, dy = (torch.randn(64, 128, generator=gen).cuda() for _ in range(3))
    one, labels = torch.ones(128, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    _, _, rstd = ff.rms_norm(x, None)
    p = ff.label_logprobs(x, labels)
    q8, q4 = ff.fp8_quantize(x), ff.fp4_quantize(x)
    wide = torch.randn(64, 64, generator=gen).cuda()
    _, mean, rs = ff.group_norm_act(x, one, one, 4)
    mean0 = mean.clone()
    calls = {
        "rms_norm": (x, lambda t: ff.rms_norm(x, None, out=t)), "rms_norm h": (x, lambda t: ff.rms_norm(x, None, residual=r, h=t)),
        "rms_norm_fp8 h": (x, lambda t: ff.rms_norm_fp8(x, None, residual=r, h=t)),
        "rms_norm_backward": (x, lambda t: ff.rms_norm_backward(dy, x, rstd, None, out=t)),
        "label_logprobs_backward": (x, lambda t: ff.label_logprobs_backward(x, labels, p.stats, p.logp, out=t)),
        "clip in place": (x, lambda t: ff.clip_grad_norm([r.clone(), t], 1.0)),
        "clip": (x, lambda t: ff.clip_grad_norm([x], 1.0, out=[t])),
        "fp4_dequantize": (x, lambda t: ff.fp4_dequantize(q4, out=t)), "fp4_matmul": (wide, lambda t: ff.fp4_matmul(q4, q4, out=t)),
        "fp8_matmul": (wide, lambda t: ff.fp8_matmul(q8, q8, out=t)), "dropout": (x, lambda t: ff.dropout(x, 0.5, 1, out=t)),
        "group_norm_act": (x, lambda t: ff.group_norm_act(x, one, one, 4, out=t)),
        "group_norm_act mean": (mean0, lambda t: ff.group_norm_act(x, one, one, 4, mean=t)),
        "group_norm_act_backward": (x, lambda t: ff.group_norm_act_backward(dy, x, mean, rs, one, one, 4, out=t)),
    }
    for name, (like, call) in calls.items():
        saved, w = like.clone(), torch.ones_like(like).requires_grad_()
        loss = (w * saved).sum()
        call(saved)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        # a buffer that nothing waits for, and one of inference mode, are written as ever
        with torch.inference_mode():
            call(torch.empty_like(like).copy_(like))
        saved = like.clone()
        loss = (w * like).sum()
        call(saved)
        loss.backward()
        assert torch.equal(w.grad, like), name
