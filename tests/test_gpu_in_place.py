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
