"""Group norm at the sizes where a 32-bit count of samples or positions runs out."""

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
MOST = (1 << 31) - 1


def test_2_31_less_one_samples():
    """Rows: a warp's walk over the samples ends at the last one.  Outputs,
    statistics and gradients of the last samples against those samples alone;
    every output is written."""
    torch = torch_cuda()
    ff = lib_ready()
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(MOST, 2, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    y = torch.full_like(x, float("nan"))
    _, m, r = ff.group_norm_act(x, None, None, 1, act="none", out=y)
    tail = x[-5000:].clone()
    y1, m1, r1 = ff.group_norm_act(tail, None, None, 1, act="none")
    assert torch.equal(y[-5000:], y1) and torch.equal(m[-5000:], m1) and torch.equal(r[-5000:], r1)
    assert not torch.isnan(y).any()
    dy = torch.zeros_like(x)
    dy[-5000:].normal_(generator=gen)
    y.fill_(float("nan"))
    dx, dg, db = ff.group_norm_act_backward(dy, x, m, r, None, None, 1, act="none", out=y)
    dx1, dg1, db1 = ff.group_norm_act_backward(dy[-5000:].clone(), tail, m1, r1, None, None, 1, act="none")
    assert torch.equal(dx[-5000:], dx1) and not torch.isnan(dx).any()
    # all other terms are zero; the sums may have another order
    size = dy[-5000:].float().abs().sum()
    assert torch.all((db - db1).abs() <= 2.0 ** -17 * size) and torch.all((dg - dg1).abs() <= 2.0 ** -17 * size)


def test_2_31_less_one_positions():
    """Column passes: the last chunk of a sample's positions.  The statistics
    and outputs against 64 bits (|x| of order 1, so that the mean errs by at
    most 64 units of 2^-24 and an output by that and its rounding, 2^-8 of
    itself); the gradient's sums of a dy that is not zero at the end only."""
    torch = torch_cuda()
    ff = lib_ready()
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty(1, MOST, 1, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    y = torch.full_like(x, float("nan"))
    _, m, r = ff.group_norm_act(x, None, None, 1, act="none", out=y)
    x64 = x.double()
    mean = x64.mean()
    rstd = ((x64 - mean).square_().mean() + 1e-5) ** -0.5
    del x64
    assert abs(float(m) - float(mean)) <= 2.0 ** -18 and abs(float(r) - float(rstd)) <= 2.0 ** -18
    assert not torch.isnan(y).any()
    want = (x[:, -40000:].double() - mean) * rstd
    assert torch.all((y[:, -40000:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -17)
    dy = torch.zeros_like(x)
    dy[:, -20000:] = 1
    y.fill_(float("nan"))
    dx, dg, db = ff.group_norm_act_backward(dy, x, m, r, None, None, 1, act="none", out=y)
    h = (x[:, -20000:].double() - float(m)) * float(r)
    assert float(db) == 20000
    assert abs(float(dg) - float(h.sum())) <= 2.0 ** -17 * float(h.abs().sum())
    assert not torch.isnan(dx).any()
    want = float(r) * (1 - 20000 / MOST - h * float(dg) / MOST)
    assert torch.all((dx[:, -20000:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -17)
