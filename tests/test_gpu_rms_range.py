"""RMS norm and its gradient on rows whose squares fp32 cannot hold, against the
definition in 64 bits.

Tolerances as for ordinary rows: u = 2^-24, a row's sum of squares within
(chain + 1) u of itself, rstd within half of that and three roundings (and where
it is below 2^-126, half a multiple of 2^-149), an output two roundings and the half
step of its type (torch.finfo(t).eps / 2).
"""

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
COLS = [7, 500, 2001, 8192, 12000, 40000]


def rows_of(torch, cols, scale, dt, seed):
    """Five rows: ordinary, of the scale, of the scale at one place, ordinary, of half of the scale."""
    t = torch.randn(5, cols, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).clamp(-3.5, 3.5) / 4.0
    t[1] *= scale
    t[2, cols // 2] = scale * 0.875
    t[4] *= scale * 0.5
    return t.to(torch.float32).to(dt).cuda()


def chain(cols):
    return 24 + cols // 4096


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [2.0 ** 58, 2.0 ** 62, 2.0 ** 63, 1e30, 2.0 ** 127])
@pytest.mark.parametrize("cols", COLS)
def test_forward(cols, scale, dtype, residual):
    torch = torch_cuda()
    ff = lib_ready()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = rows_of(torch, cols, scale, dt, 1)
    r = x.flip(1).contiguous() * 0.0625 if residual else None
    gamma = torch.randn(cols, generator=torch.Generator().manual_seed(2)).cuda()
    y, h, rstd = ff.rms_norm(x, gamma, residual=r, eps=1e-3)
    h64 = ((x.float() + r.float()).to(dt) if residual else x).double()
    assert torch.equal(h.double(), h64) and bool(h64.isfinite().all())
    exact = (h64.square().mean(1) + 1e-3) ** -0.5
    e = (chain(cols) / 2 + 4) * U + 2.0 ** -149 / exact
    assert bool(((rstd.double() - exact).abs() <= e * exact).all())
    want = h64 * (exact[:, None] * gamma.double())
    tol = want.abs() * (e[:, None] + 2 * U + torch.finfo(dt).eps / 2) + 2.0 ** -130
    assert bool(((y.double() - want).abs() <= tol).all())
    a, h8, rstd8 = ff.rms_norm_fp8(x, gamma, residual=r, eps=1e-3)
    assert torch.equal(rstd8, rstd) and torch.equal(h8, h)
    kb = -(-cols // 128)
    full = torch.zeros(5, kb * 128, dtype=torch.float64, device="cuda")
    full[:, :cols] = want.abs()
    scales = (full.view(5, kb, 128).amax(2) / 448).clamp(min=2.0 ** -126)
    assert bool(((a.scale.t().double() - scales).abs() <= (e[:, None] + 4 * U) * scales).all())
    per = a.scale.t().double().repeat_interleave(128, 1)[:, :cols]
    tol = want.abs() * (2.0 ** -4 + e[:, None] + 6 * U) + per * 2.0 ** -10
    assert bool(((a.q.double()[:, :cols] * per - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("h_scale,dy_scale", [(2.0 ** 58, 1.0), (2.0 ** 62, 2.0 ** 70), (2.0 ** 100, 1.0), (2.0 ** 100, 2.0 ** 60),
                                              (2.0 ** 40, 2.0 ** 100), (2.0 ** -30, 2.0 ** 90)])
@pytest.mark.parametrize("cols", COLS + [20000])
def test_backward(cols, h_scale, dy_scale, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    h = rows_of(torch, cols, h_scale, dt, 1)
    gen = torch.Generator().manual_seed(3)
    dy = (torch.randn(5, cols, generator=gen, dtype=torch.float64) * dy_scale).to(torch.float32).to(dt).cuda()
    gamma = torch.randn(cols, generator=gen).cuda()
    _, _, rstd = ff.rms_norm(h, gamma)
    for joined in (None, rows_of(torch, cols, dy_scale / h_scale, dt, 4)):
        dx, dgamma = ff.rms_norm_backward(dy, h, rstd, gamma, dh=joined)
        r = rstd.double()[:, None]
        n, du = h.double() * r, dy.double() * gamma.double()
        mean, mean_abs = (du * n).mean(1, keepdim=True), (du * n).abs().mean(1, keepdim=True)
        want = r * (du - n * mean) + (0.0 if joined is None else joined.double())
        tol = U * r * (8 * du.abs() + n.abs() * mean_abs * (chain(cols) + 16)) + want.abs() * (2 * U + torch.finfo(dt).eps / 2)
        assert bool(((dx.double() - want).abs() <= tol + 2.0 ** -130).all())
        terms = dy.double() * n
        assert bool(((dgamma.double() - terms.sum(0)).abs() <= 20 * U * terms.abs().sum(0) + 2.0 ** -140).all())


@pytest.mark.parametrize("cols", [500, 2001, 8192, 40000])
def test_in_place(cols):
    """Rows past fp32's range are read again after their residual's sum is written, and before their output is."""
    torch = torch_cuda()
    ff = lib_ready()
    gamma = torch.randn(cols, generator=torch.Generator().manual_seed(2)).cuda()
    for dt in (torch.bfloat16, torch.float32):
        x = rows_of(torch, cols, 2.0 ** 80, dt, 1)
        r = x.flip(1).contiguous() * 0.0625
        y, _, rstd = ff.rms_norm(x, gamma)
        a = x.clone()
        assert torch.equal(ff.rms_norm(a, gamma, out=a)[2], rstd) and torch.equal(a, y)
        y, h, rstd = ff.rms_norm(x, gamma, residual=r)
        a, b = x.clone(), r.clone()
        ff.rms_norm(a, gamma, residual=b, out=a, h=b)
        assert torch.equal(a, y) and torch.equal(b, h)
        a, b = x.clone(), r.clone()
        ff.rms_norm(a, gamma, residual=b, out=b, h=a)
        assert torch.equal(b, y) and torch.equal(a, h)
        graph, a = torch.cuda.CUDAGraph(), torch.zeros_like(x)
        with torch.cuda.graph(graph):
            held = ff.rms_norm(a, gamma, residual=r)
        a.copy_(x)
        graph.replay()
        assert torch.equal(held[0], y) and torch.equal(held[1], h) and torch.equal(held[2], rstd)
