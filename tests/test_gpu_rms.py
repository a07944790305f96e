"""RMS norm with the residual's addition, in either type and as e4m3 blocks, and
its gradient, against the definition in 64 bits.

Tolerances.  u = 2^-24 is a rounding to fp32.  A row's sum of squares adds
positive terms: a lane's units, then shuffles over lanes and warps, at most
`chain` additions deep, so it is within (chain + 1) u of itself, and rstd within
half of that and three roundings.  An output adds two roundings and the half
step of its type (torch.finfo(t).eps / 2).
"""

import numpy as np
import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [(1, 1), (1, 2000), (3, 7), (5, 128), (2, 129), (300, 500), (33, 1024), (9, 1025), (700, 4097), (2432, 1024), (40, 8192),
         (1300, 2000), (3, 32768), (2, 32769), (4, 40000), (20000, 16)]


def half_step(torch, dt):
    return torch.finfo(dt).eps / 2


def chain(cols):
    return 24 + cols // 4096


def data(torch, rows, cols, dt, pad, lead, seed):
    """[rows, cols] in rows that lie cols + pad apart, `lead` elements into its buffer."""
    gen = torch.Generator().manual_seed(seed)
    t = torch.randn(rows, cols, generator=gen) * torch.exp(torch.randn(rows, 1, generator=gen))
    buf = torch.full((lead + rows * (cols + pad),), float("nan"), dtype=dt, device="cuda")
    view = buf[lead:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


def layout(i):
    return ((0, 0), (8, 8), (3, 1), (0, 0), (2, 2), (4, 4))[i % 6]


def gamma_of(torch, cols, i):
    return None if i % 5 == 4 else torch.randn(cols, generator=torch.Generator().manual_seed(i)).cuda()


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES)
def test_forward(size, dtype, residual):
    torch = torch_cuda()
    ff = lib_ready()
    rows, cols = size
    i = SIZES.index(size)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = data(torch, rows, cols, dt, *layout(i), seed=i)
    r = data(torch, rows, cols, dt, *layout(i + (i % 2)), seed=50 + i) if residual else None
    gamma = gamma_of(torch, cols, i)
    y, h, rstd = ff.rms_norm(x, gamma, residual=r, eps=1e-3)
    h64 = ((x.float() + r.float()).to(dt) if residual else x).double()
    assert h is x if not residual else torch.equal(h.double(), h64)
    exact = (h64.square().mean(1) + 1e-3) ** -0.5
    e_rstd = (chain(cols) / 2 + 4) * U
    assert bool(((rstd.double() - exact).abs() <= e_rstd * exact).all())
    want = h64 * exact[:, None] * (1.0 if gamma is None else gamma.double())
    tol = want.abs() * (e_rstd + 2 * U + half_step(torch, dt)) + 2.0 ** -130
    assert y.shape == x.shape and y.dtype == dt and bool(((y.double() - want).abs() <= tol).all())
    # 8 bits
    a, h8, rstd8 = ff.rms_norm_fp8(x, gamma, residual=r, eps=1e-3)
    assert torch.equal(rstd8, rstd) and torch.equal(h8, h)
    kb = -(-cols // 128)
    full = torch.zeros(rows, kb * 128, dtype=torch.float64, device="cuda")
    full[:, :cols] = want.abs()
    scale = (full.view(rows, kb, 128).amax(2) / 448).clamp(min=2.0 ** -126)
    assert bool(((a.scale.t().double() - scale).abs() <= (e_rstd + 4 * U) * scale).all())
    q = a.q.double()
    assert q.shape == (rows, -(-cols // 16) * 16) and bool((q[:, cols:] == 0).all())
    per = a.scale.t().double().repeat_interleave(128, 1)[:, :cols]
    # e4m3: half a step is 2^-4 of the value, 2^-10 of the scale below the normal range; x * (1 / scale) rounds three times
    tol = want.abs() * (2.0 ** -4 + e_rstd + 6 * U) + per * 2.0 ** -10
    assert bool(((q[:, :cols] * per - want).abs() <= tol).all())


@pytest.mark.parametrize("joined", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES + [(3000, 100), (200, 16385), (1, 16400)])
def test_backward(size, dtype, joined):
    torch = torch_cuda()
    ff = lib_ready()
    rows, cols = size
    i = (SIZES + [(3000, 100), (200, 16385), (1, 16400)]).index(size)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    h = data(torch, rows, cols, dt, *layout(i), seed=i)
    dy = data(torch, rows, cols, dt, *layout(i + 2 * (i % 2)), seed=100 + i)
    dh = data(torch, rows, cols, dt, *layout(i), seed=200 + i) if joined else None
    gamma = gamma_of(torch, cols, i)
    _, _, rstd = ff.rms_norm(h, gamma)
    dx, dgamma = ff.rms_norm_backward(dy, h, rstd, gamma, dh=dh)
    r = rstd.double()[:, None]
    n, du = h.double() * r, dy.double() * (1.0 if gamma is None else gamma.double())
    mean, mean_abs = (du * n).mean(1, keepdim=True), (du * n).abs().mean(1, keepdim=True)
    want = r * (du - n * mean) + (dh.double() if joined else 0.0)
    tol = U * r * (8 * du.abs() + n.abs() * mean_abs * (chain(cols) + 16)) + want.abs() * (2 * U + half_step(torch, dt))
    assert bool(((dx.double() - want).abs() <= tol + 2.0 ** -130).all())
    terms = dy.double() * n
    # up to 128 rows one after the other, then at most rows / 128 / 32 partials one after the other and a tree
    depth = 128 + rows // 4096 + 32
    assert bool(((dgamma.double() - terms.sum(0)).abs() <= (depth + 3) * U * terms.abs().sum(0) + 2.0 ** -140).all())
    again = ff.rms_norm_backward(dy, h, rstd, gamma, dh=dh)
    assert torch.equal(dx, again[0]) and torch.equal(dgamma, again[1])


def test_gradient_follows_differences():
    """The central difference of sum(y w) + sum(h v) in 64 bits, of the formula the kernels are held to above."""
    torch = torch_cuda()
    ff = lib_ready()
    gen = torch.Generator().manual_seed(3)
    x, res, w, v = (torch.randn(6, 40, generator=gen).cuda() for _ in range(4))
    gamma = torch.randn(40, generator=gen).cuda()
    y, h, rstd = ff.rms_norm(x, gamma, residual=res)
    dx, dgamma = ff.rms_norm_backward(w, h, rstd, gamma, dh=v)

    def loss(x64, g64):
        h64 = x64 + res.double()
        return ((h64 * (h64.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * g64) * w.double()).sum() + (h64 * v.double()).sum()

    step = 1e-5
    for which, grad in ((0, dx), (1, dgamma)):
        base = [x.double(), gamma.double()]
        for k in (0, 7, 33):
            hi, lo = [b.clone() for b in base], [b.clone() for b in base]
            hi[which].view(-1)[k] += step
            lo[which].view(-1)[k] -= step
            slope = float(loss(*hi) - loss(*lo)) / (2 * step)
            # difference error step^2 and 64-bit cancellation are below 1e-8; fp32 sums of 40 and rounded inputs below 1e-5
            assert abs(slope - float(grad.view(-1)[k])) <= 1e-4 * (1 + abs(slope))


@pytest.mark.parametrize("cols", [500, 1999, 33000])
def test_in_place_and_inside_larger_buffers(cols):
    torch = torch_cuda()
    ff = lib_ready()
    rows = 37
    x, r = (data(torch, rows, cols, torch.bfloat16, 0, 0, s) for s in (1, 2))
    gamma = gamma_of(torch, cols, 1)
    y, h, rstd = ff.rms_norm(x, gamma, residual=r)
    a, b = x.clone(), r.clone()
    y2, h2, _ = ff.rms_norm(a, gamma, residual=b, out=a, h=b)
    assert y2 is a and h2 is b and torch.equal(a, y) and torch.equal(b, h)
    a, b = x.clone(), r.clone()
    ff.rms_norm(a, gamma, residual=b, out=b, h=a)
    assert torch.equal(b, y) and torch.equal(a, h)
    dy = data(torch, rows, cols, torch.bfloat16, 0, 0, 3)
    dx, dg = ff.rms_norm_backward(dy, h, rstd, gamma, dh=y)
    for which in range(3):
        d, k, e = dy.clone(), h.clone(), y.clone()
        into = (d, k, e)[which]
        got, dg2 = ff.rms_norm_backward(d, k, rstd, gamma, dh=e, out=into)
        assert got is into and torch.equal(into, dx) and torch.equal(dg, dg2)
    for pad, lead in ((5, 3), (8, 8), (2, 2)):
        bufs = [torch.full((lead + rows * (cols + pad) + 64,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        views = [t[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] for t in bufs]
        ff.rms_norm(x, gamma, residual=r, out=views[0], h=views[1])
        ff.rms_norm_backward(dy, h, rstd, gamma, dh=y, out=views[2])
        # rows alike but for the order of a row's sum, which the alignment may change: half a step of bf16 each
        for view, want in zip(views, (y, h, dx)):
            assert torch.allclose(view.float(), want.float(), rtol=2.0 ** -7, atol=1e-6)
            view.fill_(7.0)
        assert all(bool((t == 7.0).all()) for t in bufs)


def test_matrices_side_by_side_in_one_buffer():
    torch = torch_cuda()
    ff = lib_ready()
    cols = 500
    x, r, dy = (data(torch, 37, cols, torch.bfloat16, 0, 0, s) for s in (1, 2, 3))
    gamma = gamma_of(torch, cols, 1)
    y, h, rstd = ff.rms_norm(x, gamma, residual=r)
    wide = torch.zeros(37, 4 * cols, dtype=torch.bfloat16, device="cuda")
    a, b, c, d = (wide[:, i * cols:(i + 1) * cols] for i in range(4))
    a.copy_(x), b.copy_(r)
    ff.rms_norm(a, gamma, residual=b, out=d, h=c)
    assert torch.equal(c, h) and torch.equal(d, y) and torch.equal(a, x) and torch.equal(b, r)
    dx, dg = ff.rms_norm_backward(dy, h, rstd, gamma)
    a.copy_(dy)
    assert ff.rms_norm_backward(a, c, rstd, gamma, out=b)[0] is b and torch.equal(b, dx) and torch.equal(c, h)
    with pytest.raises(ff.FFError):
        ff.rms_norm(a, gamma, out=wide[:, 4:cols + 4])


@pytest.mark.parametrize("size", [(5, 1), (37, 129), (900, 301), (170, 4097), (2000, 2001), (40, 9001), (3, 15999), (700, 7)])
def test_gradient_of_odd_rows_at_every_offset(size):
    """Rows of single bf16 values that start anywhere: the same bits, whatever lies around them."""
    torch = torch_cuda()
    ff = lib_ready()
    rows, cols = size
    gamma = gamma_of(torch, cols, 1)
    dy, h, dh = (data(torch, rows, cols, torch.bfloat16, 0, 0, s) for s in (1, 2, 3))
    rstd = torch.rand(rows, generator=torch.Generator().manual_seed(4)).cuda() + 0.5

    def at(t, pad, lead):
        buf = torch.full((lead + rows * (cols + pad) + 3,), float("nan"), dtype=torch.bfloat16, device="cuda")
        view = buf[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        view.copy_(t)
        return view

    for joined in (dh, None):
        dx, dg = ff.rms_norm_backward(dy, h, rstd, gamma, dh=joined)
        for k, (pads, leads) in enumerate((((0, 0, 0), (1, 1, 1)), ((1, 3, 0), (1, 0, 3)), ((2, 1, 5), (0, 1, 2)), ((0, 4, 1), (3, 5, 0)))):
            a, b = at(dy, pads[0], leads[0]), at(h, pads[1], leads[1])
            c = None if joined is None else at(dh, pads[2], leads[2])
            got, dg2 = ff.rms_norm_backward(a, b, rstd, gamma, dh=c, out=(None, a, b, None)[k])
            assert torch.equal(got, dx) and torch.equal(dg2, dg), (pads, leads)


def test_rows_that_are_not_finite_and_rows_of_zeros():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(5, 300, device="cuda")
    clean, _, _ = ff.rms_norm(x, None)
    x[1, 7], x[2, 280] = float("nan"), float("inf")
    x[3] = 0
    y, _, rstd = ff.rms_norm(x, None)
    a, _, _ = ff.rms_norm_fp8(x, None)
    assert bool(y[1].isnan().all()) and bool(y[2, 280].isnan()) and float(rstd[2]) == 0.0
    assert bool((y[3] == 0).all()) and torch.equal(y[[0, 4]], clean[[0, 4]])
    assert bool(a.scale[:, 1].isnan().all()) and bool(a.scale[2, 2].isnan()) and bool((a.q[3].float() == 0).all())
    assert bool(torch.isfinite(a.scale[:, [0, 3, 4]]).all())


def test_empty_and_shaped():
    torch = torch_cuda()
    ff = lib_ready()
    y, h, rstd = ff.rms_norm(torch.empty(0, 12, device="cuda"), None)
    assert y.shape == (0, 12) and rstd.shape == (0,)
    dx, dg = ff.rms_norm_backward(torch.empty(0, 12, device="cuda"), h, rstd, None)
    assert dx.shape == (0, 12) and dg.tolist() == [0.0] * 12
    x = torch.randn(3, 5, 64, device="cuda")
    y, _, rstd = ff.rms_norm(x, None)
    assert y.shape == x.shape and rstd.shape == (15,)
    assert torch.equal(y.view(15, 64), ff.rms_norm(x.view(15, 64), None)[0])


def test_graph_replays_on_new_inputs():
    torch = torch_cuda()
    ff = lib_ready()
    x, r, dy = (torch.randn(300, 2000, device="cuda") for _ in range(3))
    gamma = torch.rand(2000, device="cuda")

    def step():
        y, h, rstd = ff.rms_norm(x, gamma, residual=r)
        return (y, h, rstd) + ff.rms_norm_backward(dy, h, rstd, gamma, dh=y)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(2):
        torch.manual_seed(seed)
        for t in (x, r, dy):
            t.normal_()
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_refusals():
    torch = torch_cuda()
    ff = lib_ready()
    x, g = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    _, _, rstd = ff.rms_norm(x, g)
    for bad, call in ((TypeError, lambda: ff.rms_norm(x.half(), g)), (TypeError, lambda: ff.rms_norm(3, g)),
                      (ValueError, lambda: ff.rms_norm(x.cpu(), g)), (ValueError, lambda: ff.rms_norm(x, g[:63])),
                      (TypeError, lambda: ff.rms_norm(x, g.bfloat16())), (ValueError, lambda: ff.rms_norm(x.t(), g)),
                      (ValueError, lambda: ff.rms_norm(x, g, residual=x[:3])), (ValueError, lambda: ff.rms_norm(x, g, h=x)),
                      (ValueError, lambda: ff.rms_norm(x, g, out=x.bfloat16())), (ff.FFError, lambda: ff.rms_norm(x, g, eps=0.0)),
                      (ff.FFError, lambda: ff.rms_norm(x, g, residual=x, out=x, h=x)),
                      (ValueError, lambda: ff.rms_norm_backward(x, x, rstd[:3], g)),
                      (ValueError, lambda: ff.rms_norm_backward(x, x, None, g)),
                      (ValueError, lambda: ff.rms_norm_backward(x, x[:2], rstd, g))):
        with pytest.raises(bad):
            call()
