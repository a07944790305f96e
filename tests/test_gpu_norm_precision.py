"""Group norm where the mean is large beside the spread, in fp32: what is formed
from x - mean keeps its bits.

Tolerances (U = 2^-24).  With the kernel's own mean and rstd as given, x - mean
and its product with rstd round once each, so h errs by at most 2 U |h| (4 are
allowed), whatever the mean; a form that multiplies first errs by U |mean| rstd.
The rest is as in test_gpu_norm.py: u adds 4 U (|u| + |beta|), the activations
2^-20 of a value, sums 64 U of their magnitudes.  The kernels read y, dx and the
sums that way on every path."""

import numpy as np
import pytest

from .gpu_common import lib_ready, torch_cuda
from .test_gpu_norm import U, act, make, per_channel, slope

pytestmark = pytest.mark.gpu

# rows: of a warp, a block, several positions; slabs of one group and several, one unit a block and several; column passes
SHAPES = [(5, 1, 500, 10), (9, 1, 6000, 1), (3, 7, 48, 6), (40, 49, 256, 32), (300, 784, 64, 8), (512, 196, 64, 4),
          (2, 4100, 320, 32), (1, 9000, 250, 2), (3, 20001, 8, 2), (2, 700, 130, 2)]


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradient_of_a_large_mean(shape, kind):
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    x, x64, gen = make(torch, n, S, C, "fp32", seed=SHAPES.index(shape), offset=2000.0)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=gen), 0.3 * torch.randn(C, generator=gen)
    dy = torch.randn(n, S, C, generator=gen)
    _, m, r = ff.group_norm_act(x, gamma.cuda(), beta.cuda(), G, act=kind)
    m64, r64 = m.double().cpu().numpy(), r.double().cpu().numpy()
    g64, b64 = gamma.double().numpy(), beta.double().numpy()
    R = per_channel(r64, S, C)
    h = (x64 - per_channel(m64, S, C)) * R
    u = h * g64 + b64
    DH = 4 * U * np.abs(h)
    DUU = np.abs(g64) * DH + 4 * U * (np.abs(u) + np.abs(b64))
    dy[torch.from_numpy(np.abs(u) <= DUU)] = 0  # no gradient at the ReLU's kink, where either side is right
    d64 = dy.double().numpy()
    dx, dgam, dbet = ff.group_norm_act_backward(dy.cuda(), x, m, r, gamma.cuda(), beta.cuda(), G, act=kind)
    du = d64 * slope(u, kind)
    Ddu = np.abs(d64) * ((0.5 if kind == "silu" else 0.0) * DUU) + (4 * U + 2.0 ** -20) * np.abs(d64) * 1.1
    if kind != "silu":
        Ddu = 0 * Ddu
    tb = Ddu.sum((0, 1)) + 64 * U * np.abs(du).sum((0, 1))
    tg = (Ddu * np.abs(h) + np.abs(du) * DH).sum((0, 1)) + 64 * U * np.abs(du * h).sum((0, 1))
    assert np.all(np.abs(dbet.double().cpu().numpy() - du.sum((0, 1))) <= tb + 1e-30)
    assert np.all(np.abs(dgam.double().cpu().numpy() - (du * h).sum((0, 1))) <= tg + 1e-30)

    def avg(t):
        return per_channel(t.reshape(n, S, G, C // G).mean(axis=(1, 3)), S, C)

    w, Dw = g64 * du, np.abs(g64) * Ddu
    a1, a2 = avg(w), avg(w * h)
    D1 = avg(Dw) + 64 * U * avg(np.abs(w))
    D2 = avg(Dw * np.abs(h) + np.abs(w) * DH) + 64 * U * avg(np.abs(w * h))
    dx64 = R * (w - a1 - h * a2)
    tol = R * (Dw + D1 + np.abs(h) * D2 + DH * np.abs(a2) + 4 * U * (np.abs(w) + np.abs(a1) + np.abs(h * a2)))
    assert np.all(np.abs(dx.double().cpu().numpy() - dx64) <= tol + 2.0 ** -23 * np.abs(dx64) + 1e-30)


@pytest.mark.parametrize("kind", ["none", "relu", "silu"])
@pytest.mark.parametrize("shape", SHAPES)
def test_outputs_of_a_large_mean(shape, kind):
    """With the returned mean and rstd as given; the two may be rounded once more than what the outputs are formed from."""
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    x, x64, gen = make(torch, n, S, C, "fp32", seed=SHAPES.index(shape), offset=2000.0)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=gen), 0.3 * torch.randn(C, generator=gen)
    y, m, r = ff.group_norm_act(x, gamma.cuda(), beta.cuda(), G, act=kind)
    h = (x64 - per_channel(m.double().cpu().numpy(), S, C)) * per_channel(r.double().cpu().numpy(), S, C)
    u = h * gamma.double().numpy() + beta.double().numpy()
    DU = 6 * U * (np.abs(h * gamma.double().numpy()) + np.abs(beta.double().numpy()))
    y64 = act(u, kind)
    assert np.all(np.abs(y.double().cpu().numpy() - y64) <= 1.1 * DU + (2.0 ** -23 + 2.0 ** -20) * np.abs(y64) + 1e-30)
