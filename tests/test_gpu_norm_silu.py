"""SiLU and its slope from far below zero to far above, on every path of the
group norm: with gamma = 0 the pre-activation of a channel is its beta, and one
row of ones as dy makes dbeta the slope.

Tolerances, relative: bf16 outputs 2^-8 (their rounding).  fp32 outputs 2^-17:
an exponential whose argument, up to 88 log2 e = 127, is rounded to 2^-24 of itself
errs by 127 ln 2 2^-24 < 2^-17.5, and the rest adds a few 2^-23.  Slopes, formed
in fp32, the same of p (1 + |u|), which bounds what cancels in p (1 + u (1 - p)).
Absolute: 1e-35 where results leave the normal range."""

import numpy as np
import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu

# rows of a warp, a block and one by one; slabs; column passes
SHAPES = [(1, 1, 512, 8), (1, 1, 6000, 1), (1, 1, 501, 3), (1, 49, 256, 8), (1, 7000, 64, 2)]


def preactivations(C, seed):
    """C values of u: small ones, the range where the exponential leaves fp32, and beyond."""
    r = np.random.RandomState(seed)
    far = np.array([-1e38, -1e30, -1e20, -1e18, -1e6, -200.0, -104.0, -88.0, -60.0, -41.7, -41.5, 0.0, 60.0, 1e6, 1e20])
    u = np.concatenate([far, r.uniform(-90, 90, C - far.size)])
    return r.permutation(u).astype(np.float32)


def definition(u):
    with np.errstate(over="ignore"):
        e = np.exp(-np.abs(u))
    p = np.where(u >= 0, 1 / (1 + e), e / (1 + e))
    q = np.where(u >= 0, e / (1 + e), 1 / (1 + e))  # 1 - p
    return u * p, p * (1 + u * q), p


def results(torch, ff, shape, dtype, seed):
    n, S, C, G = shape
    u = preactivations(C, seed)
    x = torch.randn(n, S, C, generator=torch.Generator().manual_seed(seed)).cuda()
    x = x.bfloat16() if dtype == "bf16" else x
    gamma, beta = torch.zeros(C, device="cuda"), torch.from_numpy(u).cuda()
    y, m, r = ff.group_norm_act(x, gamma, beta, G, act="silu")
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    _, _, slope = ff.group_norm_act_backward(dy, x, m, r, gamma, beta, G, act="silu")
    return u.astype(np.float64), y.double().cpu().numpy(), slope.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_silu_far_out(shape, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    u, y, slope = results(torch, ff, shape, dtype, SHAPES.index(shape))
    want, ds, p = definition(u)
    rel = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -17
    assert np.all(np.abs(y - want) <= rel * np.abs(want) + 1e-35)
    with np.errstate(over="ignore", invalid="ignore"):
        tol = 2.0 ** -17 * np.where(p > 0, p * (1 + np.abs(u)), 0.0) + 1e-35
    assert np.all(np.abs(slope - ds) <= tol)


@pytest.mark.parametrize("shape", SHAPES)
def test_silu_of_fp32_in_full(shape):
    """fp32, where results are in the normal range (u >= -80): the exponential within two units, 1 + e and the products
    half a unit each, the reciprocal one, so a value is within 2^-21 of itself, and a slope of p (1 + |u|)."""
    torch = torch_cuda()
    ff = lib_ready()
    u, y, slope = results(torch, ff, shape, "fp32", 10 + SHAPES.index(shape))
    want, ds, p = definition(u)
    at = (u >= -80) & (u <= 1e6)
    assert np.all(np.abs(y - want)[:, :, at] <= 2.0 ** -21 * np.abs(want[at]))
    assert np.all(np.abs(slope - ds)[at] <= 2.0 ** -21 * (p * (1 + np.abs(u)))[at])
