"""Gradient clipping at the ends of its range: limits and norms that are not
finite, and gradients whose squares fp32 cannot hold."""

import math

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
COUNTS = {"cluster": [5000, 7], "two passes": [400000, 7], "several tables": [3000] * 130}


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("path", list(COUNTS))
def test_an_infinite_limit_asks_for_the_norm_alone(path, dtype, value):
    torch = torch_cuda()
    ff = lib_ready()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = [torch.randn(n, device="cuda").to(dt) for n in COUNTS[path]]
    g[0][g[0].numel() // 2] = value
    keep, out = [t.clone() for t in g], [torch.empty_like(t) for t in g]
    for into in (out, None):
        norm = float(ff.clip_grad_norm(g, math.inf, out=into))
        assert math.isnan(norm) if math.isnan(value) else norm == math.inf
        for t, k in zip(g if into is None else into, keep):
            assert torch.equal(t.nan_to_num(nan=-1.0), k.nan_to_num(nan=-1.0)) and torch.equal(t.isnan(), k.isnan())
            assert torch.equal(t.isinf(), k.isinf())


# Magnitudes: squares that overflow fp32 alone (1e30, 2^127) or added up (2^62 by
# the thread, 2^58 by the warp or the block), lose bits (1e-20) or vanish (1e-25, 1e-38,
# and 2^-140, which fp32 itself holds in nine bits).
SCALES = {"2^127": 2.0 ** 127, "1e30": 1e30, "2^62": 2.0 ** 62, "2^60": 2.0 ** 60, "2^58": 2.0 ** 58, "2^48": 2.0 ** 48, "2^-45": 2.0 ** -45, "2^-57": 2.0 ** -57, "2^-60": 2.0 ** -60,
          "1e-20": 1e-20, "2^-70": 2.0 ** -70, "1e-25": 1e-25, "1e-38": 1e-38, "2^-140": 2.0 ** -140}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("path", list(COUNTS))
@pytest.mark.parametrize("scale", list(SCALES))
def test_norms_of_any_finite_gradients(scale, path, dtype):
    """u = 2^-24.  A thread's 32 squares and their sum round 33 times at most (once more each where they are scaled), the
    fp32 sum over pieces once, a warp's five times; the root halves that and rounds once: 21 u.  A factor adds one
    rounding (two where it is two), a product one and the half step of its type; results and norms below 2^-126 round to
    multiples of 2^-149 (twice)."""
    torch = torch_cuda()
    ff = lib_ready()
    u = 2.0 ** -24
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    # +-[1/2, 1] of the scale for half of the values, else zero
    gen = torch.Generator().manual_seed(5)
    g = []
    for n in COUNTS[path]:
        t = (torch.rand(n, generator=gen, dtype=torch.float64) * 0.5 + 0.5) * (torch.randint(0, 2, (n,), generator=gen) * 2 - 1)
        t = t * (torch.rand(n, generator=gen) < 0.5) * SCALES[scale]
        g.append(t.float().cuda().to(dt))
    if scale == "2^127" and path == "cluster":  # three of them are not past fp32 together
        for t in g:
            t.zero_()
        g[0][:3] = torch.tensor([0.75, -0.5, 1.0]) * SCALES[scale]
    exact = math.sqrt(math.fsum(float(t.double().square().sum()) for t in g))
    for limit in (exact * 0.3, 1.0, 0.0, 1e-30):
        limit = float(torch.tensor(limit, dtype=torch.float32)) if limit < 2.0 ** 128 else 3e38
        out = [torch.full_like(t, 7.0) for t in g]
        norm = ff.clip_grad_norm(g, limit, out=out)
        got = float(norm)
        if exact >= 2.0 ** 128:  # past fp32
            assert got == math.inf and all(bool((o == 0).all()) for o in out)
            continue
        assert abs(got - exact) <= 21 * u * exact + 2.0 ** -148
        if exact == 0.0:  # 2^-140 in bf16
            assert all(bool((o == 0).all()) for o in out)
            continue
        by = min(1.0, limit / exact)
        # a norm below the normal range is itself off by half a multiple of 2^-149
        e = 24 * u + (2.0 ** -149 / exact if exact < 2.0 ** -126 else 0.0)
        for t, o in zip(g, out):
            want = t.double() * by
            tol = want.abs() * (e + torch.finfo(dt).eps / 2) + (2.0 ** -133 if dtype == "bf16" else 2.0 ** -148)
            assert bool(((o.double() - want).abs() <= tol).all())
        mine = [t.clone() for t in g]
        assert torch.equal(ff.clip_grad_norm(mine, limit), norm) and all(torch.equal(a, b) for a, b in zip(mine, out))


@pytest.mark.parametrize("path", ["cluster", "two passes"])
def test_large_small_and_moderate_gradients_together(path):
    """Each thread's sums take their own way; the same tolerance."""
    torch = torch_cuda()
    ff = lib_ready()
    n = COUNTS[path][0]
    for scales in ((1e-25, 1e-22), (1e-22, 1e-14), (1e-14, 1.0, 1e-30), (1.0, 1e14), (1e14, 1e20, 1e-25), (1e20, 1e35)):
        t = torch.randn(n, generator=torch.Generator().manual_seed(len(scales))).cuda()
        for i, s in enumerate(scales):
            t[i * 17 % 1024::1024] *= s
        exact = math.sqrt(float(t.double().square().sum()))
        out = torch.empty_like(t)
        norm = float(ff.clip_grad_norm([t], exact / 2, out=[out]))
        assert abs(norm - exact) <= 21 * 2.0 ** -24 * exact
        want = t.double() * (float(torch.tensor(exact / 2)) / exact)
        assert bool(((out.double() - want).abs() <= 24 * 2.0 ** -24 * want.abs() + 2.0 ** -148).all())


@pytest.mark.parametrize("lead", [0, 1, 61, 64])
def test_gradients_left_alone_keep_their_neighbours(lead):
    """Nothing is clipped: what the second pass does with the lines that the first one left in L2 changes no value, at
    whatever place in a line the tensors start and end."""
    torch = torch_cuda()
    ff = lib_ready()
    for dt in (torch.float32, torch.bfloat16):
        buf = torch.randn(3_000_001, device="cuda").to(dt)
        keep, g = buf.clone(), [buf[lead:lead + 1_000_003], buf[1_500_000:1_500_003], buf[1_500_007:2_999_999]]
        for limit in (math.inf, 1e9):
            ff.clip_grad_norm(g, limit)
            assert torch.equal(buf, keep)
