"""Group norm with an activation and its gradient, against the definition in
64 bits.

Tolerances (u = 2^-24).  The input is exact on both sides.  A sum of m terms
formed in fp32 by blocked sums errs by at most 64 u times the sum of the
magnitudes for the block sizes the kernels use; a group's centred sum of
squares by at most 64 u of itself (each thread's pivot is one of its own
values); so |d mean| <= 64 u <|x|> and |d rstd| <= 64 u rstd.  The
pre-activation u = gamma (x - mean) rstd + beta then errs by DU = 80 u
(|gamma| rstd (|x| + <|x|>) + |beta|), the activations have slopes of at
most 1.1 and curvatures of at most 0.5, and the fast exponential and division
add 2^-20 of the value.  bf16 outputs add their rounding, 2^-8 of the value.
"""

import numpy as np
import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def silu(u):
    return u / (1 + np.exp(-u))


def act(u, kind):
    return np.maximum(u, 0) if kind == "relu" else silu(u) if kind == "silu" else u


def slope(u, kind):
    if kind == "relu":
        return (u > 0).astype(np.float64)
    if kind == "silu":
        p = 1 / (1 + np.exp(-u))
        return p * (1 + u * (1 - p))
    return np.ones_like(u)


def forward64(x, gamma, beta, G, kind, eps):
    """x [n, S, C] float64."""
    n, S, C = x.shape
    g = x.reshape(n, S, G, C // G)
    mean = g.mean(axis=(1, 3))
    var = ((g - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    rstd = 1 / np.sqrt(var + eps)
    h = ((g - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(n, S, C)
    u = h * gamma + beta
    return act(u, kind), mean, rstd, h, u


def per_channel(stat, S, C):
    """[n, G] -> [n, S, C]"""
    n, G = stat.shape
    return np.repeat(np.repeat(stat, C // G, axis=1)[:, None, :], S, axis=1)


def du_bound(x, gamma, beta, rstd, G):
    n, S, C = x.shape
    ax = np.abs(x).reshape(n, S, G, C // G).mean(axis=(1, 3))
    return 80 * U * (np.abs(gamma) * per_channel(rstd, S, C) * (np.abs(x) + per_channel(ax, S, C)) + np.abs(beta))


def make(torch, n, S, C, dtype, seed, pad=0, offset=0.0, lead=0):
    """x as [n, S, C] on the GPU (rows of C + pad elements, starting `lead` elements into the buffer) and in 64 bits."""
    gen = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = (2 * torch.randn(n, S, C, generator=gen) + torch.randn(C, generator=gen) + offset).to(dt)
    buf = torch.full((n * S * (C + pad) + lead,), float("nan"), dtype=dt, device="cuda")
    view = buf[lead:].view(n, S, C + pad)[:, :, :C]
    view.copy_(x)
    return view, x.double().numpy(), gen


# n, S, C, G: groups of one value and of a whole row, odd widths, one position and many, ragged chunks
SHAPES = [
    (1, 1, 1, 1), (3, 1, 8, 8), (5, 1, 500, 10), (7, 1, 2000, 16), (4, 1, 2000, 8), (2, 1, 6000, 1), (70, 1, 96, 3),
    (2, 3, 30, 2), (2, 2, 1000, 4), (3, 7, 48, 6), (1, 100, 24, 2), (2, 257, 40, 4), (3, 1000, 64, 32), (1, 5000, 16, 1),
    (2, 4100, 320, 32), (1, 20001, 8, 2), (1, 3, 9000, 3), (9, 33, 130, 13), (1, 70000, 4, 2), (1, 9000, 256, 2),
    (33, 1, 8192, 1), (700, 1, 2001, 1), (6, 1, 4100, 2), (900, 1, 8200, 1), (3, 1, 1200, 2), (40, 49, 256, 32), (300, 784, 64, 8),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_gradient(shape, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    k = SHAPES.index(shape)
    kind = ("none", "relu", "silu")[k % 3]
    pad, lead = ((0, 0), (8, 0), (3, 1), (0, 8))[k % 4]
    x, x64, gen = make(torch, n, S, C, dtype, seed=k, pad=pad, lead=lead)
    gamma = 1 + 0.3 * torch.randn(C, generator=gen)
    beta = 0.3 * torch.randn(C, generator=gen)
    dy = torch.randn(n, S, C, generator=gen).to(x.dtype)
    y64, mean, rstd, h, u = forward64(x64, gamma.double().numpy(), beta.double().numpy(), G, kind, 1e-5)
    DU = du_bound(x64, gamma.double().numpy(), beta.double().numpy(), rstd, G)
    dy[torch.from_numpy(np.abs(u) <= DU)] = 0  # no gradient at the ReLU's kink, where either side is right
    gg, bb = gamma.cuda(), beta.cuda()
    y, m, r = ff.group_norm_act(x, gg, bb, G, act=kind, eps=1e-5)
    dx, dgam, dbet = ff.group_norm_act_backward(dy.cuda(), x, m, r, gg, bb, G, act=kind)
    torch.cuda.synchronize()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    ax = np.abs(x64).reshape(n, S, G, C // G).mean(axis=(1, 3))
    assert np.all(np.abs(m.double().cpu().numpy() - mean) <= 64 * U * ax + 1e-30)
    assert np.all(np.abs(r.double().cpu().numpy() - rstd) <= 64 * U * rstd * (1 + (ax * rstd) ** 2 * U * 64))
    assert np.all(np.abs(y.double().cpu().numpy() - y64) <= 1.1 * DU + (half + 2.0 ** -20) * np.abs(y64) + 1e-30)

    # the gradient, with the forward's own mean and rstd as its inputs
    m64, r64 = m.double().cpu().numpy(), r.double().cpu().numpy()
    g64, b64, d64 = gamma.double().numpy(), beta.double().numpy(), dy.double().numpy()
    R = per_channel(r64, S, C)
    h = (x64 - per_channel(m64, S, C)) * R
    u = h * g64 + b64
    DH = 4 * U * R * (np.abs(x64) + np.abs(per_channel(m64, S, C)))  # rounding of h
    DUU = np.abs(g64) * DH + 4 * U * (np.abs(u) + np.abs(b64))
    du = d64 * slope(u, kind)
    Ddu = np.abs(d64) * ((0.5 if kind == "silu" else 0.0) * DUU) + (4 * U + 2.0 ** -20) * np.abs(d64) * 1.1
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
    assert np.all(np.abs(dx.double().cpu().numpy() - dx64) <= tol + half * np.abs(dx64) + 1e-30)


@pytest.mark.parametrize("kind", ["none", "silu"])
@pytest.mark.parametrize("shape", [(2, 1, 40, 4), (2, 9, 24, 3)])
def test_gradient_against_differences(shape, kind):
    """d/dt of sum w . y along random directions of x, gamma and beta, by central differences of the 64-bit definition
    (step 1e-5: truncation of order 1e-10, rounding of order 1e-11), against the kernel's gradients."""
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    x, x64, gen = make(torch, n, S, C, "fp32", seed=50)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=gen), 0.3 * torch.randn(C, generator=gen)
    w = torch.randn(n, S, C, generator=gen)
    _, m, r = ff.group_norm_act(x, gamma.cuda(), beta.cuda(), G, act=kind, eps=1e-5)
    grads = ff.group_norm_act_backward(w.cuda(), x, m, r, gamma.cuda(), beta.cuda(), G, act=kind)
    at = [x64, gamma.double().numpy(), beta.double().numpy()]
    for i, got in enumerate(grads):
        got = got.double().cpu().numpy().reshape(at[i].shape)
        for seed in range(3):
            v = np.random.RandomState(seed).randn(*at[i].shape)

            def f(t):
                a = [q + t * v if j == i else q for j, q in enumerate(at)]
                return float((forward64(a[0], a[1], a[2], G, kind, 1e-5)[0] * w.double().numpy()).sum())

            diff = (f(1e-5) - f(-1e-5)) / 2e-5
            assert abs(diff - float((got * v).sum())) <= 2e-5 * float(np.abs(got * v).sum()) + 1e-7


@pytest.mark.parametrize("shape", [(3, 1, 64, 4), (2, 300, 32, 4)])
def test_no_parameters_and_partial_outputs(shape):
    """gamma and beta of NULL are ones and zeros, bit for bit; a large mean does not cancel the spread."""
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    x, x64, _ = make(torch, n, S, C, "fp32", seed=3, offset=1000.0)
    one, zero = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    a = ff.group_norm_act(x, None, None, G, act="none")
    b = ff.group_norm_act(x, one, zero, G, act="none")
    dy = torch.randn(n, S, C, device="cuda")
    ga = ff.group_norm_act_backward(dy, x, a[1], a[2], None, None, G, act="none")
    gb = ff.group_norm_act_backward(dy, x, a[1], a[2], one, zero, G, act="none")
    for p, q in zip(a + ga, b + gb):
        assert torch.equal(p, q)
    y64, mean, rstd, _, _ = forward64(x64, 1.0, 0.0, G, "none", 1e-5)
    assert np.all(np.abs(a[2].double().cpu().numpy() - rstd) <= 64 * U * rstd * (1 + 1e-3))
    assert np.all(np.abs(a[0].double().cpu().numpy() - y64) <= du_bound(x64, np.ones(C), np.zeros(C), rstd, G))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(4, 1, 500, 10), (2, 500, 40, 4), (1, 30000, 16, 2)])
def test_in_place_and_repeated_calls_give_the_same_bits(shape, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    x, _, gen = make(torch, n, S, C, dtype, seed=9)
    gamma, beta = torch.randn(C, generator=gen).cuda(), torch.randn(C, generator=gen).cuda()
    dy = torch.randn(n, S, C, generator=gen).to(x.dtype).cuda()
    first = ff.group_norm_act(x, gamma, beta, G)
    grads = ff.group_norm_act_backward(dy, x, first[1], first[2], gamma, beta, G)
    again = ff.group_norm_act(x, gamma, beta, G)
    for p, q in zip(first, again):
        assert torch.equal(p, q)
    into_dy, into_x, x2 = dy.clone(), x.clone(), x.clone()
    for out, args in ((into_dy, (into_dy, x)), (into_x, (dy, into_x))):
        g = ff.group_norm_act_backward(*args, first[1], first[2], gamma, beta, G, out=out)
        assert g[0] is out
        for p, q in zip(g, grads):
            assert torch.equal(p, q)
    y, _, _ = ff.group_norm_act(x2, gamma, beta, G, out=x2)
    assert y is x2 and torch.equal(y, first[0])


@pytest.mark.parametrize("shape", [(4, 1, 60, 6), (3, 200, 24, 3), (1, 40000, 8, 2)])
def test_nan_stays_in_its_group(shape):
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    for bad in (float("nan"), float("inf")):
        x, _, _ = make(torch, n, S, C, "fp32", seed=11)
        clean = ff.group_norm_act(x, None, None, G, act="relu")
        x = x.clone()
        x[0, S // 2, C // G] = bad  # first channel of group 1 of sample 0
        y, m, r = ff.group_norm_act(x, None, None, G, act="relu")
        hit = torch.zeros(n, S, C, dtype=torch.bool, device="cuda")
        hit[0, :, C // G:2 * (C // G)] = True
        assert torch.isnan(y[hit]).all()
        assert torch.equal(y[~hit], clean[0][~hit])


def test_constant_groups():
    """No spread at all: rstd = 1 / sqrt(eps), outputs act(beta)."""
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.full((2, 50, 16), 3.0, device="cuda")
    beta = torch.randn(16, device="cuda")
    y, m, r = ff.group_norm_act(x, None, beta, 2, act="none", eps=1e-4)
    assert torch.equal(y, beta.expand_as(y)) and torch.equal(m, torch.full_like(m, 3.0))
    assert torch.allclose(r, torch.full_like(r, 100.0), rtol=4 * U * 2, atol=0)


def test_empty_inputs():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.empty(0, 8, device="cuda")
    y, m, r = ff.group_norm_act(x, None, None, 2)
    assert y.shape == (0, 8) and m.shape == (0, 2)
    _, dg, db = ff.group_norm_act_backward(x, x, m, r, None, None, 2)
    assert torch.equal(dg, torch.zeros(8, device="cuda")) and torch.equal(db, torch.zeros(8, device="cuda"))
    x = torch.empty(3, 0, 8, device="cuda")
    y, m, r = ff.group_norm_act(x, None, None, 2)
    assert y.shape == (3, 0, 8) and torch.equal(m, torch.zeros(3, 2, device="cuda")) and torch.equal(r, m)


def test_refusals():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(4, 10, 12, device="cuda")
    ok = dict(gamma=None, beta=None, groups=3)
    for bad in (x.cpu(), x.half(), x.transpose(1, 2), x.expand(2, 4, 10, 12), x[:, ::2].transpose(0, 1)[:, :, :5], x[0, 0]):
        with pytest.raises((TypeError, ValueError)):
            ff.group_norm_act(bad, **ok)
    for kw in (dict(groups=5), dict(groups=0), dict(act="tanh"), dict(gamma=torch.ones(11, device="cuda")),
               dict(gamma=torch.ones(12, device="cuda", dtype=torch.bfloat16)), dict(beta=torch.ones(12)),
               dict(mean=torch.empty(5, 3, device="cuda")), dict(out=torch.empty(4, 10, 13, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            ff.group_norm_act(x, **{**ok, **kw})
    with pytest.raises(ff.FFError):
        ff.group_norm_act(x, None, None, 3, eps=0.0)
    y, m, r = ff.group_norm_act(x, None, None, 3)
    with pytest.raises(ValueError):
        ff.group_norm_act_backward(y[:, :5], x, m, r, None, None, 3)
    with pytest.raises(ValueError):
        ff.group_norm_act_backward(y, x, m[:2], r, None, None, 3)
    with pytest.raises(ValueError):
        ff.group_norm_act_backward(y, x, None, None, None, None, 3)


@pytest.mark.parametrize("shape", [(1100000, 1, 2000, 16), (70, 16384, 2048, 32), (70000, 64, 512, 32)])
def test_more_than_2_31_values(shape):
    """Rows, column passes and blocks: the last sample of a large batch as that
    sample alone.  The sums may have another order (statistics a few units of
    2^-24 apart), so an output may round to the next bf16."""
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    assert n * S * C > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty(n, S, C, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)
    y, m, r = ff.group_norm_act(x, None, None, G)
    last = x[-1:].clone()
    y1, m1, r1 = ff.group_norm_act(last, None, None, G)
    near = lambda a, b: torch.all((a.float() - b.float()).abs() <= 2.0 ** -7 * b.float().abs() + 1e-5)
    assert near(y[-1:], y1) and near(m[-1:], m1) and near(r[-1:], r1)
    assert torch.isfinite(y.view(-1)[::997].float()).all()
    dx, _, _ = ff.group_norm_act_backward(x, x, m, r, None, None, G, out=y)  # dy = x
    d1, _, _ = ff.group_norm_act_backward(last, last, m1, r1, None, None, G)
    assert near(dx[-1:], d1)


@pytest.mark.parametrize("shape", [(3, 1, 500, 10), (1, 3, 500, 10), (1, 3, 512, 8)])
def test_row_strides_past_31_bits(shape):
    """Rows 2^30 elements and more apart, against the same rows side by side."""
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    x = torch.randn(n, S, C, device="cuda")
    wide = torch.empty(3 * ((1 << 30) + 8), device="cuda")
    v = wide.as_strided((n, S, C), ((S if n == 1 else 1) * ((1 << 30) + 8), (1 << 30) + 8, 1))
    v.copy_(x)
    y, m, r = ff.group_norm_act(x, None, None, G)
    w, p, q = ff.group_norm_act(v, None, None, G)
    near = lambda a, b: torch.allclose(a, b, rtol=1e-5, atol=1e-5)
    assert near(w, y) and near(p, m) and near(q, r)
    dx, dg, db = ff.group_norm_act_backward(x, x, m, r, None, None, G)
    dv, eg, eb = ff.group_norm_act_backward(v, v, m, r, None, None, G, out=v)
    assert near(dv, dx) and near(eg, dg) and near(eb, db)


def test_a_mean_near_zero_keeps_its_bits():
    """Groups of zero mean whose first value is three spreads off: the mean must
    not come out as a difference of numbers of that size.  A group's mean is
    averaged from more than 10,000 threads' means of up to 64 values, each off
    by a few rounding units of the spread and independent of the others, so it
    is a few hundredths of a unit off; half a unit is asked for.  Held relative
    to the first value, the sum's own rounding alone is one to three."""
    torch = torch_cuda()
    ff = lib_ready()
    gen = torch.Generator().manual_seed(5)
    n, S, C, G = 2, 9000, 64, 4
    x = torch.randn(n, S, C, generator=gen)
    x -= x.reshape(n, S, G, C // G).mean(dim=(1, 3)).repeat_interleave(C // G, dim=1)[:, None, :]
    x[:, 0, ::C // G], x[:, 0, 1::C // G] = 3.0, -1.0
    _, m, _ = ff.group_norm_act(x.cuda(), None, None, G, act="none")
    x64 = x.double().reshape(n, S, G, C // G)
    mean, size = x64.mean(dim=(1, 3)), x64.abs().mean(dim=(1, 3))
    assert torch.all((m.double().cpu() - mean).abs() <= 0.5 * U * size)


@pytest.mark.parametrize("shape", [(2, 100, 8, 2), (16, 1, 500, 10), (4, 50000, 8, 2)])
def test_a_short_workspace_is_refused(shape):
    """Less than the size query's answer is refused for every stride and
    alignment, also where this call's own path would need less.  The buffers
    are real and of full size: only the size that is stated is too small."""
    torch = torch_cuda()
    ff = lib_ready()
    L = ff.lib()
    n, S, C, G = shape
    x = torch.randn(n * S, C, device="cuda")
    y, dg, db = torch.zeros_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    m, r = torch.zeros(n, G, device="cuda"), torch.ones(n, G, device="cuda")
    f, g = (L.ff_group_norm_workspace(n, S, C, G, 0, b) for b in (0, 1))
    ws = torch.empty(max(f, g) + 16, dtype=torch.uint8, device="cuda")

    def forward(p, size):
        return L.ff_group_norm_act(x.data_ptr(), C, n, S, C, G, None, None, 1e-5, 2, 0, y.data_ptr(), C, m.data_ptr(),
                                   r.data_ptr(), p, size, None)

    def backward(p, size):
        return L.ff_group_norm_act_backward(x.data_ptr(), C, x.data_ptr(), C, n, S, C, G, m.data_ptr(), r.data_ptr(),
                                            None, None, 2, 0, y.data_ptr(), C, dg.data_ptr(), db.data_ptr(), p, size,
                                            None)

    for call, need in ((forward, f), (backward, g)):
        if need:
            for p, size in ((ws.data_ptr(), need - 1), (ws.data_ptr() + 8, need), (None, need)):
                assert call(p, size) == 1
        assert call(ws.data_ptr() if need else None, need) == 0
    torch.cuda.synchronize()


@pytest.mark.parametrize("shape", [(64, 1, 500, 10), (8, 1024, 64, 8), (1, 60000, 16, 2)])
def test_another_stream_and_a_captured_graph(shape):
    """On a side stream that is behind, with the caller's stream free to reuse
    memory; and replayed from a CUDA graph on new inputs."""
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    x, _, _ = make(torch, n, S, C, "bf16", seed=21)
    x = x.contiguous()
    want = ff.group_norm_act(x, None, None, G)
    wantg = ff.group_norm_act_backward(want[0], x, want[1], want[2], None, None, G)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(5):
            big = big @ big * 1e-3
    got = ff.group_norm_act(x, None, None, G, stream=side)
    gotg = ff.group_norm_act_backward(got[0], x, got[1], got[2], None, None, G, stream=side)
    for _ in range(20):  # would overwrite a workspace handed back too early
        torch.full((1 << 20,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    for p, q in zip(got + gotg, want + wantg):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    static = x.clone()
    with torch.cuda.graph(graph):
        y = ff.group_norm_act(static, None, None, G)
        gr = ff.group_norm_act_backward(y[0], static, y[1], y[2], None, None, G)
    for k in range(3):
        x2, _, _ = make(torch, n, S, C, "bf16", seed=30 + k)
        static.copy_(x2)
        graph.replay()
        torch.cuda.synchronize()
        ref = ff.group_norm_act(static, None, None, G)
        refg = ff.group_norm_act_backward(ref[0], static, ref[1], ref[2], None, None, G)
        for p, q in zip(y + gr, ref + refg):
            assert torch.equal(p, q)
