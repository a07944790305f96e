"""Label log-probabilities, entropies and likeliest classes, and their gradient,
against the definition in 64 bits.

Tolerances.  u = 2^-24 is a rounding to fp32; the approximate exponential is
within 2^-22 of itself.  A term e^d has a rounded d and a rounded product
with log2 e, so it is within e1(d) = 2^-22 + 3 u |d| of itself.  Sums of positive
terms add `chain` roundings and, each time a maximum grows (at most once a vector
of a thread, and once for each of 12 joins), one exponential's error.
"""

import numpy as np
import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
U, EXP = 2.0 ** -24, 2.0 ** -22
SIZES = [(1, 1), (1, 2), (7, 10), (5, 33), (200, 100), (160, 2048), (3, 2049), (40, 1000), (1, 5000), (2, 49999), (1, 131072), (700, 4099),
         (1, 200003), (20, 30000), (5000, 17)]


def logits_of(torch, rows, classes, dt, i, masked=0.0):
    gen = torch.Generator().manual_seed(1000 + i)
    x = torch.randn(rows, classes, generator=gen) * (1 + 3 * torch.rand(rows, 1, generator=gen)) + 5
    labels = torch.randint(0, classes, (rows,), generator=gen, dtype=torch.int32)
    if masked:
        x[torch.rand(rows, classes, generator=gen) < masked] = float("-inf")
        x[torch.arange(rows), labels.long()] = 1.5
    if rows > 2:
        labels[1], labels[2] = -1, classes
    pad, lead = ((0, 0), (8, 8), (3, 1), (1, 0))[i % 4]
    buf = torch.full((lead + rows * (classes + pad),), float("nan"), dtype=dt, device="cuda")
    view = buf[lead:].view(rows, classes + pad)[:, :classes]
    view.copy_(x)
    return view, labels.cuda()


def definition(torch, x, labels, classes, threads=256):
    """logp, entropy, z, p, ln p of x in 64 bits, and the bounds of the sums' and the entropy's errors (`threads` a row)."""
    x = x.double()
    m = x.amax(1, keepdim=True)
    z = torch.logsumexp(x, 1, keepdim=True)
    lp = x - z
    p = lp.exp()
    d = torch.where(p > 0, x - m, 0.0)
    has = (labels >= 0) & (labels < classes)
    logp = torch.where(has, lp.gather(1, labels.clamp(0, classes - 1).long()[:, None])[:, 0], 0.0)
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(1)
    e1 = EXP + 3 * U * d.abs()
    raises = classes // (4 * threads) + 14
    sums = raises * (EXP + 8 * U) + (classes // threads + 40) * U
    es = (p * e1).sum(1) + sums
    t = (p * d.abs()).sum(1)
    et = (p * d.abs() * e1).sum(1) + t * sums
    ln = (z - m)[:, 0]
    eh = 1.1 * (es + et + t * es + 4 * U * (ln + t))
    return logp, entropy, m[:, 0], ln, p, lp, d, has, 1.1 * es + 4 * U * ln, eh


@pytest.mark.parametrize("masked", [0.0, 0.3])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES)
def test_forward_and_backward(size, dtype, masked):
    torch = torch_cuda()
    ff = lib_ready()
    rows, classes = size
    i = SIZES.index(size)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, labels = logits_of(torch, rows, classes, dt, i, masked)
    logp, entropy, m, ln, p, lp, d, has, e_ln, e_h = definition(torch, x, labels, classes)
    order = torch.sort(x.double(), dim=1, descending=True, stable=True).indices
    for top in sorted({0, 1, min(5, classes), min(32, classes)}):
        r = ff.label_logprobs(x, labels, top=top)
        e_label = e_ln + 2 * U * (logp.abs() + ln)
        assert bool(((r.logp.double() - logp).abs() <= torch.where(has, e_label, 0.0)).all())
        assert bool(((r.entropy.double() - entropy).abs() <= e_h).all())
        assert torch.equal(r.stats[:, 0].double(), m) and bool(((r.stats[:, 1].double() - ln).abs() <= e_ln).all())
        assert r.top_index.shape == (rows, top) and torch.equal(r.top_index.long(), order[:, :top])
        want = lp.gather(1, order[:, :top])
        tol = e_ln[:, None] + 2 * U * (want.abs() + ln[:, None])
        assert bool(((r.top_logp.double() == want) | ((r.top_logp.double() - want).abs() <= tol)).all())
    gen = torch.Generator().manual_seed(i)
    g, ge = ((torch.rand(rows, generator=gen) - 0.5).cuda() for _ in range(2))
    for dlogp, dent in ((g, None), (g, ge), (None, ge)):
        dx = ff.label_logprobs_backward(x, labels, r.stats, dlogp, entropy=r.entropy, dentropy=dent)
        a = torch.where(has, dlogp.double(), 0.0)[:, None] if dlogp is not None else torch.zeros(rows, 1, device="cuda").double()
        b = dent.double()[:, None] if dent is not None else torch.zeros(rows, 1, device="cuda").double()
        # from the stats and the entropy that were passed
        L, H = r.stats[:, 1:].double(), r.entropy.double()[:, None]
        q = torch.where(p > 0, (d - L).exp(), 0.0)
        inner = a + b * (d - L + H)
        want = -q * inner
        rows_with = torch.nonzero(has)[:, 0]
        want[rows_with, labels[rows_with].long()] += a[rows_with, 0]
        size_of = q * (a.abs() + b.abs() * (d.abs() + L.abs() + H.abs()))
        tol = size_of * (2 * EXP + 4 * U * (d.abs() + L.abs()) + 6 * U) + U * a.abs() + want.abs() * (torch.finfo(dt).eps / 2)
        assert dx.shape == x.shape and bool(((dx.double() - want).abs() <= tol + 2.0 ** -120).all())


def test_ties_go_to_the_lowest_index():
    """Few values, so that most are equal, in every layout of warps and blocks; and rows of one value only."""
    torch = torch_cuda()
    ff = lib_ready()
    for rows, classes in ((1, 131072), (3, 4999), (300, 700), (900, 6000), (2, 40)):
        gen = torch.Generator().manual_seed(classes)
        for values in (1, 2, 3, 40):
            x = torch.randint(0, values, (rows, classes), generator=gen).float().cuda() - 1.0
            x = torch.where(x == 0, -x, x)  # zeros of both signs are equal
            want = torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :32]
            for dt in (torch.float32, torch.bfloat16):
                assert torch.equal(ff.label_logprobs(x.to(dt), None, top=32).top_index.long(), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("classes", [1, 2, 3, 4, 5, 8, 9, 16, 17, 31, 32, 33, 48, 63, 64, 65, 97, 128, 129])
def test_short_rows(classes, dtype):
    """Several rows a warp: labels everywhere, rows of few values, masks that leave less than `top`, and rows
    without a distribution beside proper ones."""
    torch = torch_cuda()
    ff = lib_ready()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(classes)
    rows = 2 * classes + 75
    x = torch.randn(rows, classes, generator=gen) * 3
    x[::3] = x[::3].round()
    x[1::4][torch.rand(len(x[1::4]), classes, generator=gen) < 0.6] = float("-inf")
    labels = torch.arange(rows, dtype=torch.int32) % (classes + 2) - 1
    x[torch.arange(rows), labels.clamp(0, classes - 1).long()] = 0.5
    x[40] = float("-inf")
    x[41, classes // 2] = float("nan")
    x[42, classes - 1] = float("inf")
    x = x.to(dt).cuda()
    labels = labels.cuda()
    proper = torch.tensor([r for r in range(rows) if not 40 <= r < 43], device="cuda")
    logp, entropy, m, ln, p, lp, d, has, e_ln, e_h = definition(torch, x[proper], labels[proper], classes)
    order = torch.sort(x.double() + 0.0, dim=1, descending=True, stable=True).indices
    for top in sorted({0, 1, min(3, classes), min(32, classes)}):
        r = ff.label_logprobs(x, labels, top=top)
        assert bool(((r.logp[proper].double() - logp).abs() <= torch.where(has, e_ln + 2 * U * (logp.abs() + ln), 0.0)).all())
        assert bool(((r.entropy[proper].double() - entropy).abs() <= e_h).all())
        assert torch.equal(r.stats[proper, 0].double(), m) and bool(((r.stats[proper, 1].double() - ln).abs() <= e_ln).all())
        assert torch.equal(r.top_index[proper].long(), order[proper, :top])
        want = lp.gather(1, order[proper, :top])
        got, tol = r.top_logp[proper].double(), e_ln[:, None] + 2 * U * (want.abs() + ln[:, None])
        assert bool(((got == want) | ((got - want).abs() <= tol)).all())
        odd = slice(40, 43)
        assert bool(r.entropy[odd].isnan().all()) and bool(r.stats[odd, 1].isnan().all()) and bool(r.top_logp[odd].isnan().all())
        assert bool(((r.top_index[odd] >= 0) & (r.top_index[odd] < classes)).all())
        for one in r.top_index[odd].tolist():
            assert len(set(one)) == top
    g = torch.rand(rows, generator=gen).cuda()
    dx = ff.label_logprobs_backward(x, labels, r.stats, g)[proper].double()
    a = torch.where(has, g[proper].double(), 0.0)[:, None]
    q = torch.where(p > 0, (d - r.stats[proper, 1:].double()).exp(), 0.0)
    want = -q * a
    want[has, labels[proper][has].long()] += a[has, 0]
    tol = q * a * (2 * EXP + 4 * U * (d.abs() + ln[:, None]) + 6 * U) + U * a + want.abs() * (torch.finfo(dt).eps / 2)
    assert bool(((dx - want).abs() <= tol + 2.0 ** -120).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(4100, 3001), (1900, 5001), (2000, 997), (1600, 2500), (750, 9000), (720, 700), (300, 1500)])
def test_many_rows(size, dtype):
    """One, two, four and eight warps a row; every other row of few values, one of them with a mask."""
    torch = torch_cuda()
    ff = lib_ready()
    rows, classes = size
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, labels = logits_of(torch, rows, classes, dt, classes % 4, 0.0)
    x[::2] = (x[::2].float() * 2).round().to(dt) / 2
    x[4, 9:] = float("-inf")
    labels[4] = 3
    logp, entropy, m, ln, p, lp, d, has, e_ln, e_h = definition(torch, x, labels, classes, threads=32)
    order = torch.sort(x.double(), dim=1, descending=True, stable=True).indices
    for top in (0, 3, 16, 20, 32):
        r = ff.label_logprobs(x, labels, top=top)
        assert bool(((r.logp.double() - logp).abs() <= torch.where(has, e_ln + 2 * U * (logp.abs() + ln), 0.0)).all())
        assert bool(((r.entropy.double() - entropy).abs() <= e_h).all())
        assert torch.equal(r.stats[:, 0].double(), m) and bool(((r.stats[:, 1].double() - ln).abs() <= e_ln).all())
        assert torch.equal(r.top_index.long(), order[:, :top])
        want = lp.gather(1, order[:, :top])
        tol = e_ln[:, None] + 2 * U * (want.abs() + ln[:, None])
        assert bool(((r.top_logp.double() == want) | ((r.top_logp.double() - want).abs() <= tol)).all())


def test_sorted_rows():
    torch = torch_cuda()
    ff = lib_ready()
    for classes in (3000, 70000):
        up = torch.arange(classes, dtype=torch.float32, device="cuda")[None] / 1000
        r = ff.label_logprobs(torch.cat((up, up.flip(1))), None, top=32)
        ref = torch.arange(32, device="cuda")
        assert torch.equal(r.top_index[0].long(), classes - 1 - ref) and torch.equal(r.top_index[1].long(), ref)
        assert r.logp is None


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("classes", [50, 5000, 140000])
def test_masks_that_leave_little(classes, dtype):
    """One class left, none left, all at the type's lowest value, an infinity, a NaN."""
    torch = torch_cuda()
    ff = lib_ready()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    low = torch.finfo(dt).min
    x = torch.full((8, classes), float("-inf"), dtype=dt, device="cuda")
    x[0, classes - 3] = 2.0
    x[2] = low
    x[3] = low
    x[3, 7] = -5.0
    x[4] = 1.0
    x[4, 9] = float("inf")
    x[5] = 1.0
    x[5, classes // 2] = float("nan")
    x[6] = 1.0
    x[7, 0], x[7, 1] = low, low
    labels = torch.tensor([classes - 3, 0, 1, 7, 9, 0, 3, 1], dtype=torch.int32, device="cuda")
    r = ff.label_logprobs(x, labels, top=3)
    logn, half = np.log(classes), np.log(2.0)
    for row, logp, entropy in ((0, 0.0, 0.0), (2, -logn, logn), (3, 0.0, 0.0), (6, -logn, logn), (7, -half, half)):
        # sums of equal terms: chain roundings as above, then one logarithm
        tol = (classes // 256 + 60) * U + 14 * EXP + 4 * U * logn
        assert abs(float(r.logp[row]) - logp) <= tol and abs(float(r.entropy[row]) - entropy) <= 2 * tol
    assert r.top_index[0].tolist() == [classes - 3, 0, 1] and r.top_index[3].tolist() == [7, 0, 1]
    assert r.top_index[2].tolist() == [0, 1, 2] and r.top_index[7].tolist() == [0, 1, 2]
    assert r.top_logp[0].tolist() == [0.0, float("-inf"), float("-inf")]
    for row in (1, 4, 5):
        assert bool(r.logp[row].isnan()) and bool(r.entropy[row].isnan()) and bool(r.stats[row, 1].isnan())
        assert bool(((r.top_index[row] >= 0) & (r.top_index[row] < classes)).all())
    assert float(r.stats[1, 0]) == float("-inf")
    ones = torch.ones(8, device="cuda")
    labels[1] = labels[4] = -1
    dx = ff.label_logprobs_backward(x, labels, r.stats, ones)
    assert bool((dx[1] == 0).all()) and bool((dx[4] == 0).all()) and bool((dx[0] == 0).all())
    assert bool(dx[5].isnan().all()) and bool(torch.isfinite(dx[[2, 3, 6, 7]]).all())
    ge = torch.zeros(8, device="cuda")
    ge[0] = 1.0
    dx = ff.label_logprobs_backward(x, None, r.stats, None, entropy=r.entropy, dentropy=ge)
    assert bool((dx == 0).all())


def test_gradient_follows_differences():
    torch = torch_cuda()
    ff = lib_ready()
    gen = torch.Generator().manual_seed(5)
    x = torch.randn(4, 30, generator=gen).cuda()
    labels = torch.tensor([3, -1, 29, 0], dtype=torch.int32, device="cuda")
    g, ge = torch.randn(4, generator=gen).cuda(), torch.randn(4, generator=gen).cuda()
    r = ff.label_logprobs(x, labels)
    dx = ff.label_logprobs_backward(x, labels, r.stats, g, entropy=r.entropy, dentropy=ge)

    def loss(v):
        lp = torch.log_softmax(v, 1)
        picked = torch.where(labels >= 0, lp.gather(1, labels.clamp(min=0).long()[:, None])[:, 0], 0.0)
        return (g.double() * picked - ge.double() * (lp.exp() * lp).sum(1)).sum()

    for k in range(0, 120, 7):
        hi, lo = x.double(), x.double()
        hi.view(-1)[k] += 1e-5
        lo.view(-1)[k] -= 1e-5
        slope = float(loss(hi) - loss(lo)) / 2e-5
        assert abs(slope - float(dx.view(-1)[k])) <= 1e-5 * (1 + abs(slope))


def test_in_place_strided_and_replayed():
    torch = torch_cuda()
    ff = lib_ready()
    x, labels = logits_of(torch, 60, 5001, torch.bfloat16, 0)
    g = torch.rand(60, device="cuda")
    r = ff.label_logprobs(x, labels)
    want = ff.label_logprobs_backward(x, labels, r.stats, g)
    for pad, lead in ((3, 1), (7, 0), (8, 8)):
        buf = torch.full((lead + 60 * (5001 + pad) + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
        view = buf[lead:lead + 60 * (5001 + pad)].view(60, 5001 + pad)[:, :5001]
        assert torch.equal(ff.label_logprobs_backward(x, labels, r.stats, g, out=view), want)
        view.fill_(7.0)
        assert bool((buf == 7.0).all())
    a = x.clone()
    assert torch.equal(ff.label_logprobs_backward(a, labels, r.stats, g, out=a), want)
    logits = torch.randn(2, 60000, device="cuda")
    two = labels[:2].contiguous()
    ff.label_logprobs(logits, two, top=9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = ff.label_logprobs(logits, two, top=9)
    logits.normal_()
    graph.replay()
    now = ff.label_logprobs(logits, two, top=9)
    for name in ff.LabelLogprobs.__slots__:
        assert torch.equal(getattr(held, name), getattr(now, name))


def test_empty_and_refusals():
    torch = torch_cuda()
    ff = lib_ready()
    x, l = torch.randn(4, 64, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    r = ff.label_logprobs(x[:0], l[:0], top=4)
    assert r.logp.shape == (0,) and r.top_index.shape == (0, 4)
    assert ff.label_logprobs_backward(x[:0], l[:0], r.stats, r.logp).shape == (0, 64)
    r, g = ff.label_logprobs(x, l), torch.ones(4, device="cuda")
    for bad, call in ((TypeError, lambda: ff.label_logprobs(x.half(), l)), (TypeError, lambda: ff.label_logprobs(x, l.long())),
                      (ValueError, lambda: ff.label_logprobs(x, l[:3])), (ValueError, lambda: ff.label_logprobs(x, l, top=33)),
                      (ValueError, lambda: ff.label_logprobs(x[:, :5], l, top=6)), (ValueError, lambda: ff.label_logprobs(x, l, top=-1)),
                      (ValueError, lambda: ff.label_logprobs(x.cpu(), l)), (ValueError, lambda: ff.label_logprobs(x.t(), l)),
                      (ValueError, lambda: ff.label_logprobs_backward(x, None, r.stats, g)),
                      (ValueError, lambda: ff.label_logprobs_backward(x, l, None, g)),
                      (ValueError, lambda: ff.label_logprobs_backward(x, l, r.stats, g[:2])),
                      (ValueError, lambda: ff.label_logprobs_backward(x, l, r.stats, g, dentropy=g)),
                      (ValueError, lambda: ff.label_logprobs_backward(x, l, r.stats, g, out=x[:2]))):
        with pytest.raises(bad):
            call()
