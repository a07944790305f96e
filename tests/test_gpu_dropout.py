"""Dropout against its definition: the mask bit by bit from the generator that
synth defines, the values to one fp32 rounding (|err| <= 2^-23 (|scaled x| +
|residual|)) and, for bf16, one bf16 rounding more (2^-8 of the value)."""

import numpy as np
import pytest

from paper_2404_08573_gb300 import synth

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu


def keep_mask(seed, offset, rows, cols, p):
    words = -(-cols // 4)
    w = synth.raw_u64(seed, 7, offset, rows * words)
    bits = np.stack([(w >> np.uint64(16 * e)) & np.uint64(0xFFFF) for e in range(4)], axis=1)
    return bits.reshape(rows, words * 4)[:, :cols] >= round(p * 65536)


def reference(x, res, keep, p):
    t = round(p * 65536)
    y = np.where(keep, x * (65536.0 / (65536 - t)) if t < 65536 else 0.0, 0.0)
    return y if res is None else y + res


def strided(torch, t, pad, lead):
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + lead,), float("nan"), dtype=t.dtype, device="cuda")
    view = buf[lead:].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view


SIZES = [(1, 1), (1, 3), (3, 5), (128, 500), (7, 1999), (64, 2000), (5, 4096), (1000, 8), (33, 17), (2, 100003), (4001, 31)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES)
def test_against_the_definition(size, dtype):
    torch = torch_cuda()
    ff = lib_ready()
    rows, cols = size
    k = SIZES.index(size)
    p = (0.1, 0.5, 0.0, 0.9)[k % 4]
    pad, lead = ((0, 0), (8, 0), (3, 1), (0, 4), (4, 8))[k % 5]
    seed, offset = 12345 + k, (0, 7, 1 << 33, (1 << 62) + 5)[k % 4]
    gen = torch.Generator().manual_seed(k)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, res = (torch.randn(rows, cols, generator=gen).to(dt) for _ in range(2))
    keep = keep_mask(seed, offset, rows, cols, p)
    for r in (None, res):
        got = ff.dropout(strided(torch, x, pad, lead), p, seed, offset,
                         residual=None if r is None else strided(torch, r, lead, pad))
        ref = reference(x.double().numpy(), None if r is None else r.double().numpy(), keep, p)
        tol = 2.0 ** -23 * (np.abs(reference(np.abs(x.double().numpy()), None, keep, p)) +
                            (0 if r is None else np.abs(r.double().numpy())))
        tol = tol + (2.0 ** -8 if dtype == "bf16" else 0.0) * np.abs(ref)
        g = got.double().cpu().numpy()
        assert np.all(np.abs(g - ref) <= tol)
        base = np.zeros_like(ref) if r is None else r.double().numpy()
        assert np.array_equal(g[~keep], base[~keep])  # what is dropped is exactly the residual


def test_gradient_is_the_same_mask():
    """y is linear in x: the derivative of sum w . y along v is the difference
    of two calls (exact here: small integers), and equals sum dropout(w) . v."""
    torch = torch_cuda()
    ff = lib_ready()
    gen = torch.Generator().manual_seed(1)
    x, v, w = (torch.randint(-8, 9, (37, 203), generator=gen).float().cuda() for _ in range(3))
    p, seed, off = 0.5, 99, 1234
    r = torch.zeros_like(x)
    f = [ff.dropout(t, p, seed, off, residual=r).double() for t in (x + v, x - v)]
    diff = ((f[0] - f[1]) / 2 * w.double()).sum()
    grad = ff.dropout(w, p, seed, off)
    assert float(diff) == float((grad.double() * v.double()).sum())


def test_dropped_values_do_not_leak():
    """NaN and infinities under the mask leave zeros (or the residual) behind."""
    torch = torch_cuda()
    ff = lib_ready()
    keep = torch.from_numpy(keep_mask(5, 0, 64, 333, 0.5)).cuda()
    x = torch.ones(64, 333, device="cuda")
    for bad in (float("nan"), float("inf"), -float("inf"), torch.finfo(torch.float32).min):
        y = ff.dropout(torch.where(keep, x, bad), 0.5, 5)
        assert torch.equal(y, torch.where(keep, 2.0, 0.0))
    for dt in (torch.float32, torch.bfloat16):
        x = torch.full((8, 64), float("nan"), device="cuda", dtype=dt)
        assert torch.equal(ff.dropout(x, 1.0, 3), torch.zeros_like(x))
        x = torch.randn(8, 64, device="cuda").to(dt)
        assert torch.equal(ff.dropout(x, 0.0, 3), x)


def test_masks_of_apart_offsets_and_their_rate():
    """The kept share of n = 2^20 draws lies within 6 standard deviations of 1 - p; masks dropout_words apart, and of
    another seed, agree as independent ones do."""
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.ones(1024, 1024, device="cuda")
    step = ff.dropout_words(1024, 1024)
    assert step == 1024 * 256
    p, n = 0.3, 1 << 20
    masks = [ff.dropout(x, p, 7, 0) > 0, ff.dropout(x, p, 7, step) > 0, ff.dropout(x, p, 8, 0) > 0]
    for m in masks:
        assert abs(float(m.float().mean()) - (1 - p)) <= 6 * (p * (1 - p) / n) ** 0.5
    agree = (1 - p) ** 2 + p ** 2
    for i, j in ((0, 1), (0, 2), (1, 2)):
        assert abs(float((masks[i] == masks[j]).float().mean()) - agree) <= 6 * (agree * (1 - agree) / n) ** 0.5


def test_in_place_streams_and_a_captured_graph():
    torch = torch_cuda()
    ff = lib_ready()
    x = torch.randn(300, 777, device="cuda").bfloat16()
    r = torch.randn(300, 777, device="cuda").bfloat16()
    want = ff.dropout(x, 0.2, 4, 50, residual=r)
    a, b = x.clone(), r.clone()
    assert torch.equal(ff.dropout(a, 0.2, 4, 50, residual=r, out=a), want)
    assert torch.equal(ff.dropout(x, 0.2, 4, 50, residual=b, out=b), want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = ff.dropout(x, 0.2, 4, 50, residual=r, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    # the offset lives on the device, so every replay draws its own mask
    off = torch.zeros(1, dtype=torch.int64, device="cuda")
    static = torch.empty_like(x)
    ff.dropout(x, 0.2, 4, off, residual=r, out=static)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ff.dropout(x, 0.2, 4, off, residual=r, out=static)
        off += ff.dropout_words(300, 777)
    off.fill_(50)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(static, ff.dropout(x, 0.2, 4, 50 + k * ff.dropout_words(300, 777), residual=r))
    assert int(off) == 50 + 3 * ff.dropout_words(300, 777)


def test_more_than_2_to_32_elements():
    """Element indices past 32 bits: the last rows of a matrix of 2^32 + 2^21 elements."""
    torch = torch_cuda()
    ff = lib_ready()
    rows, cols = 2049, 1 << 21
    x = torch.ones(rows, cols, device="cuda", dtype=torch.bfloat16)
    ff.dropout(x, 0.5, 11, 3, out=x)
    for row in (0, 2047, 2048):
        keep = torch.from_numpy(keep_mask(11, 3 + row * (cols // 4), 1, cols, 0.5))
        assert torch.equal(x[row].cpu() > 0, keep[0])


def test_empty_and_refused():
    torch = torch_cuda()
    ff = lib_ready()
    assert ff.dropout(torch.empty(0, 5, device="cuda"), 0.5, 1).shape == (0, 5)
    assert ff.dropout(torch.empty(5, 0, device="cuda"), 0.5, 1).shape == (5, 0)
    x = torch.randn(6, 8, device="cuda")
    for bad in (x.cpu(), x.half(), x.t(), x[:1].expand(6, 8)):
        with pytest.raises((TypeError, ValueError)):
            ff.dropout(bad, 0.5, 1)
    for kw in (dict(residual=x.bfloat16()), dict(residual=x[:3]), dict(out=x[:, :4]), dict(offset=torch.zeros(1)),
               dict(offset=torch.zeros(2, dtype=torch.int64, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            ff.dropout(x, 0.5, 1, **kw)
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(ff.FFError):
            ff.dropout(x, p, 1)
