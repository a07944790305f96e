"""The gradient norm over many tensors and clipping, against the definition in 64 bits.

Tolerances.  u = 2^-24.  A thread adds at most 32 fp32 squares before they are
added up in 64 bits, so the sum is within 33 u of itself and the norm within 17 u
and its own rounding; a factor adds one rounding, a product one and the half step
of its type.
"""

import math

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SETS = {
    "one": [1], "few": [20000, 2000, 10, 2000], "pieces": [4096, 4097, 8192, 1, 12288], "full_cluster": [4096 * 64],
    "past_cluster": [4096 * 64 + 1], "large": [3_000_000, 17, 1_000_001], "many": [37 * i + 1 for i in range(250)],
    "very_many": [5] * 130, "empties": [0, 5, 0, 70000, 0],
}


def tensors(torch, counts, kind, lead=0):
    out = []
    for i, n in enumerate(counts):
        dt = {"bf16": torch.bfloat16, "fp32": torch.float32, "both": (torch.float32, torch.bfloat16)[i % 2]}[kind]
        t = torch.empty(n + lead, device="cuda", dtype=dt)[lead:]
        out.append(t.copy_(torch.randn(n, generator=torch.Generator().manual_seed(i)) * math.exp(-(i % 5))))
    return out


@pytest.mark.parametrize("kind", ["bf16", "fp32", "both"])
@pytest.mark.parametrize("name", list(SETS))
def test_norm_and_copies(name, kind):
    torch = torch_cuda()
    ff = lib_ready()
    for lead in (0, 1):
        g = tensors(torch, SETS[name], kind, lead)
        exact = math.sqrt(math.fsum(float(t.double().square().sum()) for t in g))
        for limit in (0.5 * exact, 2.0 * exact, 0.0, math.inf):
            keep = [t.clone() for t in g]
            out = [torch.full_like(t, 7.0) for t in g]
            norm = ff.clip_grad_norm(g, limit, out=out)
            assert norm.shape == (1,) and abs(float(norm) - exact) <= 20 * U * exact
            by = min(1.0, limit / exact)
            for t, k, o in zip(g, keep, out):
                assert torch.equal(t, k)
                want = k.double() * by
                tol = want.abs() * (22 * U + torch.finfo(t.dtype).eps / 2) + 2.0 ** -130
                assert bool(((o.double() - want).abs() <= tol).all())
                if by == 1.0:
                    assert torch.equal(o, k)
            mine = [k.clone() for k in keep]
            again = ff.clip_grad_norm(mine, limit)
            assert torch.equal(again, norm) and all(torch.equal(a, o) for a, o in zip(mine, out))


def test_shapes_streams_and_replays():
    torch = torch_cuda()
    ff = lib_ready()
    for sizes in ([(300, 784), (300,), (10, 300)], [(2000, 2000), (2000,), (3,)]):
        g = [torch.randn(*s, device="cuda") for s in sizes]
        out = [torch.empty_like(t) for t in g]
        ff.clip_grad_norm(g, 1.0, out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norm = ff.clip_grad_norm(g, 1.0, out=out)
        for t in g:
            t.normal_()
        graph.replay()
        other = [torch.empty_like(t) for t in g]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        n2 = ff.clip_grad_norm(g, 1.0, out=other, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(norm, n2) and all(torch.equal(a, b) for a, b in zip(out, other))


def test_norms_that_are_not_finite():
    torch = torch_cuda()
    ff = lib_ready()
    for n in (500, 400000):
        for value in (float("nan"), float("inf")):
            g = [torch.ones(n, device="cuda"), torch.ones(7, device="cuda")]
            g[0][n // 2] = value
            norm = ff.clip_grad_norm(g, 1.0)
            assert bool(norm.isnan()) if value != value else float(norm) == float("inf")
            assert bool(g[1].isnan().all()) if value != value else bool((g[1] == 0).all())
        g = [torch.zeros(n, device="cuda")]
        assert float(ff.clip_grad_norm(g, 0.0)) == 0.0 and bool((g[0] == 0).all())


def test_refusals():
    torch = torch_cuda()
    ff = lib_ready()
    a, b = torch.randn(100, device="cuda"), torch.randn(100, device="cuda")
    big = torch.randn(250, device="cuda")
    keep = [t.clone() for t in (a, b, big)]
    for bad, call in ((ValueError, lambda: ff.clip_grad_norm([], 1.0)), (ValueError, lambda: ff.clip_grad_norm([a, 3], 1.0)),
                      (TypeError, lambda: ff.clip_grad_norm([a, b.double()], 1.0)), (ValueError, lambda: ff.clip_grad_norm([a.cpu()], 1.0)),
                      (ValueError, lambda: ff.clip_grad_norm([a, b[::2]], 1.0)), (ff.FFError, lambda: ff.clip_grad_norm([a, a], 1.0)),
                      (ff.FFError, lambda: ff.clip_grad_norm([a], -1.0)), (ff.FFError, lambda: ff.clip_grad_norm([a], math.nan)),
                      (ff.FFError, lambda: ff.clip_grad_norm([big[:100], big[50:150]], 1.0)),
                      (ff.FFError, lambda: ff.clip_grad_norm([big[:100]], 1.0, out=[big[50:150]])),
                      (ff.FFError, lambda: ff.clip_grad_norm([a, b], 1.0, out=[b, a])),
                      (ff.FFError, lambda: ff.clip_grad_norm([a, b], 1.0, out=[big[:100], big[:100]])),
                      (ValueError, lambda: ff.clip_grad_norm([a], 1.0, out=[])), (ValueError, lambda: ff.clip_grad_norm([a], 1.0, out=[b[:50]]))):
        with pytest.raises(bad):
            call()
    assert all(torch.equal(t, k) for t, k in zip((a, b, big), keep))
    # the same gradients read twice into outputs of their own are fine
    out = [torch.empty_like(a), torch.empty_like(a)]
    ff.clip_grad_norm([a, a], math.inf, out=out)
    assert torch.equal(out[0], a) and torch.equal(out[1], a)
