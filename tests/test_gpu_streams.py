"""Calls on a stream that is not the current one: their buffers are nobody
else's.  The current stream is made to lag behind with work on blocks that the
caller has already freed; a call on another stream that was handed one of them
would see it overwritten, or overwrite what the lagging work reads."""

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu


def flat(r):
    if isinstance(r, (tuple, list)):
        return [t for v in r for t in flat(v)]
    return [r.q, r.scale] if hasattr(r, "scale") else [r]


def check(call, blocks=()):
    """call(stream) gives the same outputs on a side stream while the current one still fills and reads freed blocks of
    the outputs' sizes and of `blocks` (bytes)."""
    torch = torch_cuda()
    side = torch.cuda.Stream()
    want = [t.clone() for t in flat(call(None))]
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    sizes = [t.numel() * t.element_size() for t in want] + list(blocks)
    temps = [torch.zeros(s, dtype=torch.uint8, device="cuda") for s in sizes]
    seen = [torch.empty_like(t) for t in temps]
    torch.cuda.synchronize()
    for _ in range(50):
        big = (big @ big) * 1e-4
    for t, s in zip(temps, seen):
        t.fill_(7)
        s.copy_(t)
        t.fill_(255)
    del t, s, temps
    got = call(side)
    side.synchronize()
    early = [t.clone() for t in flat(got)]  # behind the lagging work: what is left once it is done
    torch.cuda.synchronize()
    for p, q in zip(early, want):
        assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))
    for s in seen:
        assert bool((s == 7).all())


def inputs(torch, *shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda()


@pytest.mark.parametrize("shape", [(700, 1, 500, 10), (2, 30000, 16, 2)])
def test_group_norm(shape):
    torch = torch_cuda()
    ff = lib_ready()
    n, S, C, G = shape
    x = inputs(torch, n, S, C)
    _, m, r = ff.group_norm_act(x, None, None, G)
    work = [ff.lib().ff_group_norm_workspace(n, S, C, G, 0, b) for b in (0, 1)]
    check(lambda s: ff.group_norm_act(x, None, None, G, stream=s), work[:1])
    check(lambda s: ff.group_norm_act_backward(x, x, m, r, None, None, G, stream=s), work[1:])


def test_dropout_and_8_bit():
    torch = torch_cuda()
    ff = lib_ready()
    x, w = inputs(torch, 500, 784), inputs(torch, 300, 784, seed=1)
    a, b = ff.fp8_quantize(x), ff.fp8_quantize(w, tile=True)
    check(lambda s: ff.dropout(x, 0.3, 5, stream=s))
    check(lambda s: ff.fp8_quantize_both(x, stream=s))
    check(lambda s: ff.fp8_matmul(a, b, out_dtype=torch.float32, stream=s))


def test_inputs_freed_after_the_call():
    """The call's stream lags; the input is freed and its block filled on the current stream."""
    torch = torch_cuda()
    ff = lib_ready()
    x = inputs(torch, 500, 784)
    want = ff.dropout(x, 0.3, 5)
    big = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(50):
            big = (big @ big) * 1e-4
    got = ff.dropout(x, 0.3, 5, stream=side)
    del x
    for _ in range(8):
        torch.full((500, 784), 9.0, device="cuda")
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_stream_given_by_its_number():
    torch = torch_cuda()
    ff = lib_ready()
    x = inputs(torch, 64, 100)
    want = ff.dropout(x, 0.3, 5)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = ff.dropout(x, 0.3, 5, stream=side.cuda_stream)
    with torch.cuda.stream(side):
        back = ff.dropout(x, 0.3, 5, stream=0)  # the default stream, from another one
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(back, want)


def test_labels_and_predictions():
    torch = torch_cuda()
    ff = lib_ready()
    from paper_2404_08573_gb300 import synth
    layers = [ff.Layer(784, 256, prec="bf16", init_seed=3), ff.Layer(256, 136, prec="bf16", init_seed=4)]
    x = torch.from_numpy(synth.mnist_like(3000, seed=20)).cuda()
    y = torch.from_numpy(synth.labels(3000, seed=21)).cuda()
    head, block = ff.Head(136, lr=1e-3, max_rows=512), ff.Head(136, lr=1e-3)
    check(lambda s: ff.overlay_label(x, y, stream=s))
    check(lambda s: ff.predict(layers, x, stream=s)[0])
    check(lambda s: ff.adaptive_negatives(layers, x, y, stream=s)[0])
    check(lambda s: head.predict(layers, x, stream=s)[0])
    check(lambda s: ff.po_predict(layers, block, x, stream=s)[0])
