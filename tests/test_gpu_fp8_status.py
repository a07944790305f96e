"""A timed-out wait of an 8-bit product is reported, also where the caller gives no status word."""

import pytest

from .gpu_common import lib_ready, torch_cuda

pytestmark = pytest.mark.gpu


def test_a_timeout_is_reported_without_a_status_word():
    """A bounded wait that nothing ends, latched where the products latch theirs."""
    torch = torch_cuda()
    ff = lib_ready()
    a, b = ff.fp8_quantize(torch.ones(40, 300, device="cuda")), ff.fp8_quantize(torch.ones(50, 300, device="cuda"), tile=True)
    ff.fp8_check()
    ff.fp8_selftest_wait(2000)
    with pytest.raises(ff.FFError) as e:
        ff.fp8_check()
    assert e.value.status == 4  # FF_ERR_TIMEOUT
    ff.fp8_check()  # cleared
    c = ff.fp8_matmul(a, b)
    ff.fp8_check()
    assert bool((c == 300).all())
    with pytest.raises(ff.FFError):
        ff.fp8_selftest_wait(0)


def test_the_word_outlives_a_captured_graph():
    torch = torch_cuda()
    ff = lib_ready()
    a, b = ff.fp8_quantize(torch.ones(1, 300, device="cuda")), ff.fp8_quantize(torch.ones(50, 300, device="cuda"), tile=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = ff.fp8_matmul(a, b)
    ff.fp8_selftest_wait(2000)
    graph.replay()  # does not clear what was latched
    with pytest.raises(ff.FFError):
        ff.fp8_check()
    graph.replay()
    ff.fp8_check()
    assert bool((c == 300).all())
