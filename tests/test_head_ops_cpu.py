"""The operators of a deep head without a GPU: the C entries refuse bad arguments
on the host, before anything is enqueued, and size helpers follow their formulas."""

import ctypes

import pytest
import torch

from .gpu_common import lib_ready

# The addresses are invented: where a GPU could act on a call that is not
# refused, nothing here runs.
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="invented addresses: without a GPU only")

P = 4096  # a 16-byte aligned address that no refused call may touch
OK, BAD = 0, 1
BIG = 0x7FFFFF01


@pytest.fixture(scope="module")
def L():
    return lib_ready().lib()


def rms(L, x=P, ldx=8, r=None, ldr=8, rows=2, cols=8, gamma=P, eps=1e-5, prec=1, h=None, ldh=8, y=P, ldy=8, q=None, scale=None,
        rstd=P):
    return L.ff_rms_norm(x, ldx, r, ldr, rows, cols, gamma, eps, prec, h, ldh, y, ldy, q, scale, rstd, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(rows=-1), dict(cols=0), dict(cols=BIG), dict(eps=0.0), dict(eps=-1.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(prec=2), dict(ldx=7), dict(ldy=7), dict(r=P), dict(h=P),
    dict(r=P, h=P, ldr=7), dict(r=P, h=P, ldh=7), dict(r=P, h=P), dict(q=P), dict(scale=P), dict(q=P + 8, scale=P), dict(q=P, scale=P + 2),
    dict(x=P + 1), dict(y=P + 1), dict(gamma=P + 2), dict(rstd=P + 2)])
def test_rms_norm_refuses(L, bad):
    assert rms(L, **bad) == BAD


def rms_grad(L, dy=P, lddy=8, h=P, ldh=8, rows=2, cols=8, rstd=P, gamma=P, dh=None, lddh=8, prec=1, dx=P, lddx=8, dgamma=P, ws=P,
             ws_bytes=1 << 30):
    return L.ff_rms_norm_backward(dy, lddy, h, ldh, rows, cols, rstd, gamma, dh, lddh, prec, dx, lddx, dgamma, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [
    dict(dy=None), dict(h=None), dict(rstd=None), dict(rows=-1), dict(cols=0), dict(prec=2), dict(lddy=7), dict(ldh=7), dict(lddx=7),
    dict(dh=P, lddh=7), dict(dx=P + 1), dict(dy=P + 1), dict(dgamma=P + 2), dict(rstd=P + 2), dict(rows=1000, ws=None),
    dict(rows=1000, ws_bytes=8), dict(rows=1000, ws=P + 8)])
def test_rms_norm_backward_refuses(L, bad):
    assert rms_grad(L, **bad) == BAD


def test_rms_norm_sizes(L):
    assert rms(L, rows=0, x=None, y=None) == OK and rms_grad(L, dx=None, dgamma=None) == OK
    assert rms_grad(L, rows=0, dy=None, h=None, rstd=None, dgamma=None) == OK
    assert [L.ff_rms_norm_workspace(r, c) for r, c in ((0, 8), (1, 8), (-1, 8), (1, 0), (1, BIG))] == [0, 0, -1, -1, -1]
    assert L.ff_rms_norm_workspace(1, 20000) >= 4 and L.ff_rms_norm_workspace(4096, 8192) % 16 == 0


def logprobs(L, x=P, ld=8, rows=2, classes=8, prec=1, labels=P, logp=P, entropy=P, top=2, top_logp=P, top_index=P, stats=P):
    return L.ff_label_logprobs(x, ld, rows, classes, prec, labels, logp, entropy, top, top_logp, top_index, stats, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(rows=-1), dict(classes=0), dict(classes=BIG), dict(prec=2), dict(ld=7), dict(labels=None), dict(top=-1),
    dict(top=9), dict(top=33, classes=40, ld=40), dict(top_logp=None), dict(top_index=None), dict(x=P + 1), dict(labels=P + 2),
    dict(logp=P + 2), dict(entropy=P + 1), dict(top_logp=P + 2), dict(top_index=P + 2), dict(stats=P + 4)])
def test_label_logprobs_refuses(L, bad):
    assert logprobs(L, **bad) == BAD


def logprobs_grad(L, x=P, ld=8, rows=2, classes=8, prec=1, labels=P, stats=P, dlogp=P, entropy=None, dentropy=None, dx=P, lddx=8):
    return L.ff_label_logprobs_backward(x, ld, rows, classes, prec, labels, stats, dlogp, entropy, dentropy, dx, lddx, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(dx=None), dict(stats=None), dict(rows=-1), dict(classes=0), dict(prec=2), dict(ld=7), dict(lddx=7),
    dict(labels=None), dict(dentropy=P), dict(x=P + 1), dict(dx=P + 1), dict(stats=P + 4), dict(dlogp=P + 2),
    dict(entropy=P + 2, dentropy=P), dict(entropy=P, dentropy=P + 2)])
def test_label_logprobs_backward_refuses(L, bad):
    assert logprobs_grad(L, **bad) == BAD


# rows of 8 bf16 values are 16 bytes: two rows at P end at P + 32 (apart by 16: 48)
@pytest.mark.parametrize("call,shared", [
    (rms, dict(y=P + 16)), (rms, dict(y=P + 2)), (rms, dict(y=P, ldy=16)), (rms, dict(x=P, ldx=16, y=P + 8, ldy=16)),
    (rms, dict(x=P, ldx=16, y=P + 30, ldy=16)), (rms, dict(rows=1, y=P + 8)),
    (rms, dict(x=P + 4096, r=P, h=P + 16, y=P + 8192)), (rms, dict(x=P, r=P + 4096, h=P + 16, y=P + 8192)),
    (rms, dict(x=P + 4096, r=P, h=P + 8192, y=P + 16)), (rms, dict(x=P + 4096, r=P + 8192, h=P, y=P + 16)),
    (rms, dict(x=P, ldx=16, r=P + 4096, h=P, ldh=8, y=P + 8192)), (rms_grad, dict(dx=P + 16, h=P + 4096)),
    (rms_grad, dict(dy=P + 4096, dx=P + 16)), (rms_grad, dict(dy=P + 4096, h=P + 8192, dh=P + 16)), (rms_grad, dict(lddx=16)),
    (logprobs_grad, dict(dx=P + 16)), (logprobs_grad, dict(lddx=16)), (logprobs_grad, dict(ld=16, dx=P + 14, lddx=16))])
def test_outputs_that_share_values_in_part_are_refused(L, call, shared):
    assert call(L, **shared) == BAD


def test_empty_logprobs(L):
    assert logprobs(L, rows=0, x=None) == OK and logprobs_grad(L, rows=0, x=None, dx=None, stats=None) == OK


def clip(L, grads, out, counts, precs=None, max_norm=1.0, norm=P, ws=P, ws_bytes=1 << 30):
    n = len(grads)
    precs = precs or [0] * n
    return L.ff_clip_grad_norm((ctypes.c_void_p * n)(*grads), (ctypes.c_void_p * n)(*out), (ctypes.c_longlong * n)(*counts),
                               (ctypes.c_int * n)(*precs), n, max_norm, norm, ws, ws_bytes, None)


def test_clip_refuses(L):
    Q = P + 4096
    for args in (dict(precs=[2]), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(norm=None), dict(norm=P + 2), dict(ws=None),
                 dict(ws=P + 8), dict(ws_bytes=64)):
        assert clip(L, [P], [P], [4], **args) == BAD
    for grads, out, counts in (([None], [P], [4]), ([P], [None], [4]), ([P + 2], [P + 2], [4]), ([P], [P], [-1]), ([P], [P], [1 << 61]),
                               ([P, P], [P, P], [4, 4]), ([P, P + 8], [P, P + 8], [4, 4]), ([P], [P + 8], [4]),
                               ([P, Q], [Q, P], [4, 4]), ([P, P], [Q, Q], [4, 4]), ([P, Q], [Q + 8, Q], [64, 4]),
                               ([P, P + 400], [P, Q], [101, 4])):
        assert clip(L, grads, out, counts) == BAD
    assert L.ff_clip_grad_norm(None, None, None, None, 1, 1.0, P, P, 1 << 30, None) == BAD
    assert L.ff_clip_grad_norm(None, None, None, None, -1, 1.0, P, P, 1 << 30, None) == BAD
    assert L.ff_clip_grad_norm_workspace(-1) == -1 and L.ff_clip_grad_norm_workspace(0) > 0
    assert L.ff_clip_grad_norm_workspace(1000) > L.ff_clip_grad_norm_workspace(100)


def quantize(L, x=P, ldx=32, rows=2, k=32, prec=1, q=P, scale=P, qt=P, scale_t=P):
    return L.ff_fp4_quantize(x, ldx, rows, k, prec, q, scale, qt, scale_t, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(rows=-1), dict(k=0), dict(k=BIG), dict(prec=2), dict(ldx=31), dict(q=None), dict(scale=None), dict(qt=None),
    dict(scale_t=None), dict(q=None, scale=None, qt=None, scale_t=None), dict(q=P + 8), dict(qt=P + 8), dict(scale=P + 4),
    dict(scale_t=P + 8), dict(x=P + 1)])
def test_fp4_quantize_refuses(L, bad):
    assert quantize(L, **bad) == BAD


def dequantize(L, q=P, scale=P, rows=2, k=32, prec=1, y=P, ldy=32):
    return L.ff_fp4_dequantize(q, scale, rows, k, prec, y, ldy, None)


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(scale=None), dict(y=None), dict(rows=-1), dict(k=0), dict(prec=2), dict(ldy=31), dict(q=P + 8),
    dict(scale=P + 8), dict(y=P + 1)])
def test_fp4_dequantize_refuses(L, bad):
    assert dequantize(L, **bad) == BAD


def matmul(L, a=P, sa=P, b=P, sb=P, m=4, n=8, k=32, bias=None, prec=1, c=P, ldc=8, status=None):
    return L.ff_fp4_matmul(a, sa, b, sb, m, n, k, bias, 0, prec, c, ldc, status, None)


@pytest.mark.parametrize("bad", [
    dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(c=None), dict(m=-1), dict(n=-1), dict(k=0), dict(k=BIG),
    dict(prec=2), dict(ldc=7), dict(a=P + 8), dict(b=P + 1), dict(sa=P + 8), dict(sb=P + 8), dict(c=P + 1), dict(bias=P + 2),
    dict(status=P + 2)])
def test_fp4_matmul_refuses(L, bad):
    assert matmul(L, **bad) == BAD


def test_fp4_sizes(L):
    assert quantize(L, rows=0, x=None) == OK and dequantize(L, rows=0, q=None, y=None) == OK
    assert matmul(L, m=0, a=None, c=None) == OK and matmul(L, n=0, b=None, c=None) == OK
    assert [L.ff_fp4_stride(k) for k in (0, 1, 32, 33, 2000, 1337)] == [0, 16, 16, 32, 1008, 672]
    assert [L.ff_fp4_scale_bytes(r, k) for r, k in ((0, 1), (1, 1), (128, 128), (129, 129), (2000, 784), (-1, 4), (4, 0))] == [
        0, 512, 512, 2048, 16 * 7 * 512, -1, -1]
