"""Layer operators without a GPU: the C entries refuse bad arguments on the
host, before anything is enqueued, and size helpers follow their formulas."""

import ctypes

import pytest
import torch

from .gpu_common import lib_ready

# The addresses are invented: where a GPU could act on a call that is not
# refused, nothing here runs.
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="invented addresses: without a GPU only")

P = 4096  # a 16-byte aligned address that no refused call may touch
OK, BAD = 0, 1


@pytest.fixture(scope="module")
def L():
    return lib_ready().lib()


def norm(L, x=P, ldx=8, n=2, spatial=1, channels=8, groups=2, gamma=P, beta=P, eps=1e-5, act=2, prec=1, y=P, ldy=8,
         mean=P, rstd=P, ws=P, ws_bytes=1 << 30):
    return L.ff_group_norm_act(x, ldx, n, spatial, channels, groups, gamma, beta, eps, act, prec, y, ldy, mean, rstd, ws,
                               ws_bytes, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(n=-1), dict(spatial=-1), dict(channels=0), dict(groups=0), dict(groups=3),
    dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(act=3), dict(act=-1),
    dict(prec=2), dict(ldx=7), dict(ldy=7), dict(mean=None), dict(rstd=None), dict(x=P + 1), dict(y=P + 1)])
def test_group_norm_refuses(L, bad):
    assert norm(L, **bad) == BAD


def test_group_norm_workspace_is_checked(L):
    need = L.ff_group_norm_workspace(2, 50000, 8, 2, 1, 0)
    assert need >= 0
    if need:
        assert norm(L, spatial=50000, ws=None) == BAD
        assert norm(L, spatial=50000, ws_bytes=need - 1) == BAD
        assert norm(L, spatial=50000, ws=P + 8) == BAD
    assert L.ff_group_norm_workspace(2, 4, 8, 3, 1, 0) == -1
    assert L.ff_group_norm_workspace(0, 4, 8, 2, 1, 1) == 0


def test_empty_norms_need_no_buffers(L):
    assert norm(L, n=0, x=None, y=None, ws=None, ws_bytes=0) == OK
    assert L.ff_group_norm_act_backward(None, 8, None, 8, 0, 1, 8, 2, None, None, None, None, 2, 1, None, 8, None, None,
                                        None, 0, None) == OK


def grad(L, dy=P, lddy=8, x=P, ldx=8, n=2, spatial=1, channels=8, groups=2, mean=P, rstd=P, act=2, prec=1, dx=P, lddx=8,
         dgamma=P, dbeta=P, ws=P, ws_bytes=1 << 30):
    return L.ff_group_norm_act_backward(dy, lddy, x, ldx, n, spatial, channels, groups, mean, rstd, None, None, act,
                                        prec, dx, lddx, dgamma, dbeta, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", [
    dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dgamma=None), dict(dbeta=None), dict(groups=3),
    dict(lddy=7), dict(ldx=7), dict(lddx=7), dict(act=9), dict(prec=5), dict(dx=P + 1)])
def test_group_norm_backward_refuses(L, bad):
    assert grad(L, **bad) == BAD


def test_group_norm_backward_without_outputs_is_a_no_op(L):
    assert grad(L, dx=None, dgamma=None, dbeta=None) == OK


def drop(L, x=P, ldx=8, rows=2, cols=8, p=0.5, offset_dev=None, residual=None, ldr=8, prec=1, y=P, ldy=8):
    return L.ff_dropout(x, ldx, rows, cols, p, 1, 0, offset_dev, residual, ldr, prec, y, ldy, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(rows=-1), dict(cols=-1), dict(p=-0.1), dict(p=1.1), dict(p=float("nan")),
    dict(prec=2), dict(ldx=7), dict(ldy=7), dict(residual=P, ldr=7), dict(residual=P + 1), dict(offset_dev=P + 4),
    dict(x=P + 1), dict(rows=1 << 61, cols=64, ldx=64, ldy=64)])
def test_dropout_refuses(L, bad):
    assert drop(L, **bad) == BAD


def test_dropout_sizes(L):
    assert drop(L, rows=0, x=None, y=None) == OK and drop(L, cols=0, x=None, y=None) == OK
    assert [L.ff_dropout_words(r, c) for r, c in ((3, 4), (3, 5), (0, 5), (2, 0), (1 << 20, 1 << 20))] == [
        3, 6, 0, 0, 1 << 38]


def quantize(L, x=P, ldx=32, rows=2, k=32, prec=1, blocks=0, q=P, scale=P, qt=P, scale_t=P):
    return L.ff_fp8_quantize(x, ldx, rows, k, prec, blocks, q, scale, qt, scale_t, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(rows=-1), dict(k=0), dict(prec=2), dict(blocks=2), dict(ldx=31), dict(q=None), dict(scale=None),
    dict(qt=None), dict(scale_t=None), dict(q=None, scale=None, qt=None, scale_t=None), dict(q=P + 8), dict(qt=P + 8),
    dict(scale=P + 2), dict(scale_t=P + 1), dict(x=P + 1)])
def test_quantize_refuses(L, bad):
    assert quantize(L, **bad) == BAD


def matmul(L, a=P, a_scale=P, b=P, b_scale=P, blocks=1, m=4, n=8, k=32, bias=None, prec=1, c=P, ldc=8, status=None):
    return L.ff_fp8_matmul(a, a_scale, b, b_scale, blocks, m, n, k, bias, 0, prec, c, ldc, status, None)


@pytest.mark.parametrize("bad", [
    dict(a=None), dict(a_scale=None), dict(b=None), dict(b_scale=None), dict(c=None), dict(m=-1), dict(n=-1), dict(k=0),
    dict(blocks=2), dict(prec=2), dict(ldc=7), dict(a=P + 8), dict(b=P + 1), dict(a_scale=P + 2), dict(c=P + 1),
    dict(bias=P + 2), dict(status=P + 2)])
def test_matmul_refuses(L, bad):
    assert matmul(L, **bad) == BAD


def test_empty_8_bit_calls_are_no_ops(L):
    assert quantize(L, rows=0, x=None) == OK
    assert matmul(L, m=0, a=None, c=None) == OK and matmul(L, n=0, b=None, c=None) == OK
    assert [L.ff_fp8_stride(k) for k in (0, 1, 16, 17, 2000, 1337)] == [0, 16, 16, 32, 2000, 1344]
