"""Refusals of the adapter-training operators: before any GPU work, so without a GPU."""
import ctypes

import pytest

from paper_2012_10557_amd import binding

P = ctypes.c_void_p(4096)  # never read: the calls end at their checks
BIG = 1 << 40


def _groupnorm(precision=1, x=4096, N=2, HW=8, C=32, G=4, gamma=P, beta=P, eps=1e-5, act=0,
               y=1 << 20, mean=P, rstd=P, ws=P, nbytes=BIG):
    return binding.load().ekya_op_groupnorm(precision, x, N, HW, C, G, gamma, beta, eps, act, y,
                                            mean, rstd, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(precision=2), dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(N=-1),
    dict(HW=0), dict(C=0), dict(C=65537, G=1), dict(G=0), dict(G=5), dict(gamma=None),
    dict(beta=None), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(act=4),
    dict(act=-1), dict(x=4097), dict(y=4099), dict(y=4096 + 2), dict(ws=None), dict(nbytes=8),
    dict(ws=ctypes.c_void_p(4104)), dict(HW=1 << 36), dict(HW=1 << 62), dict(N=1 << 30, HW=1 << 30)])
def test_groupnorm_refuses(bad):
    assert _groupnorm(**bad) == binding.EKYA_ERR_INVALID_ARG
    assert binding.load().ekya_last_error(None)


def _groupnorm_backward(precision=1, dy=1 << 16, x=4096, N=2, HW=8, C=32, G=4, gamma=P, beta=P,
                        mean=P, rstd=P, act=0, dx=1 << 20, dgamma=P, dbeta=P, ws=P, nbytes=BIG):
    return binding.load().ekya_op_groupnorm_backward(precision, dy, x, N, HW, C, G, gamma, beta, mean,
                                                     rstd, act, dx, dgamma, dbeta, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(precision=-1), dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None),
    dict(rstd=None), dict(gamma=None), dict(dgamma=None), dict(dbeta=None), dict(G=3), dict(act=9),
    dict(dx=4096 + 16), dict(dx=(1 << 16) - 2), dict(dy=4097), dict(ws=None), dict(nbytes=0)])
def test_groupnorm_backward_refuses(bad):
    assert _groupnorm_backward(**bad) == binding.EKYA_ERR_INVALID_ARG


def test_no_samples_need_no_tensors():
    assert _groupnorm(N=0, x=None, y=None, mean=None, rstd=None, ws=None, nbytes=0) == binding.EKYA_OK
    lib = binding.load()
    assert lib.ekya_op_groupnorm_workspace(1, 0, 8, 32, 4) == 0
    assert lib.ekya_op_groupnorm_workspace(1, 2, 8, 32, 5) == 0
    assert lib.ekya_op_groupnorm_backward_workspace(7, 2, 8, 32, 4) == 0
    assert lib.ekya_op_groupnorm_workspace(1, 2, 8, 32, 4) > 0


def _adamw_tensor(**kw):
    t = dict(w=1 << 20, g=1 << 21, m=1 << 22, v=1 << 23, scale=None, low=1 << 24, n=1000,
             weight_decay=0.0)
    t.update(kw)
    return binding.AdamwTensor(**t)


def _adamw(tensors, prec=0, bits=32, count=None):
    h = ctypes.c_void_p()
    arr = (binding.AdamwTensor * max(1, len(tensors)))(*tensors)
    st = binding.load().ekya_adamw_create(ctypes.byref(h), arr, len(tensors) if count is None else count,
                                          prec, bits)
    assert (st == binding.EKYA_OK) == bool(h)
    return st, h


@pytest.mark.parametrize("bad", [
    dict(w=None), dict(g=None), dict(m=None), dict(v=None), dict(n=-1), dict(n=(1 << 38) + 1),
    dict(scale=1 << 25), dict(weight_decay=-0.1), dict(weight_decay=float("nan")),
    dict(w=(1 << 20) + 2), dict(low=(1 << 24) + 1), dict(m=(1 << 20) + 3996), dict(g=(1 << 20) + 3996),
    dict(g=(1 << 22) - 3996), dict(low=1 << 23)])
def test_adamw_refuses(bad):
    assert _adamw([_adamw_tensor(**bad)])[0] == binding.EKYA_ERR_INVALID_ARG


def test_adamw_list_and_options():
    lib = binding.load()
    assert _adamw([_adamw_tensor()] * 2)[0] == binding.EKYA_ERR_INVALID_ARG  # the same tensor twice
    assert _adamw([_adamw_tensor()], prec=2)[0] == binding.EKYA_ERR_INVALID_ARG
    assert _adamw([_adamw_tensor()], bits=16)[0] == binding.EKYA_ERR_INVALID_ARG
    assert _adamw([_adamw_tensor()], bits=8)[0] == binding.EKYA_ERR_INVALID_ARG  # no scale
    assert _adamw([], count=-1)[0] == binding.EKYA_ERR_INVALID_ARG
    assert _adamw([], count=65537)[0] == binding.EKYA_ERR_INVALID_ARG
    st, h = _adamw([_adamw_tensor(scale=1 << 25), _adamw_tensor(w=0, g=0, m=0, v=0, low=0, n=0)], bits=8)
    assert st == binding.EKYA_OK
    P2 = ctypes.c_void_p * 2
    assert lib.ekya_adamw_set_grads(h, P2(1 << 26, None), 2) == binding.EKYA_OK
    for grads, count in ((P2(1 << 26, None), 1), (P2(None, None), 2), (P2(1 << 22, None), 2),
                         (P2((1 << 25) + 8, None), 2), (P2((1 << 26) + 2, None), 2)):
        assert lib.ekya_adamw_set_grads(h, grads, count) == binding.EKYA_ERR_INVALID_ARG
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, step_device=None, seed=0)
    for bad in (dict(lr=-1.0), dict(lr=float("inf")), dict(lr=1e39), dict(beta1=1.0), dict(beta2=-0.1),
                dict(beta2=float("nan")), dict(eps=-1e-8), dict(step=0), dict(step_device=4)):
        opts = binding.AdamwOpts(**dict(good, **bad))
        assert lib.ekya_adamw_step(h, ctypes.byref(opts), None) == binding.EKYA_ERR_INVALID_ARG, bad
    assert lib.ekya_adamw_step(None, ctypes.byref(binding.AdamwOpts(**good)), None) != binding.EKYA_OK
    lib.ekya_adamw_destroy(h)
    lib.ekya_adamw_destroy(None)


def _matmul(ws=P, nbytes=BIG, **kw):
    a = dict(precision=1, M=64, N=32, K=16, x=1 << 20, ldx=16, w=1 << 21, ldw=16, bias=1 << 22, act=0,
             residual=1 << 23, ldr=32, residual_first=0, y=1 << 24, ldy=32, z=1 << 25, ldz=32)
    a.update(kw)
    return binding.load().ekya_op_matmul(ctypes.byref(binding.MatmulArgs(**a)), ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(precision=5), dict(M=-1), dict(N=0), dict(K=0), dict(N=(1 << 24) + 1), dict(K=(1 << 24) + 1, ldx=1 << 25, ldw=1 << 25),
    dict(M=1 << 36), dict(act=7), dict(x=None), dict(w=None), dict(y=None), dict(ldx=15), dict(ldw=0),
    dict(ldy=31), dict(ldz=-32), dict(ldr=1), dict(x=(1 << 20) + 1), dict(bias=(1 << 22) + 2),
    dict(y=(1 << 20) + 32), dict(y=(1 << 21) + 2), dict(y=1 << 25), dict(z=1 << 23),
    dict(y=(1 << 23) + 2), dict(y=1 << 23, ldy=64), dict(y=1 << 22), dict(z=(1 << 22) - 64),
    dict(ldx=1 << 62)])
def test_matmul_refuses(bad):
    assert _matmul(**bad) == binding.EKYA_ERR_INVALID_ARG


def test_matmul_workspace_is_checked():
    big = dict(M=8, N=8, K=1 << 16, ldx=1 << 16, ldw=1 << 16, x=1 << 30, w=1 << 32, ldr=8, ldy=8, ldz=8)
    a = binding.MatmulArgs(precision=1, **big)
    need = binding.load().ekya_op_matmul_workspace(ctypes.byref(a))
    assert need > 0
    assert _matmul(nbytes=need - 1, **big) == binding.EKYA_ERR_INVALID_ARG
    assert _matmul(ws=None, **big) == binding.EKYA_ERR_INVALID_ARG
    assert _matmul(ws=ctypes.c_void_p(4104), **big) == binding.EKYA_ERR_INVALID_ARG
    assert binding.load().ekya_op_matmul_workspace(None) == 0
    assert binding.load().ekya_op_matmul(None, P, BIG, None) == binding.EKYA_ERR_INVALID_ARG
    assert _matmul(M=0, x=None, w=None, y=None, ws=None, nbytes=0) == binding.EKYA_OK


def _matmul_backward(ws=P, nbytes=BIG, **kw):
    a = dict(precision=1, M=64, N=32, K=16, dy=1 << 20, lddy=32, z=1 << 21, ldz=32, act=1, x=1 << 22, ldx=16,
             w=1 << 23, ldw=16, dz=1 << 24, lddz=32, dx=1 << 25, lddx=16, dw=1 << 26, dw_precision=0, db=1 << 27)
    a.update(kw)
    return binding.load().ekya_op_matmul_backward(ctypes.byref(binding.MatmulBackwardArgs(**a)), ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(precision=2), dict(M=-5), dict(N=0), dict(K=1 << 25), dict(act=4), dict(dy=None), dict(z=None),
    dict(dz=None), dict(x=None), dict(w=None), dict(lddy=31), dict(ldx=15), dict(lddx=15), dict(dw_precision=2),
    dict(precision=0, dw_precision=1, ldx=16), dict(dw=(1 << 26) + 2), dict(db=(1 << 27) + 1),
    dict(dz=(1 << 20) + 2), dict(dz=1 << 20, lddz=64), dict(dx=1 << 20), dict(dx=1 << 22), dict(dx=1 << 23),
    dict(dx=1 << 24), dict(dw=1 << 22), dict(db=1 << 26), dict(dz=1 << 23)])
def test_matmul_backward_refuses(bad):
    assert _matmul_backward(**bad) == binding.EKYA_ERR_INVALID_ARG
    assert binding.load().ekya_op_matmul_backward(None, P, BIG, None) == binding.EKYA_ERR_INVALID_ARG
