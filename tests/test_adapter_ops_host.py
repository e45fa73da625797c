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
