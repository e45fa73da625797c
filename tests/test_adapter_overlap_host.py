"""Arguments of group norm that share memory: refused before any GPU work, so without a GPU.
Every tensor has a place of its own unless a test moves it, so that one reason is left to refuse."""
import ctypes

import pytest

from paper_2012_10557_amd import binding

N, HW, C, G = 2, 8, 32, 4
BYTES = N * HW * C * 2  # of x, y, dy and dx (bf16)
PLACES = {name: (i + 1) << 20 for i, name in enumerate(
    ["x", "y", "dy", "dx", "gamma", "beta", "mean", "rstd", "dgamma", "dbeta", "ws"])}


def _forward(**kw):
    a = dict(PLACES, prec=1, N=N, HW=HW, C=C, G=G, eps=1e-5, act=0, nbytes=1 << 16)
    a.update(kw)
    lib = binding.load()
    st = lib.ekya_op_groupnorm(a["prec"], a["x"], a["N"], a["HW"], a["C"], a["G"], a["gamma"], a["beta"], a["eps"],
                               a["act"], a["y"], a["mean"], a["rstd"], a["ws"], a["nbytes"], None)
    return st, lib.ekya_last_error(None).decode()


def _backward(**kw):
    a = dict(PLACES, prec=1, N=N, HW=HW, C=C, G=G, act=0, nbytes=1 << 16)
    a.update(kw)
    lib = binding.load()
    st = lib.ekya_op_groupnorm_backward(a["prec"], a["dy"], a["x"], a["N"], a["HW"], a["C"], a["G"], a["gamma"],
                                        a["beta"], a["mean"], a["rstd"], a["act"], a["dx"], a["dgamma"],
                                        a["dbeta"], a["ws"], a["nbytes"], None)
    return st, lib.ekya_last_error(None).decode()


def _at(name, offset=0):
    return PLACES[name] + offset


@pytest.mark.parametrize("bad", [
    dict(mean=_at("rstd")), dict(mean=_at("rstd", 28)), dict(mean=_at("rstd", -28)), dict(mean=_at("x", BYTES - 4)),
    dict(mean=_at("y")), dict(rstd=_at("y", BYTES - 4)), dict(mean=_at("gamma")), dict(rstd=_at("beta", 124)),
    dict(y=_at("gamma")), dict(y=_at("beta", 124)), dict(y=_at("x", 2)), dict(y=_at("x", 2 - BYTES))])
def test_groupnorm_refuses_shared_outputs(bad):
    st, why = _forward(**bad)
    assert st == binding.EKYA_ERR_INVALID_ARG and "overlap" in why


@pytest.mark.parametrize("bad", [
    dict(dgamma=_at("gamma")), dict(dbeta=_at("beta")), dict(dgamma=_at("dbeta")), dict(dgamma=_at("dbeta", 124)),
    dict(dgamma=_at("beta", -124)), dict(dbeta=_at("gamma", 4)), dict(dgamma=_at("mean")), dict(dbeta=_at("rstd", 28)),
    dict(dgamma=_at("x", BYTES - 4)), dict(dbeta=_at("dy")), dict(dgamma=_at("dx")), dict(dx=_at("mean")),
    dict(dx=_at("rstd", 28)), dict(dx=_at("gamma")), dict(dx=_at("beta", 124)), dict(dx=_at("x", 2)),
    dict(dx=_at("dy", BYTES - 2))])
def test_groupnorm_backward_refuses_shared_outputs(bad):
    st, why = _backward(**bad)
    assert st == binding.EKYA_ERR_INVALID_ARG and "overlap" in why


@pytest.mark.parametrize("good", [
    dict(y=_at("x")), dict(y=_at("x", BYTES)), dict(mean=_at("rstd", -4 * N * G)), dict(rstd=_at("gamma", 4 * C)),
    dict(gamma=_at("beta"))])
def test_groupnorm_takes_neighbours_and_its_own_place(good):
    """The next check is the workspace's, which is short here."""
    st, why = _forward(nbytes=0, **good)
    assert st == binding.EKYA_ERR_INVALID_ARG and "workspace" in why


@pytest.mark.parametrize("good", [
    dict(dx=_at("x")), dict(dx=_at("dy")), dict(dx=_at("x"), dy=_at("x")), dict(dgamma=_at("dbeta", -4 * C)),
    dict(dbeta=_at("gamma", 4 * C)), dict(dgamma=None, dbeta=None), dict(gamma=None, beta=None),
    dict(mean=_at("rstd"), gamma=_at("beta")),
    # no samples: nothing but the parameters' gradients is touched
    dict(N=0, x=None, dy=None, dx=None, mean=None, rstd=None), dict(N=0, dx=_at("dgamma"), mean=_at("dbeta"))])
def test_groupnorm_backward_takes_neighbours_and_its_own_place(good):
    st, why = _backward(nbytes=0, **good)
    assert st == binding.EKYA_ERR_INVALID_ARG and "workspace" in why


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(gamma=None), dict(beta=None),
    dict(x=_at("x", 1)), dict(y=_at("y", 1)), dict(mean=_at("mean", 2)), dict(rstd=_at("rstd", 2)), dict(N=-1),
    dict(gamma=_at("gamma", 1)), dict(beta=_at("beta", 2)), dict(ws=None), dict(ws=_at("ws", 8)), dict(nbytes=8),
    dict(prec=2), dict(HW=0), dict(C=0), dict(C=65537, G=1), dict(G=0), dict(G=5), dict(eps=0.0),
    dict(eps=float("nan")), dict(eps=float("inf")), dict(act=4), dict(act=-1), dict(HW=1 << 36), dict(HW=1 << 62),
    dict(N=1 << 30, HW=1 << 30)])
def test_groupnorm_refuses_each_argument_alone(bad):
    assert _forward(**bad)[0] == binding.EKYA_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(gamma=None), dict(dgamma=None),
    dict(dbeta=None), dict(dy=_at("dy", 1)), dict(dgamma=_at("dgamma", 2)), dict(ws=None), dict(nbytes=8),
    dict(prec=-1), dict(G=3), dict(act=9), dict(HW=0)])
def test_groupnorm_backward_refuses_each_argument_alone(bad):
    assert _backward(**bad)[0] == binding.EKYA_ERR_INVALID_ARG


def test_the_places_themselves_are_distinct():
    lib = binding.load()
    need = max(lib.ekya_op_groupnorm_workspace(1, N, HW, C, G),
               lib.ekya_op_groupnorm_backward_workspace(1, N, HW, C, G))
    assert need <= 1 << 16 and ctypes.sizeof(ctypes.c_void_p) == 8
