"""Activations and their derivatives in 64 bits, for the tests of the
adapter-training operators."""
import math

ACTS = ["none", "relu", "silu", "gelu"]
U = 2.0 ** -24  # half a step of fp32, relative


def half_step(dtype):
    import torch
    return torch.finfo(dtype).eps / 2


def act64(u, act):
    """(act(u), act'(u)) of float64 u."""
    import torch
    if act == "none":
        return u, torch.ones_like(u)
    if act == "relu":
        return u.clamp(min=0), (u > 0).double()
    if act == "silu":
        p = torch.sigmoid(u)
        return u * p, p * (1 + u * (1 - p))
    p = torch.special.ndtr(u)
    return u * p, p + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)


def slope_error(du, u, act):
    """Bound on the error of act'(u) in fp32 when u is off by du: |act''| is at
    most 0.5 (silu) and 0.8 (gelu), ReLU's slope is right unless u may have
    changed sign; act' itself takes a few operations on values up to 1 + |u|,
    its exponential off by (|u| + 2) halves of a step."""
    import torch
    if act == "none":
        return torch.zeros_like(u)
    if act == "relu":
        return (u.abs() <= du).double()
    return du + 8 * U * (2 + u.abs())


def act_error(du, u, act):
    """The same for act(u): slopes are at most 1.13."""
    if act in ("none", "relu"):
        return du
    return 1.13 * du + 8 * U * (2 + u.abs()) * u.abs().clamp(max=1e4)


def strided(t, ld, offset=0):
    """A copy of t [M, N] whose rows are ld elements apart, `offset` elements into its storage;
    what lies between the rows is NaN."""
    import torch
    M, N = t.shape
    buf = torch.full((offset + M * ld + 1,), float("nan"), dtype=t.dtype, device=t.device)
    v = buf[offset:offset + M * ld].view(M, ld)[:, :N]
    v.copy_(t)
    return v
