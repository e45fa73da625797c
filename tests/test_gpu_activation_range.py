"""The activations over the whole range of their argument, against float64.

A product of one input with the weight 1 is exact, so the argument is the input
itself, and y and z (as the gradient's dy is 1) show the activation alone.
Tolerances are relative to the result.  U = 2^-24 is half an fp32 step."""
import pytest

from tests.adapter_ref import ACTS, U, act64, half_step

pytestmark = pytest.mark.gpu
SILU, GELU = 2, 3
BEYOND = [100.0, 1e30, 2.3e38, 2.5e38, 3e38, float("inf")]


def _apply(u, act):
    """(act(u), act'(u)) of the operators for u [n]."""
    import torch
    from paper_2012_10557_amd import binding
    x, one = u.view(-1, 1), torch.ones(1, 1, dtype=u.dtype, device="cuda")
    y, z = binding.ekya_op_matmul(x, one, act=act, keep_z=True)
    assert torch.equal(z, x)
    dz = binding.ekya_op_matmul_backward(torch.ones_like(x), x, one, act=act, z=z, need_dx=False,
                                         need_dw=False, need_db=False)[3]
    return y.view(-1), x if dz is None else dz.view(-1)


def _check(got, ref, rel, floor):
    """got within rel (relative) of ref and a rounding to its type; values below `floor` may be 0."""
    import torch
    finite = torch.isfinite(ref)
    a = got.double()
    same = (a == ref) | (torch.isnan(a) & torch.isnan(ref))
    close = (a - ref).abs() <= ref.abs() * (rel + half_step(got.dtype) * (1 + rel)) + floor
    ok = torch.where(finite, close, same)
    assert ok.all(), [(float(r), float(g)) for r, g in zip(ref[~ok], a[~ok])][:8]


def _values(dtype):
    import torch
    near = torch.linspace(-80, 80, 1281, dtype=torch.float64)
    far = torch.tensor(BEYOND + [-v for v in BEYOND] + [-86.0, -87.0, -88.0, -89.0, 87.0, 88.0, 89.0],
                       dtype=torch.float64)
    u = torch.cat([near, far]).cuda().to(dtype)
    return u[torch.isfinite(u) | torch.isinf(u)]


@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_silu_over_its_whole_range(prec):
    """The sigmoid p is off by r p, r = 8 U in fp32 (its exponential 3, the sum, the reciprocal and a
    Newton step 3, the product 1) and (2 |u| + 8) U in bf16 (the exponent's rounding as well); below
    2^-126 it is 0.  The slope p (1 + u (1 - p)) takes that twice, as a factor and in 1 - p, where it
    meets |u|, and five roundings."""
    import torch
    dtype = torch.float32 if prec == "f32" else torch.bfloat16
    u = _values(dtype)
    y, slope = _apply(u, SILU)
    u64 = u.double()
    ref, dref = u64 / (1 + torch.exp(-u64)), act64(u64, "silu")[1]
    size = u64.abs().clamp(max=128)
    rel = 8 * U if prec == "f32" else (2 * size + 8) * U
    _check(y, ref, rel, 2.0 ** -126 * size)
    p = torch.sigmoid(u64)
    q = 1 - p
    err = p * (rel * (1 + size * q) + size * (rel * p + 2 * U * q) + 3 * U * (1 + size * q))
    ok = torch.where(torch.isfinite(dref),
                     (slope.double() - dref).abs() <= 1.01 * err + half_step(dtype) * (dref.abs() + 1.01 * err) +
                     2.0 ** -126 * size, torch.isnan(slope) & torch.isnan(dref))
    assert ok.all(), [(float(a), float(b)) for a, b in zip(u64[~ok], slope[~ok])][:8]


@pytest.mark.parametrize("hw", [9, 4000])
@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_silu_of_large_values_behind_group_norm(prec, hw):
    """gamma 0 and a beta near the type's largest value: u is beta."""
    import torch
    from paper_2012_10557_amd import binding
    dtype = torch.float32 if prec == "f32" else torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(hw)
    x = torch.randn(2, hw, 16, generator=gen, device="cuda").to(dtype)
    beta = torch.tensor([2.2e38, 2.4e38, 3e38, -3e38] * 4, device="cuda")
    gamma = torch.zeros(16, device="cuda")
    y, mean, rstd = binding.ekya_op_groupnorm(x, 4, gamma, beta, act=SILU)
    want = beta.clamp(min=0).to(dtype).expand(2, hw, 16)
    assert torch.equal(y, want)
    dy = torch.ones_like(x)
    dx, dgamma, dbeta = binding.ekya_op_groupnorm_backward(dy, x, 4, gamma, beta, mean, rstd, act=SILU)
    assert not dx.any()
    assert torch.equal(dbeta, (beta > 0).float() * (2 * hw))


def test_the_other_activations_of_large_values():
    import torch
    for dtype in (torch.float32, torch.bfloat16):
        u = torch.tensor(BEYOND + [-v for v in BEYOND[:-1]], device="cuda").to(dtype)
        for act in ("none", "relu", "gelu"):
            y, slope = _apply(u, ACTS.index(act))
            assert torch.equal(y, u if act == "none" else u.clamp(min=0)), act
            fin = torch.isfinite(u)  # u phi(u) of inf is not a number
            assert act == "none" or torch.equal(slope[fin], (u > 0).to(dtype)[fin]), act


@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_gelu_keeps_its_digits_far_below_zero(prec):
    """The normal distribution's lower tail P is off by r P.  fp32: erfc of an argument off by 3 U,
    which its tail takes u^2 times, and 64 U of the function's own.  bf16: the fit's 1.04e-4 (a 37th of
    half a step), an exponential whose argument u^2 / 2 is off by 2 U of itself, and 32 U of the
    polynomial and its constants.  Above 0 the result is 1 - P.  The slope P + u phi adds the error
    of phi, the same as the exponential's; three roundings each."""
    import math
    import torch
    dtype = torch.float32 if prec == "f32" else torch.bfloat16
    u = torch.linspace(-13, 13, 6657, dtype=torch.float64).cuda().to(dtype)
    y, slope = _apply(u, GELU)
    u64, size = u.double(), u.double().abs()
    exponential = (2 * size * size + 8) * U
    rel = (4 * size * size + 64) * U if prec == "f32" else 1.04e-4 + exponential + 32 * U
    tail = 0.5 * torch.special.erfc(size / math.sqrt(2))
    P, dens = 0.5 * torch.special.erfc(-u64 / math.sqrt(2)), torch.exp(-0.5 * u64 * u64) / math.sqrt(2 * math.pi)
    dP = rel * tail + 2 * U * P
    half = half_step(dtype)
    for got, ref, err in ((y, u64 * P, size * (dP + U * P)),
                          (slope, P + u64 * dens, dP + size * dens * (exponential + 3 * U) + 2 * U * (P + size * dens))):
        bound = 1.01 * err + half * (ref.abs() + 1.01 * err) + 2.0 ** -126 * 14
        ok = (got.double() - ref).abs() <= bound
        assert ok.all(), [(float(a), float(g), float(r)) for a, g, r in zip(u64[~ok], got[~ok], ref[~ok])][:8]
