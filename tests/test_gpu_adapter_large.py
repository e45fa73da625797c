"""Group norm and the matrix product with more samples and rows than a launch takes (2^21 blocks), and
rows as long as they may be, against float64 (tolerances as in test_gpu_groupnorm and
test_gpu_matmul)."""
import pytest

from tests.adapter_ref import U, half_step
from tests.test_gpu_groupnorm import _backward, _forward, _inputs, check_backward, check_forward
from tests.test_gpu_matmul import _check, _product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,HW,C,G,prec", [(2200000, 3, 6, 3, "f32"), (2200000, 2, 8, 2, "bf16")])
def test_groupnorm_of_more_samples_than_a_launch_takes(N, HW, C, G, prec):
    import torch
    x, dy, gamma, beta = _inputs(N, HW, C, torch.float32 if prec == "f32" else torch.bfloat16)
    y, mean, rstd = _forward(x, G, gamma, beta, "silu")
    check_forward(x, G, gamma, beta, "silu", y, mean, rstd)
    dx, dgamma, dbeta = _backward(dy, x, G, gamma, beta, mean, rstd, "silu")
    check_backward(dy, x, G, gamma, beta, mean, rstd, "silu", dx, dgamma, dbeta)


def test_matmul_of_more_rows_than_a_launch_takes():
    """2^21 tiles of 64 rows, and 200 rows more: the same bits as calls of 2^22 rows (one stage of one
    part either way), which are compared with float64 where a launch ends and the next begins.  dw and
    db are sums of M terms that a path of 2^20 roundings at most adds up, since 512 parts share them."""
    import torch
    from paper_2012_10557_amd import binding
    M, N, K, piece = 2 ** 27 + 200, 8, 8, 1 << 22
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(M, K, generator=gen, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(N, K, generator=gen, device="cuda", dtype=torch.bfloat16)
    y, _ = binding.ekya_op_matmul(x, w)
    dx, dw, db, _ = binding.ekya_op_matmul_backward(y, x, w)
    half = half_step(torch.bfloat16)
    sums = torch.zeros(4, N, K, dtype=torch.float64, device="cuda")
    for a in range(0, M, piece):
        part, dy = x[a:a + piece], y[a:a + piece]
        assert torch.equal(binding.ekya_op_matmul(part, w)[0], dy), a
        got = binding.ekya_op_matmul_backward(dy, part, w, need_dw=False, need_db=False)[0]
        assert torch.equal(got, dx[a:a + piece]), a
        for n in range(N):  # products of bf16 are exact in fp32
            t = dy[:, n:n + 1].float() * part.float()
            sums[0, n] += t.sum(0, dtype=torch.float64)
            sums[1, n] += t.abs().sum(0, dtype=torch.float64)
        sums[2, :, 0] += dy.float().sum(0, dtype=torch.float64)
        sums[3, :, 0] += dy.float().abs().sum(0, dtype=torch.float64)
    for a in (0, 2 ** 27 - 500, M - 500):
        ref, err = _product(x[a:a + 500], w)
        _check(y[a:a + 500], ref, err + half * (ref.abs() + err), ("y", a))
        ref, err = _product(y[a:a + 500], w.t())
        _check(dx[a:a + 500], ref, err + half * (ref.abs() + err), ("dx", a))
    _check(dw, sums[0], 2 ** 20 * U * sums[1], "dw")
    _check(db, sums[2, :, 0], 2 ** 20 * U * sums[3, :, 0], "db")


@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_matmul_of_the_widest_rows(prec):
    import torch
    from paper_2012_10557_amd import binding
    dtype = torch.float32 if prec == "f32" else torch.bfloat16
    half, n = half_step(dtype), 1 << 24
    gen = torch.Generator(device="cuda").manual_seed(2)

    def randn(*s):
        return torch.randn(*s, generator=gen, device="cuda").to(dtype)
    x, w, dy = randn(3, 8), randn(n, 8), randn(3, n)  # many outputs
    y, _ = binding.ekya_op_matmul(x, w)
    ref, err = _product(x, w)
    _check(y, ref, err + half * (ref.abs() + err), "y")
    dx, dw, db, _ = binding.ekya_op_matmul_backward(dy, x, w)
    ref, err = _product(dy.t(), x.t())
    _check(dw, ref, err + half_step(dw.dtype) * (ref.abs() + err), "dw")
    _check(db, dy.double().sum(0), 5 * U * dy.double().abs().sum(0) + 1e-37, "db")
    # a sum of n products, in 16 parts at least, each a chain of n / 16 roundings at most
    ref, mag = dy.double() @ w.double(), dy.double().abs() @ w.double().abs()
    _check(dx, ref, (n // 16 + 18) * U * mag + half * ref.abs() * 2, "dx")
    del w, dy, y, dw
    x, w, dy = randn(2, n), randn(3, n), randn(2, 3)  # many inputs
    y, _ = binding.ekya_op_matmul(x, w)
    ref, mag = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t()
    _check(y, ref, (n // 16 + 18) * U * mag + half * ref.abs() * 2, "y")
    dx, dw, db, _ = binding.ekya_op_matmul_backward(dy, x, w)
    ref, err = _product(dy, w.t())
    _check(dx, ref, err + half * (ref.abs() + err), "dx")
    ref, err = _product(dy.t(), x.t())
    _check(dw, ref, err + half_step(dw.dtype) * (ref.abs() + err), "dw")
