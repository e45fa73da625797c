"""Group norm where a block keeps its samples in registers, at the sizes between which its kernels
change: 3, 8 and 16 units a thread, and one more than the largest holds (tolerances as in
test_gpu_groupnorm)."""
import pytest

from tests.test_gpu_groupnorm import _backward, _forward, _inputs, check_backward, check_forward

pytestmark = pytest.mark.gpu


# a unit is 4 channels; 1024 threads take 256 rows of 16 channels, 1024 of 4 and 128 of 32
@pytest.mark.parametrize("N,HW,C,G", [
    (2, 768, 16, 4), (2, 769, 16, 4), (3, 2048, 16, 1), (3, 2049, 16, 4), (2, 3840, 16, 2), (2, 4095, 16, 4),
    (2, 4096, 16, 4), (2, 4097, 16, 4), (1, 4096, 64, 32), (513, 300, 64, 32), (2, 16384, 8, 2), (1, 16385, 8, 2),
    (2, 1024, 32, 1), (2, 1025, 32, 1), (2, 2048, 64, 2), (65, 1030, 96, 3)])
@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_units_of_a_thread(prec, N, HW, C, G):
    import torch
    dtype = torch.float32 if prec == "f32" else torch.bfloat16
    for act in ("gelu", "relu") if HW % 2 else ("silu", "none"):
        x, dy, gamma, beta = _inputs(N, HW, C, dtype)
        y, mean, rstd = _forward(x, G, gamma, beta, act)
        check_forward(x, G, gamma, beta, act, y, mean, rstd)
        dx, dgamma, dbeta = _backward(dy, x, G, gamma, beta, mean, rstd, act)
        check_backward(dy, x, G, gamma, beta, mean, rstd, act, dx, dgamma, dbeta)
