"""Every kernel of the matrix product over several stages and ragged edges, against float64 (tolerances
as in test_gpu_matmul).  Which kernel a size reaches is checked in test_matmul_plan_host."""
import pytest

from tests.matmul_variants import VARIANTS
from tests.test_gpu_matmul import Case, check_backward, check_forward

pytestmark = pytest.mark.gpu


def _id(v):
    return "-".join([v[1], v[2], v[0].replace(" ", "_")])


@pytest.mark.parametrize("v", VARIANTS, ids=_id)
def test_variant_matches_float64(v):
    import torch
    _, prec, which, (M, N, K), aligned, _ = v
    dtype = torch.float32 if prec == "fp32" else torch.bfloat16
    # rows next to each other, then further apart (in units, or off them)
    for pad, offset in ((0, 0), (24, 8) if aligned else (3, 1)):
        c = Case(M, N, K, dtype, pad, offset)
        if which == "forward":
            check_forward(c, "silu", True, True, False, True)
            check_forward(c, "gelu", True, True, True, False)
        else:
            for dw in {dtype, torch.float32}:
                check_backward(c, "gelu", dw)


@pytest.mark.parametrize("v", [v for v in VARIANTS if v[4]], ids=_id)
def test_variant_gives_the_same_bits_again(v):
    """On another stream, while the same kernels run, and in a graph: no result depends on timing."""
    import torch
    from paper_2012_10557_amd import binding
    _, prec, which, (M, N, K), _, _ = v
    c = Case(M, N, K, torch.float32 if prec == "fp32" else torch.bfloat16)

    def run():
        if which == "forward":
            return binding.ekya_op_matmul(c.x, c.w, c.bias, act=2, residual=c.res, keep_z=True)
        return binding.ekya_op_matmul_backward(c.dy, c.x, c.w, act=1, z=c.z)
    first = run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(4):
        got.append(run())
        with torch.cuda.stream(s):
            got.append(run())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for _ in range(3):
        graph.replay()
        got.append(run())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, first))
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, first))


@pytest.mark.parametrize("M,N,K", [(77, 45, 40), (130, 261, 24), (2000, 2001, 40), (3, 1001, 300)])
@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_residual_in_place_off_16_bytes(prec, M, N, K):
    """Rows that no 16-byte unit divides: a lane's columns are read ahead of those it has finished."""
    import torch
    from paper_2012_10557_amd import binding
    from tests.adapter_ref import strided
    dtype = torch.float32 if prec == "f32" else torch.bfloat16
    c = Case(M, N, K, dtype)
    for act in ("none", "relu", "silu", "gelu"):
        for first in (False, True):
            y, _ = check_forward(c, act, True, True, first, False)
            for ld, offset in ((N, 0), (N + 3, 1)):
                res = strided(c.res, ld, offset)
                got, _ = binding.ekya_op_matmul(c.x, c.w, c.bias, act=["none", "relu", "silu", "gelu"].index(act),
                                                residual=res, residual_first=first, y=res)
                assert got is res and torch.equal(got, y), (act, first, ld)
