"""What the binding of the adapter-training operators checks itself, without a GPU: tensors on the
meta device have sizes and no memory."""
import pytest

from paper_2012_10557_amd import binding

WIDE = (1 << 32) + 8  # its lower 32 bits are a size that would be taken


def _meta(*shape):
    import torch
    return torch.empty(*shape, dtype=torch.bfloat16, device="meta")


@pytest.mark.parametrize("shape,groups", [((WIDE, 1, 8), 4), ((1, WIDE), 4), ((2, 3, 8), WIDE)])
def test_groupnorm_sizes_beyond_an_int_are_refused(shape, groups):
    x = _meta(*shape)
    with pytest.raises(ValueError, match="above 2"):
        binding.ekya_op_groupnorm(x, groups)
    with pytest.raises(ValueError, match="above 2"):
        binding.ekya_op_groupnorm_backward(x, x, groups, None, None, x, x)


@pytest.mark.parametrize("N,K", [(WIDE, 1), (1, WIDE)])
def test_matmul_sizes_beyond_an_int_are_refused(N, K):
    x, w, dy = _meta(2, K), _meta(N, K), _meta(2, N)
    with pytest.raises(ValueError, match="above 2"):
        binding.ekya_op_matmul(x, w)
    with pytest.raises(ValueError, match="above 2"):
        binding.ekya_op_matmul_backward(dy, x, w)


def test_sizes_of_an_int_reach_the_next_check():
    import torch
    if torch.cuda.is_available():
        pytest.skip("for a machine without a GPU")
    for call in (lambda: binding.ekya_op_groupnorm(torch.empty(2, 3, 8), 4),
                 lambda: binding.ekya_op_matmul(torch.empty(2, 3), torch.empty(4, 3))):
        with pytest.raises((ValueError, RuntimeError, AssertionError)) as e:
            call()
        assert "above 2" not in str(e.value)
