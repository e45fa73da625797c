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


@pytest.fixture
def anywhere(monkeypatch):
    """Handles over CPU tensors: no step is taken, and creating one reads no tensor."""
    monkeypatch.setattr(binding, "_on_current", lambda *tensors: 0)


def _tensors(bits, sizes=(300, 7)):
    import torch
    types = (torch.float8_e4m3fn, torch.float8_e5m2) if bits == 8 else (torch.float32,) * 2
    out = []
    for n in sizes:
        t = {"w": torch.zeros(n), "g": torch.zeros(n), "low": torch.zeros(n, dtype=torch.bfloat16)}
        t.update(m=torch.zeros(n).to(types[0]), v=torch.zeros(n).to(types[1]))
        if bits == 8:
            t["scale"] = torch.ones((n + 255) // 256, 2)
        out.append(t)
    return out


@pytest.mark.parametrize("how", ["pop", "rebind", "data"])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_handle_keeps_its_tensors_whatever_becomes_of_the_dicts(anywhere, bits, how):
    import torch
    ts = _tensors(bits)
    places = [sorted(x.data_ptr() for k, x in t.items() if k != "g") for t in ts]
    opt = binding.ekya_adamw_create(ts, bits)
    for t in ts:
        for k in list(t):
            if how == "pop":
                t.pop(k)
            elif how == "rebind":
                t[k] = torch.zeros(1)
            elif k != "g":
                t[k].data = torch.zeros_like(t[k])
    held = [sorted(x.data_ptr() for x in t) for t in opt.tensors]
    assert held == places
    # new gradients are checked against the sizes that the handle was made with
    binding.ekya_adamw_set_grads(opt, [torch.zeros(300), torch.zeros(7)])
    with pytest.raises(ValueError, match="expected shape"):
        binding.ekya_adamw_set_grads(opt, [torch.zeros(1), torch.zeros(1)])
    binding.ekya_adamw_destroy(opt)


def test_gradients_that_were_replaced_are_let_go(anywhere):
    import gc
    import weakref
    import torch
    ts = _tensors(32)
    old = [weakref.ref(t["g"]) for t in ts]
    opt = binding.ekya_adamw_create(ts)
    del ts
    gc.collect()
    assert all(r() is not None for r in old)
    new = [torch.ones(300), torch.ones(7)]
    binding.ekya_adamw_set_grads(opt, new)
    gc.collect()
    assert all(r() is None for r in old)
    assert [g.data_ptr() for g in opt.grads] == [g.data_ptr() for g in new]
