"""One training step of an adapter on frozen features, by the operators as they
are used together, against float64: group norm with SiLU, a product with GELU, a
product with its residual, the mean squared distance to a target, the way back
through all of them and an AdamW step that also writes the bf16 weights which
the next step's products read."""
import pytest

from tests.adapter_ref import act64

pytestmark = pytest.mark.gpu
EPS, LR = 1e-5, 1e-3
N, HW, C, HIDDEN, GROUPS = 6, 49, 72, 136, 6


class Adapter:
    def __init__(self, dtype, bits):
        import torch
        from paper_2012_10557_amd import binding
        self.b, self.dtype = binding, dtype
        gen = torch.Generator(device="cuda").manual_seed(3)

        def randn(*s):
            return torch.randn(s, generator=gen, device="cuda")
        self.master = {"gamma": 1 + 0.1 * randn(C), "beta": 0.1 * randn(C), "w1": randn(HIDDEN, C) * C ** -0.5,
                       "b1": 0.1 * randn(HIDDEN), "w2": randn(C, HIDDEN) * HIDDEN ** -0.5, "b2": 0.1 * randn(C)}
        self.low = {k: self.master[k].to(torch.bfloat16) for k in ("w1", "w2")}
        self.grad = {k: torch.zeros_like(v) for k, v in self.master.items()}
        tensors = []
        for k, w in self.master.items():
            t = {"w": w, "g": self.grad[k], "weight_decay": 0.01 if w.dim() == 2 else 0.0,
                 "low": self.low.get(k)}
            if bits == 8:
                t.update(m=torch.zeros_like(w, dtype=torch.float8_e4m3fn),
                         v=torch.zeros_like(w, dtype=torch.float8_e5m2),
                         scale=torch.ones((w.numel() + 255) // 256, 2, device="cuda"))
            else:
                t.update(m=torch.zeros_like(w), v=torch.zeros_like(w))
            tensors.append(t)
        self.opt = binding.ekya_adamw_create(tensors, bits)
        self.step_no = torch.zeros(1, dtype=torch.int64, device="cuda")

    def weight(self, k):
        import torch
        return self.low[k] if self.dtype == torch.bfloat16 else self.master[k]

    def step(self, x, target):
        """x, target [N, HW, C]; returns the output and the features' gradient."""
        import torch
        b, p = self.b, self.master
        h, mean, rstd = b.ekya_op_groupnorm(x, GROUPS, p["gamma"], p["beta"], eps=EPS, act=b.EKYA_ACT_SILU)
        flat = h.view(N * HW, C)
        a, z = b.ekya_op_matmul(flat, self.weight("w1"), p["b1"], act=b.EKYA_ACT_GELU, keep_z=True)
        y, _ = b.ekya_op_matmul(a, self.weight("w2"), p["b2"], residual=x.view(N * HW, C))
        dy = ((y.float() - target.view(N * HW, C).float()) * (2 / y.numel())).to(self.dtype)
        da, dw2, db2, _ = b.ekya_op_matmul_backward(dy, a, self.weight("w2"))
        dh, dw1, db1, _ = b.ekya_op_matmul_backward(da, flat, self.weight("w1"), act=b.EKYA_ACT_GELU, z=z)
        dx, dgamma, dbeta = b.ekya_op_groupnorm_backward(dh.view(N, HW, C), x, GROUPS, p["gamma"], p["beta"],
                                                         mean, rstd, act=b.EKYA_ACT_SILU)
        for k, g in (("gamma", dgamma), ("beta", dbeta), ("w1", dw1), ("b1", db1), ("w2", dw2), ("b2", db2)):
            self.grad[k].copy_(g)
        self.step_no.add_(1)
        b.ekya_adamw_step(self.opt, LR, step_device=self.step_no, seed=11)
        return y.view(N, HW, C), dx


def _reference(p, x, target):
    """(y, gradients) in float64 by torch's differentiation of the formulas."""
    import torch
    p = {k: v.double().requires_grad_() for k, v in p.items()}
    x = x.double().requires_grad_()
    xg = x.view(N, HW, GROUPS, C // GROUPS)
    m, v = xg.mean((1, 3), keepdim=True), xg.var((1, 3), unbiased=False, keepdim=True)
    u = ((xg - m) * (v + EPS).rsqrt()).reshape(N, HW, C) * p["gamma"] + p["beta"]
    h = act64(u, "silu")[0].view(N * HW, C)
    a = act64(h @ p["w1"].t() + p["b1"], "gelu")[0]
    y = (a @ p["w2"].t() + p["b2"]).view(N, HW, C) + x
    loss = ((y - target.double()) ** 2).mean()
    names = list(p)
    grads = torch.autograd.grad(loss, [p[k] for k in names] + [x])
    # the residual's share of the features' gradient is not the adapter's
    share = 2 / y.numel() * (y - target.double())
    return y.detach(), dict(zip(names, grads[:-1])), (grads[-1] - share).detach()


def _data(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(9)
    x, t = (torch.randn(N, HW, C, generator=gen, device="cuda") for _ in range(2))
    return x.to(dtype), t.to(dtype)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("prec", ["f32", "bf16"])
def test_adapter_step_matches_float64(prec, bits):
    """Tolerances, relative to a tensor's largest value: what passes between the operators is rounded
    to the type eight times on the way to the last gradient (h, a, z, y, dy, da, dz, dh), each by half
    a step (2^-9 / 2^-24 with the sum behind it some K = 136 fp32 roundings, sqrt(136) of them at
    random); a tensor's largest value stands for the sum of magnitudes within a factor of 4."""
    import torch
    dtype = torch.float32 if prec == "f32" else torch.bfloat16
    tol = 4 * 8 * (2.0 ** -9 if prec == "bf16" else 12 * 2.0 ** -24)
    ad = Adapter(dtype, bits)
    x, target = _data(dtype)
    before = {k: (ad.weight(k) if k in ("w1", "w2") else v).double().clone() for k, v in ad.master.items()}
    start = {k: v.clone() for k, v in ad.master.items()}
    y, dx = ad.step(x, target)
    ry, grads, rdx = _reference(before, x, target)

    def close(got, ref, what):
        err = float((got.double() - ref).abs().max() / ref.abs().max())
        assert err <= tol, (what, err)
    close(y, ry, "y")
    close(dx, rdx, "dx")
    for k, g in grads.items():
        close(ad.grad[k], g, k)
        # the first step: m / sqrt(v) is the sign of the gradient that the step was given
        g1 = ad.grad[k].double()
        decay = 0.01 if g1.dim() == 2 else 0.0
        want = start[k].double() * (1 - LR * decay) - LR * g1 / (g1.abs() + 1e-8)
        assert (ad.master[k].double() - want).abs().max() <= 1e-6
        if k in ad.low:
            assert torch.equal(ad.low[k], ad.master[k].to(torch.bfloat16))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_adapter_step_repeats_the_eager_one(bits):
    import torch
    eager, other = Adapter(torch.bfloat16, bits), Adapter(torch.bfloat16, bits)
    x, target = _data(torch.bfloat16)
    xs = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = other.step(xs, target)
    for i in range(4):
        x = torch.roll(x, 1, 0)
        xs.copy_(x)
        ey, edx = eager.step(x, target)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ey) and torch.equal(dx, edx), i
        for k in eager.master:
            assert torch.equal(eager.master[k], other.master[k]), (i, k)
        assert int(other.step_no) == int(eager.step_no) == i + 1
