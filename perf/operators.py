"""Performance cases of the adapter-training operators: group norm with an
activation, the matrix product with its epilogue and the AdamW step, each
through the public binding (`paper_2012_10557_amd.binding`).

A case is a plain dict; `op` names the operator:

  groupnorm   ekya_op_groupnorm / _backward: x [n, hw, c] channels last
  matmul      ekya_op_matmul / _backward: x [m, k] with weights [n, k]
  adamw       ekya_adamw_step: one step over a list of tensors

With `own` false `run` computes the same in elementary torch operations in 32
bits.  `exact` computes it in 64 bits from the definitions.

Inputs stand in for what an adapter on frozen ResNet features meets:
activations whose channels have means and scales of their own, weights of
variance 1 / fan-in, gradients of a few thousandths, optimizer states of a
run in progress.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK = 256  # elements of an 8-bit state that share a scale
GOLDEN, TAG = 0x9E3779B97F4A7C15, 0xD1B54A32D192ED03
MASK64 = (1 << 64) - 1


# ------------------------------------------------------------------ cases
def _resnet18_sizes(classes=10):
    """Parameter tensors of the classifier: 20 convolutions, each with its
    BatchNorm weight and bias, and the fully connected layer."""
    sizes, cin = [64 * 3 * 49, 64, 64], 64
    for stage, width in enumerate((64, 128, 256, 512)):
        for block in range(2):
            sizes += [width * cin * 9, width, width, width * width * 9, width, width]
            if stage > 0 and block == 0:
                sizes += [width * cin, width, width]
            cin = width
    return ",".join(map(str, sizes + [classes * 512, classes]))


def _mlp_sizes(layers, width, hidden):
    return ",".join(map(str, [hidden * width, hidden, width * hidden, width, width] * layers))


def listed():
    return [
        # Layer4's output of one frame through an adapter's norm: serving, latency.
        {"name": "groupnorm_1x49x512", "op": "groupnorm", "pass": "forward", "n": 1, "hw": 49,
         "c": 512, "groups": 32, "act": "silu", "dtype": "bf16"},
        # Layer1's activations at the training batch, in place of BatchNorm + ReLU.
        {"name": "groupnorm_128x3136x64", "op": "groupnorm", "pass": "forward", "n": 128,
         "hw": 3136, "c": 64, "groups": 32, "act": "relu", "dtype": "bf16"},
        # The same layer's backward pass.
        {"name": "groupnorm_back_128x3136x64", "op": "groupnorm", "pass": "backward", "n": 128,
         "hw": 3136, "c": 64, "groups": 32, "act": "relu", "dtype": "bf16"},
        # An odd frame size in fp32, groups of 10 channels, which no 16-byte unit divides.
        {"name": "groupnorm_back_19x1147x120_fp32", "op": "groupnorm", "pass": "backward", "n": 19,
         "hw": 31 * 37, "c": 120, "groups": 12, "act": "silu", "dtype": "fp32"},
        # One frame's pooled features through a hidden layer: serving, latency.
        {"name": "matmul_1x512x1024", "op": "matmul", "pass": "forward", "m": 1, "k": 512,
         "n": 1024, "act": "relu", "residual": "none", "keep_z": False, "dtype": "bf16",
         "dw": "fp32"},
        # A batch's layer4 pixels through an adapter's first product, training.
        {"name": "matmul_6272x512x2048", "op": "matmul", "pass": "forward", "m": 128 * 49,
         "k": 512, "n": 2048, "act": "gelu", "residual": "none", "keep_z": True, "dtype": "bf16",
         "dw": "fp32"},
        # A large product with a residual added behind it: many pixels, wide layers.
        {"name": "matmul_16384x2048x8192", "op": "matmul", "pass": "forward", "m": 16384,
         "k": 2048, "n": 8192, "act": "silu", "residual": "after", "keep_z": False,
         "dtype": "bf16", "dw": "fp32"},
        # Backward of a 1 x 1 convolution with ReLU over layer3's pixels of a batch.
        {"name": "matmul_back_25088x256x1024", "op": "matmul", "pass": "backward", "m": 128 * 196,
         "k": 256, "n": 1024, "act": "relu", "residual": "none", "keep_z": True, "dtype": "bf16",
         "dw": "fp32"},
        # Ragged sizes in fp32, the residual added before the activation (a residual block).
        {"name": "matmul_1001x513x771_fp32", "op": "matmul", "pass": "forward", "m": 1001,
         "k": 513, "n": 771, "act": "relu", "residual": "before", "keep_z": False,
         "dtype": "fp32", "dw": "fp32"},
        # The classifier of 10 classes alone: two tensors, latency.
        {"name": "adamw_head", "op": "adamw", "sizes": "5120,10", "bits": 32, "grad": "fp32",
         "low": False, "step": 10},
        # Every parameter of the ResNet18, with the bf16 copy its kernels read.
        {"name": "adamw_resnet18", "op": "adamw", "sizes": _resnet18_sizes(), "bits": 32,
         "grad": "fp32", "low": True, "step": 100},
        # A wide network's layers with states in 8 bits and bf16 gradients.
        {"name": "adamw_mlp_8bit", "op": "adamw", "sizes": _mlp_sizes(8, 2048, 4096), "bits": 8,
         "grad": "bf16", "low": True, "step": 1000},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["groupnorm", "groupnorm", "matmul", "matmul", "matmul", "adamw", "adamw"])
    if op == "groupnorm":
        groups = rng.choice([1, 2, 4, 6, 8, 12, 16, 32])
        c = groups * rng.choice([1, 2, 3, 4, 5, 8, 10, 12, 16, 20, 32])
        n = _log_int(rng, 1, 128)
        most = 128 * 3136 * 64 // (n * c)
        least = -(-16 // (c // groups))  # elements of a group: fewer leave nothing of the gradient
        hw = _log_int(rng, least, max(least, min(12544, most)))
        return {"op": op, "pass": rng.choice(["forward", "backward"]), "n": n, "hw": hw, "c": c,
                "groups": groups, "act": rng.choice(["none", "relu", "silu", "gelu"]),
                "dtype": rng.choice(["bf16", "bf16", "fp32"])}
    if op == "matmul":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        which = rng.choice(["forward", "forward", "backward"])
        k, n = _log_int(rng, 16, 8192), _log_int(rng, 1, 8192)
        if rng.random() < 0.6:  # most layers' widths are multiples of 8
            k, n = -(-k // 8) * 8, -(-n // 8) * 8
        most = 2 ** 36 // (k * n) // (1 if dtype == "bf16" else 16)
        m = _log_int(rng, 1, max(1, min(32768, most)))
        act = rng.choice(["none", "relu", "silu", "gelu"])
        # weight gradients behind a smooth activation are taken in the inputs' type
        dw = dtype if act in ("silu", "gelu") else "fp32"
        return {"op": op, "pass": which, "m": m, "k": k, "n": n, "act": act,
                "residual": rng.choice(["none", "none", "after", "before"]),
                "keep_z": which == "backward" or rng.random() < 0.5, "dtype": dtype, "dw": dw}
    bits = rng.choice([32, 8])
    sizes, left = [], 2 ** 26
    for _ in range(rng.randint(1, 80)):
        sizes.append(min(max(1, left), _log_int(rng, 1, 2 ** rng.choice([8, 16, 22, 24]))))
        left -= sizes[-1]
    return {"op": op, "sizes": ",".join(map(str, sizes)), "bits": bits,
            "grad": rng.choice(["fp32", "bf16"]), "low": rng.random() < 0.5,
            "step": _log_int(rng, 1, 10000)}


# ----------------------------------------------------------------- inputs
def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _padded(sizes):
    return [-(-n // BLOCK) * BLOCK for n in sizes]


def _sizes(case):
    return [int(n) for n in case["sizes"].split(",")]


def prepare(case, seed):
    gen = _gen(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")
    s = {"case": case, "seed": seed & 0xFFFF}
    if case["op"] == "groupnorm":
        n, hw, c, g = case["n"], case["hw"], case["c"], case["groups"]
        dtype = _dtype(case["dtype"])
        s["x"] = (randn(n, hw, c) * (0.5 + randn(c).abs()) + randn(c)).to(dtype)
        s["gamma"], s["beta"] = 1 + 0.1 * randn(c), 0.1 * randn(c)
        if case["pass"] == "backward":
            s["dy"] = (0.01 * randn(n, hw, c)).to(dtype)
            x = s["x"].double().view(n, hw, g, c // g)
            mean = x.mean((1, 3))
            var = ((x - mean.view(n, 1, g, 1)) ** 2).mean((1, 3))
            s["mean"], s["rstd"] = mean.float(), (var + EPS).rsqrt().float()
    elif case["op"] == "matmul":
        m, k, n, dtype = case["m"], case["k"], case["n"], _dtype(case["dtype"])
        s["x"], s["w"] = randn(m, k).to(dtype), (randn(n, k) / math.sqrt(k)).to(dtype)
        s["bias"] = 0.1 * randn(n)
        s["residual"] = randn(m, n).to(dtype) if case["residual"] != "none" else None
        if case["pass"] == "backward":
            s["dy"] = (0.01 * randn(m, n)).to(dtype)
            s["z"] = randn(m, n).to(dtype)
    else:
        sizes = _sizes(case)
        pads = _padded(sizes)
        total = sum(pads)
        real = torch.cat([torch.arange(p, device="cuda") < n for n, p in zip(sizes, pads)])
        # matrices decay, vectors do not: the longer half of the list stands for matrices
        cut = sorted(sizes)[len(sizes) // 2]
        decays = [DECAY if n >= cut else 0.0 for n in sizes]
        s["w"] = 0.05 * randn(total) * real
        s["g"] = (0.003 * randn(total) * real).to(_dtype(case["grad"]))
        m, v = 0.001 * randn(total) * real, (0.003 * randn(total) * real) ** 2
        s["scale"] = None
        if case["bits"] == 8:
            s["scale"] = torch.empty(total // BLOCK, 2, device="cuda")
            states = []
            for i, (t, dt, top) in enumerate(((m, torch.float8_e4m3fn, 7), (v, torch.float8_e5m2, 14))):
                most = t.view(-1, BLOCK).abs().amax(1)
                s["scale"][:, i] = torch.exp2(torch.floor(torch.log2(most.clamp(min=1e-30))) - top)
                states.append((t.view(-1, BLOCK) / s["scale"][:, i:i + 1]).view(-1).to(dt))
            m, v = states
        s["m"], s["v"] = m, v
        s["low"] = s["w"].to(torch.bfloat16) if case["low"] else None
        s["decay"] = torch.cat([torch.full((p,), d, device="cuda") for d, p in zip(decays, pads)])
        s["tensors"], at = [], 0
        for n, p, d in zip(sizes, pads, decays):
            t = {name: s[name][at:at + n] for name in ("w", "g", "m", "v")}
            t["scale"] = s["scale"][at // BLOCK:(at + p) // BLOCK] if case["bits"] == 8 else None
            t["low"] = s["low"][at:at + n] if case["low"] else None
            s["tensors"].append(dict(t, weight_decay=d))
            at += p
    return s


# ------------------------------------------------------------ plain forms
def _act(u, act):
    if act == "relu":
        return u.clamp(min=0)
    if act == "silu":
        return u / (1 + torch.exp(-u))
    if act == "gelu":
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    return u


def _act_grad(u, act):
    if act == "relu":
        return (u > 0).to(u.dtype)
    if act == "silu":
        p = 1 / (1 + torch.exp(-u))
        return p * (1 + u * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)
    return torch.ones_like(u)


def _groupnorm_plain(s):
    case, x = s["case"], s["x"]
    n, hw, c, g = case["n"], case["hw"], case["c"], case["groups"]
    xg = x.float().view(n, hw, g, c // g)
    if case["pass"] == "forward":
        mean = xg.mean((1, 3))
        d = xg - mean.view(n, 1, g, 1)
        rstd = 1 / torch.sqrt((d * d).mean((1, 3)) + EPS)
        u = (d * rstd.view(n, 1, g, 1)).view(n, hw, c) * s["gamma"] + s["beta"]
        return {"y": _act(u, case["act"]).to(x.dtype), "mean": mean, "rstd": rstd}
    rstd = s["rstd"].view(n, 1, g, 1)
    xh = (xg - s["mean"].view(n, 1, g, 1)) * rstd
    u = xh.view(n, hw, c) * s["gamma"] + s["beta"]
    dyn = s["dy"].float() * _act_grad(u, case["act"])
    h = (dyn * s["gamma"]).view(n, hw, g, c // g)
    mean_h = h.mean((1, 3)).view(n, 1, g, 1)
    mean_hx = (h * xh).mean((1, 3)).view(n, 1, g, 1)
    dx = rstd * (h - mean_h - xh * mean_hx)
    return {"dx": dx.view(n, hw, c).to(x.dtype), "dgamma": (dyn * xh.view(n, hw, c)).sum((0, 1)),
            "dbeta": dyn.sum((0, 1))}


def _matmul_plain(s):
    case, x, w = s["case"], s["x"], s["w"]
    if case["pass"] == "forward":
        u = x.float() @ w.float().t() + s["bias"]
        if case["residual"] == "before":
            u = u + s["residual"].float()
        y = _act(u, case["act"])
        if case["residual"] == "after":
            y = y + s["residual"].float()
        return {"y": y.to(x.dtype), "z": u.to(x.dtype) if case["keep_z"] else None}
    dz = s["dy"].float()
    if case["act"] != "none":
        dz = dz * _act_grad(s["z"].float(), case["act"])
    return {"dx": (dz @ w.float()).to(x.dtype), "dw": (dz.t() @ x.float()).to(_dtype(case["dw"])),
            "db": dz.sum(0), "dz": dz.to(x.dtype) if case["act"] != "none" else None}


def _signed(v):
    return v - (1 << 64) if v >= 1 << 63 else v


def _bits16(count, seed, step):
    """16 random bits for each of `count` elements: output i of SplitMix64's stream
    that starts at seed + step * TAG serves elements 4 i .. 4 i + 3, lowest bits first."""
    i = torch.arange(1, count // 4 + 1, device="cuda", dtype=torch.int64)
    z = i * _signed(GOLDEN) + _signed((seed + step * TAG) & MASK64)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(0x94D049BB133111EB)
    z = z ^ ((z >> 31) & ((1 << 33) - 1))
    shifts = torch.tensor([0, 16, 32, 48], device="cuda")
    return ((z.unsqueeze(1) >> shifts) & 0xFFFF).view(-1).to(torch.int32)


def _to_8bit(x, rnd, mantissa, bias, top):
    """Codes of x [blocks, BLOCK] with `mantissa` bits and exponents biased by `bias`,
    rounded up in magnitude with the probability of the remainder, and the blocks'
    scales: the power of two that puts the largest value into [2^top, 2^(top+1))."""
    a = x.abs()
    finite = torch.isfinite(x)
    most = torch.where(finite, a, torch.zeros_like(a)).amax(1)
    k = ((most.view(torch.int32) >> 23) - 127 - top).clamp(min=-126)
    scale = ((k + 127) << 23).view(torch.float32)
    a = a * ((127 - k) << 23).view(torch.float32).unsqueeze(1)
    drop = 23 - mantissa
    r = (rnd.view_as(x) << (drop - 16)) + (1 << (drop - 17))
    bits = a.view(torch.int32)
    normal = ((bits + r) >> drop) - ((127 - bias) << mantissa)
    small = ((a * 2.0 ** (drop + bias - 1 + mantissa)).clamp(max=2.0 ** 24).to(torch.int32) + r) >> drop
    code = torch.where(bits >= (128 - bias) << 23, normal, small)
    return code, finite, scale


def _adamw_plain(s):
    case, step = s["case"], s["case"]["step"]
    g, m, v = s["g"].float(), s["m"], s["v"]
    if case["bits"] == 8:
        m = (m.float().view(-1, BLOCK) * s["scale"][:, :1]).view(-1)
        v = (v.float().view(-1, BLOCK) * s["scale"][:, 1:]).view(-1)
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    denom = torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** step)) + ADAM_EPS
    s["w"].copy_(s["w"] * (1 - LR * s["decay"]) - (LR / (1 - BETA1 ** step)) * (m / denom))
    if case["bits"] == 8:
        rnd = _bits16(m.numel(), s["seed"], step)
        code, finite, s["scale"][:, 0] = _to_8bit(m.view(-1, BLOCK), rnd, 3, 7, 7)
        code = torch.where(finite, code.clamp(max=0x7E), torch.full_like(code, 0x7F))
        code = (code | (m.view(-1, BLOCK) < 0).to(torch.int32) << 7).to(torch.uint8)
        s["m"].view(torch.uint8).copy_(code.view(-1))
        code, finite, s["scale"][:, 1] = _to_8bit(v.view(-1, BLOCK), 0xFFFF - rnd, 2, 15, 14)
        code = torch.maximum(code, (v > 0).to(torch.int32).view(-1, BLOCK)).clamp(max=0x7B)
        code = torch.where(finite, code, torch.full_like(code, 0x7F)).to(torch.uint8)
        s["v"].view(torch.uint8).copy_(code.view(-1))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if case["low"]:
        s["low"].copy_(s["w"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return {name: s[name] for name in ("w", "m", "v", "scale", "low")}


# -------------------------------------------------------------------- run
def _run_own(s):
    from paper_2012_10557_amd import binding
    case = s["case"]
    if case["op"] == "adamw":
        if "handle" not in s:
            s["handle"] = binding.ekya_adamw_create(s["tensors"], case["bits"])
        binding.ekya_adamw_step(s["handle"], lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS,
                                step=case["step"], seed=s["seed"])
        return _adamw_outputs(s)
    act = {"none": binding.EKYA_ACT_NONE, "relu": binding.EKYA_ACT_RELU,
           "silu": binding.EKYA_ACT_SILU, "gelu": binding.EKYA_ACT_GELU}[case["act"]]
    if case["op"] == "groupnorm":
        if case["pass"] == "forward":
            y, mean, rstd = binding.ekya_op_groupnorm(s["x"], case["groups"], s["gamma"], s["beta"],
                                                      eps=EPS, act=act)
            return {"y": y, "mean": mean, "rstd": rstd}
        dx, dgamma, dbeta = binding.ekya_op_groupnorm_backward(
            s["dy"], s["x"], case["groups"], s["gamma"], s["beta"], s["mean"], s["rstd"], act=act)
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if case["pass"] == "forward":
        y, z = binding.ekya_op_matmul(s["x"], s["w"], s["bias"], act=act, residual=s["residual"],
                                      residual_first=case["residual"] == "before",
                                      keep_z=case["keep_z"])
        return {"y": y, "z": z}
    dx, dw, db, dz = binding.ekya_op_matmul_backward(s["dy"], s["x"], s["w"], act=act, z=s["z"],
                                                     dw_dtype=_dtype(case["dw"]))
    return {"dx": dx, "dw": dw, "db": db, "dz": dz}


def run(s):
    if own:
        return _run_own(s)
    return {"groupnorm": _groupnorm_plain, "matmul": _matmul_plain,
            "adamw": _adamw_plain}[s["case"]["op"]](s)


# ------------------------------------------------------------------- work
def work(case):
    e = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "groupnorm":
        n = case["n"] * case["hw"] * case["c"]
        back = case["pass"] == "backward"
        small = 8 * case["n"] * case["groups"] + (16 if back else 8) * case["c"]
        return {"bytes": (3 if back else 2) * e * n + small, "flops": (24 if back else 12) * n}
    if case["op"] == "matmul":
        m, k, n = case["m"], case["k"], case["n"]
        if case["pass"] == "forward":
            outs = 1 + (case["residual"] != "none") + case["keep_z"]
            return {"bytes": e * (m * k + n * k + outs * m * n) + 4 * n, "flops": 2 * m * n * k}
        act = case["act"] != "none"
        dw = 2 if case["dw"] == "bf16" else 4
        return {"bytes": e * (2 * m * k + n * k + (3 if act else 1) * m * n) + dw * n * k + 4 * n,
                "flops": 4 * m * n * k}
    n = sum(_sizes(case))
    state = 4 + 16 / BLOCK if case["bits"] == 8 else 16
    return {"bytes": n * (8 + (2 if case["grad"] == "bf16" else 4) + state + 2 * case["low"]),
            "flops": 14 * n}


# ------------------------------------------------------------ 64-bit forms
def _activation64(u, act):
    """(act(u), act'(u)) in 64 bits."""
    if act == "none":
        return u, torch.ones_like(u)
    if act == "relu":
        return torch.where(u > 0, u, 0.0), torch.where(u > 0, 1.0, 0.0).double()
    if act == "silu":
        p = torch.sigmoid(u)
        return u * p, p + u * p * (1 - p)
    p = torch.special.ndtr(u)
    return u * p, p + u * torch.exp(-u * u / 2) * 0.3989422804014327


def _quantised64(x, r, mantissa, lowest, highest, top, keep):
    """The 8-bit values that stand for x / scale."""
    a = x.abs()
    k = torch.floor(torch.log2(a.amax(1).clamp(min=1e-300))) - top
    scale = torch.exp2(k.clamp(min=-126.0))
    a = a / scale.unsqueeze(1)
    quantum = torch.exp2(torch.floor(torch.log2(a.clamp(min=1e-300))).clamp(min=lowest) - mantissa)
    q = torch.clamp(torch.floor(a / quantum + r) * quantum, max=highest)
    if keep:
        q = torch.where((a > 0) & (q == 0), 2.0 ** (lowest - mantissa), q)
    return q * torch.sign(x)


def _random64(blocks, seed, step):
    """Fractions in (0, 1) of the elements' 16 bits (SplitMix64 in counter form)."""
    import numpy as np
    with np.errstate(over="ignore"):
        z = np.arange(1, blocks * BLOCK // 4 + 1, dtype=np.uint64) * np.uint64(GOLDEN)
        z += np.uint64((seed + step * TAG) & MASK64)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z ^= z >> np.uint64(31)
    bits = torch.from_numpy(z.view(np.int16)).cuda().to(torch.int64) & 0xFFFF  # little endian
    return bits.view(blocks, BLOCK)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "groupnorm":
        n, hw, c, g = case["n"], case["hw"], case["c"], case["groups"]
        x = s["x"].double().view(n, hw, g, c // g).permute(0, 2, 1, 3)  # n, g, hw, c / g

        def per_channel(t):
            return t.double().view(1, g, 1, c // g)

        def back(t):
            return t.permute(0, 2, 1, 3).reshape(n, hw, c)
        if case["pass"] == "forward":
            mean = x.mean((2, 3), keepdim=True)
            var = x.var((2, 3), unbiased=False, keepdim=True)
        else:
            mean, std = s["mean"].double().view(n, g, 1, 1), 1 / s["rstd"].double().view(n, g, 1, 1)
            var = std * std - EPS
        xh = (x - mean) / torch.sqrt(var + EPS)
        y, slope = _activation64(xh * per_channel(s["gamma"]) + per_channel(s["beta"]), case["act"])
        if case["pass"] == "forward":
            return {"y": back(y), "mean": mean.view(n, g), "rstd": 1 / torch.sqrt(var + EPS).view(n, g)}
        du = s["dy"].double().view(n, hw, g, c // g).permute(0, 2, 1, 3) * slope
        h = du * per_channel(s["gamma"])
        dx = (h - h.mean((2, 3), keepdim=True) - xh * (h * xh).mean((2, 3), keepdim=True)) / torch.sqrt(var + EPS)
        return {"dx": back(dx), "dgamma": (du * xh).sum((0, 2)).view(c), "dbeta": du.sum((0, 2)).view(c)}
    if case["op"] == "matmul":
        x, w = s["x"].double(), s["w"].double()
        if case["pass"] == "forward":
            z = torch.addmm(s["bias"].double(), x, w.t())
            r = s["residual"].double() if s["residual"] is not None else 0.0
            if case["residual"] == "before":
                z = z + r
            y = _activation64(z, case["act"])[0]
            return {"y": y + r if case["residual"] == "after" else y, "z": z if case["keep_z"] else None}
        dz = s["dy"].double() * _activation64(s["z"].double(), case["act"])[1]
        return {"dx": dz @ w, "dw": dz.t() @ x, "db": dz.sum(0),
                "dz": dz if case["act"] != "none" else None}
    step, bits = case["step"], case["bits"]
    blocks = s["w"].numel() // BLOCK
    w, g, decay = (s[name].double().view(blocks, BLOCK) for name in ("w", "g", "decay"))
    m, v = (s[name].double().view(blocks, BLOCK) for name in ("m", "v"))
    if bits == 8:
        m, v = m * s["scale"][:, 0:1].double(), v * s["scale"][:, 1:2].double()
    m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g * g - v)
    mh, vh = m / (1 - BETA1 ** step), v / (1 - BETA2 ** step)
    w = w - LR * decay * w - LR * mh / (vh.sqrt() + ADAM_EPS)
    # the scales follow the exponent of a 32-bit maximum, which 64 bits may put on the
    # other side of a power of two: their value here stands for nothing
    if bits == 8:
        r = _random64(blocks, s["seed"], step)
        m = _quantised64(m, (r.double() + 0.5) / 65536, 3, -6.0, 448.0, 7, False)
        v = _quantised64(v, (65535 - r.double() + 0.5) / 65536, 2, -14.0, 57344.0, 14, True)
    return {"w": w.view(-1), "m": m.view(-1), "v": v.view(-1), "scale": None,
            "low": w.view(-1) if case["low"] else None}
