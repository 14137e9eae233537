"""Cases for the operators that a training step needs around the pruned products: group norm with an activation
(channels last), embedding lookup and its gradient, and the AdamW step over many tensors.

Each operator in two forms: the library's (`own` true) and a plain one of elementary torch operations in binary32.
`exact` states the same definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "relu", "silu", "gelu")
QBLOCK = 256                     # elements that share one scale of the 8-bit optimiser states
E4M3_MAX = 448.0


def listed():
    return [
        # the deepest level of a small convolutional net, two images: latency
        {"name": "gn_fwd_8x8", "op": "gn_fwd", "n": 2, "s": 64, "c": 512, "g": 32, "act": "silu", "dtype": "bf16", "affine": "f32"},
        # the convolution layer of the library's workloads: batch 64, 56 x 56, 256 channels
        {"name": "gn_fwd_conv", "op": "gn_fwd", "n": 64, "s": 56 * 56, "c": 256, "g": 32, "act": "relu", "dtype": "bf16", "affine": "f32"},
        # full precision, an odd and large map, ten channels to a group
        {"name": "gn_fwd_map_f32", "op": "gn_fwd", "n": 3, "s": 127 * 93, "c": 320, "g": 32, "act": "silu", "dtype": "f32", "affine": "f32"},
        # the backward pass of the convolution layer, the activation with the dearer derivative
        {"name": "gn_bwd_conv", "op": "gn_bwd", "n": 64, "s": 56 * 56, "c": 256, "g": 32, "act": "silu", "dtype": "bf16", "affine": "f32"},
        # a small full-precision batch of odd maps, sixteen channels to a group
        {"name": "gn_bwd_odd_f32", "op": "gn_bwd", "n": 5, "s": 31 * 29, "c": 96, "g": 6, "act": "gelu", "dtype": "f32", "affine": "f32"},
        # one token for each of eight sequences
        {"name": "embed_decode", "op": "embed", "t": 8, "v": 32000, "d": 4096, "scale": 64.0, "dtype": "bf16"},
        # the token count of the large feed-forward workload
        {"name": "embed_16k", "op": "embed", "t": 16384, "v": 131072, "d": 4096, "scale": 64.0, "dtype": "bf16"},
        # the token count and width of the small feed-forward workload, an odd vocabulary
        {"name": "embed_grad_8k", "op": "embed_grad", "t": 8192, "v": 50257, "d": 768, "scale": 1.0, "dtype": "bf16"},
        # the token count and width of the stack of twelve layers
        {"name": "embed_grad_32k", "op": "embed_grad", "t": 32768, "v": 65536, "d": 1024, "scale": 32.0, "dtype": "bf16"},
        # biases and norm weights: many tensors of a few thousand elements
        {"name": "adamw_vectors", "op": "adamw", "tensors": 96, "rows": 1, "cols": 2500, "state": 32, "param": "f32", "grad": "f32"},
        # the weights of the stack of twelve layers, bf16 with a full-precision copy, gradients as the update products give them
        {"name": "adamw_stack", "op": "adamw", "tensors": 24, "rows": 4096, "cols": 1024, "state": 32, "param": "bf16+f32", "grad": "f32"},
        # the two weights of the large feed-forward layer, bf16 alone, states in 8 bits
        {"name": "adamw8_ffn", "op": "adamw", "tensors": 2, "rows": 14336, "cols": 4096, "state": 8, "param": "bf16", "grad": "bf16"},
    ]


def _spread(rng, low, high):
    """A whole number spread over the logarithm of [low, high]."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["gn_fwd", "gn_bwd", "embed", "embed_grad", "adamw", "adamw"])
    if op in ("gn_fwd", "gn_bwd"):
        g = rng.choice([1, 2, 5, 6, 8, 16, 30, 32, 32])
        cg = rng.choice([1, 3, 4, 7, 8, 8, 10, 12, 16, 16, 24])
        n, s = _spread(rng, 1, 64), _spread(rng, 1, 16000)
        while n * s * g * cg > 40_000_000:
            n, s = max(1, n // 2), max(1, s // 2)
        return {"op": op, "n": n, "s": s, "c": g * cg, "g": g, "act": rng.choice(ACTS), "dtype": rng.choice(["bf16", "bf16", "f32"]),
                "affine": rng.choice(["f32", "bf16"])}
    if op == "embed":
        return {"op": op, "t": _spread(rng, 1, 16384), "v": _spread(rng, 1000, 131072), "d": rng.choice([rng.randrange(33, 1100), 768, 1024, 2048, 4096]),
                "scale": rng.choice([1.0, 27.7, 64.0]), "dtype": rng.choice(["bf16", "f32"])}
    if op == "embed_grad":
        return {"op": op, "t": _spread(rng, 1, 32768), "v": _spread(rng, 1000, 65536), "d": rng.choice([rng.randrange(33, 1024), 256, 768, 1024]),
                "scale": rng.choice([1.0, 27.7, 64.0]), "dtype": rng.choice(["bf16", "f32"])}
    return {"op": op, "tensors": _spread(rng, 1, 96), "rows": 1, "cols": _spread(rng, 1, 1_000_000), "state": rng.choice([8, 32]),
            "param": rng.choice(["f32", "bf16+f32", "bf16"]), "grad": rng.choice(["f32", "bf16"])}


def _elements(case):
    """Elements of each tensor of an AdamW case: the matrices alike, vectors of lengths that differ (odd ones among them)."""
    n = case["rows"] * case["cols"]
    return [n if case["rows"] > 1 else max(1, n - 37 * (i % 7)) for i in range(case["tensors"])]


def _distinct(t, v):
    """How many different ids t tokens of _prepare_embed have (expected)."""
    k = np.arange(v)
    return float(np.sum(-np.expm1(t * np.log1p(-np.log((k + 2) / (k + 1)) / math.log(v)))))


def work(case):
    op, esize = case["op"], {"bf16": 2, "f32": 4}.get(case.get("dtype"), 0)
    if op in ("gn_fwd", "gn_bwd"):
        e = case["n"] * case["s"] * case["c"]
        return {"bytes": e * esize * (2 if op == "gn_fwd" else 3) + 8 * case["n"] * case["g"], "flops": e * (10 if op == "gn_fwd" else 25)}
    if op == "embed":
        return {"bytes": (case["t"] + _distinct(case["t"], case["v"])) * case["d"] * esize + 8 * case["t"], "flops": case["t"] * case["d"]}
    if op == "embed_grad":
        return {"bytes": case["t"] * (case["d"] * esize + 8) + case["v"] * case["d"] * 4, "flops": 2 * case["t"] * case["d"]}
    n = sum(_elements(case))
    weight = {"f32": 8, "bf16": 4, "bf16+f32": 10}[case["param"]]       # bf16 beside its copy is only written
    state = 16 if case["state"] == 32 else 4 + 16 / QBLOCK
    return {"bytes": n * (weight + state + {"f32": 4, "bf16": 2}[case["grad"]]), "flops": 15 * n}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _prepare_gn(case, seed):
    gen, dt = _generator(seed), DTYPES[case["dtype"]]
    n, s, c, g = case["n"], case["s"], case["c"], case["g"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    x = (normal(n, s, c) * (0.5 + torch.rand((c,), generator=gen, device="cuda")) + normal(c)).to(dt)   # channels have means and widths of their own
    st = {"case": case, "x": x, "g": g, "act": case["act"], "eps": 1e-5,
          "weight": (1.0 + 0.2 * normal(c)).to(DTYPES[case["affine"]]), "bias": (0.2 * normal(c)).to(DTYPES[case["affine"]])}
    if case["op"] == "gn_bwd":
        st["dy"] = (1e-3 * normal(n, s, c)).to(dt)
        # the statistics that the forward pass left
        x4 = x.float().reshape(n, s, g, c // g)
        st["mean"] = x4.mean((1, 3))
        st["rstd"] = ((x4 - st["mean"][:, None, :, None]).square().mean((1, 3)) + st["eps"]).rsqrt()
    return st


def _prepare_embed(case, seed):
    gen, dt = _generator(seed), DTYPES[case["dtype"]]
    t, v, d = case["t"], case["v"], case["d"]
    # text: few words make up most of it, and their numbers are anywhere in the vocabulary
    rank = (torch.exp(torch.rand((t,), generator=gen, device="cuda", dtype=torch.float64) * math.log(v)) - 1).long().clamp_(0, v - 1)
    ids = torch.randperm(v, generator=gen, device="cuda")[rank]
    st = {"case": case, "ids": ids, "v": v, "scale": case["scale"]}
    if case["op"] == "embed":
        st["weight"] = (0.02 * torch.randn((v, d), generator=gen, device="cuda")).to(dt)
    else:
        st["dy"] = (1e-3 * torch.randn((t, d), generator=gen, device="cuda")).to(dt)
        st["padding"] = int(ids[t // 2]) if t > 16 else -1
    return st


def _prepare_adamw(case, seed):
    gen = _generator(seed)
    sizes = _elements(case)
    blocks = [-(-n // QBLOCK) for n in sizes]
    total = sum(blocks) * QBLOCK
    starts = [sum(blocks[:i]) * QBLOCK for i in range(len(blocks))]
    # one buffer for all tensors, each on a boundary of QBLOCK elements; what lies between them is zero and stays so
    used = torch.zeros((total,), dtype=torch.bool, device="cuda")
    for a, n in zip(starts, sizes):
        used[a:a + n] = True

    def normal(std):
        return torch.randn((total,), generator=gen, device="cuda").mul_(std).mul_(used)

    st = {"case": case, "sizes": sizes, "starts": starts, "step": 100, "seed": seed * 1_000_003 + 17,
          "lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "decay": 0.1}
    weight = normal(0.02)
    st["param"] = weight.clone() if case["param"] == "f32" else weight.to(torch.bfloat16)
    st["master"] = weight if case["param"] == "bf16+f32" else None
    st["grad"] = normal(1e-3).to(DTYPES[case["grad"]])
    m, v = normal(3e-4), normal(1e-3).square_().add_(used * 1e-8)
    if case["state"] == 32:
        st["m"], st["v"], st["m_scale"], st["v_scale"] = m, v, None, None
    else:
        for name, x in (("m", m), ("v", v.sqrt_())):
            top = x.view(-1, QBLOCK).abs().amax(1, keepdim=True)
            st[name + "_scale"] = (top / E4M3_MAX).reshape(-1)
            st[name] = (x.view(-1, QBLOCK) * (E4M3_MAX / top)).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).reshape(-1)
    if own:
        # the optimiser object that a program makes once beside its weights: the list of its tensors and gradient buffers
        from paper_2203_10991_b200 import optim

        def parts(x, unit=1):
            return None if x is None else [x[a // unit:a // unit + (-(-n // unit))] for a, n in zip(starts, sizes)]

        st["plan"] = optim.AdamWPlan(parts(st["param"]), parts(st["m"]), parts(st["v"]), masters=parts(st["master"]),
                                     exp_avg_scales=parts(st["m_scale"], QBLOCK), exp_avg_sq_scales=parts(st["v_scale"], QBLOCK),
                                     grads=parts(st["grad"]))
    return st


def prepare(case, seed):
    return {"gn_fwd": _prepare_gn, "gn_bwd": _prepare_gn, "embed": _prepare_embed, "embed_grad": _prepare_embed,
            "adamw": _prepare_adamw}[case["op"]](case, seed)


# ---- the operators in plain form -------------------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(z)


def _gn_forward(st):
    x, g = st["x"], st["g"]
    n, s, c = x.shape
    x4 = x.float().reshape(n, s, g, c // g)
    mean = x4.mean((1, 3))
    d = x4 - mean[:, None, :, None]
    rstd = 1 / torch.sqrt(d.square().mean((1, 3)) + st["eps"])
    z = (d * rstd[:, None, :, None]).reshape(n, s, c) * st["weight"].float() + st["bias"].float()
    return _act(z, st["act"]).to(x.dtype), mean, rstd


def _gn_backward(st):
    x, g = st["x"], st["g"]
    n, s, c = x.shape
    w = st["weight"].float()
    xh = ((x.float().reshape(n, s, g, c // g) - st["mean"][:, None, :, None]) * st["rstd"][:, None, :, None]).reshape(n, s, c)
    dz = st["dy"].float() * _act_grad(xh * w + st["bias"].float(), st["act"])
    dbias, dweight = dz.sum((0, 1)), (dz * xh).sum((0, 1))
    dxh, xh = (dz * w).reshape(n, s, g, c // g), xh.reshape(n, s, g, c // g)
    dx = (dxh - dxh.mean((1, 3), keepdim=True) - xh * (dxh * xh).mean((1, 3), keepdim=True)) * st["rstd"][:, None, :, None]
    return dx.reshape(n, s, c).to(x.dtype), dweight, dbias


def _embed_grad(st):
    rows = st["dy"].float() * st["scale"] * (st["ids"] != st["padding"])[:, None]
    return torch.zeros((st["v"], rows.shape[1]), device=rows.device).index_add_(0, st["ids"], rows)


def _random16(units, stream, seed):
    """Sixteen-bit uniform numbers, eight for each unit: Philox4x32-10, counter (low, high word of the unit, stream, 0)."""
    low = 0xFFFFFFFF
    c0, c1, c2, c3 = units & low, units >> 32, torch.full_like(units, stream), torch.zeros_like(units)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)


def _to_e4m3(x, random, at_least_one):
    """(codes, scales): blocks of QBLOCK elements, magnitudes scaled to 448 and rounded up with the probability of their
    place between two codes; a code of at least one where asked for and x is not zero."""
    top = x.view(-1, QBLOCK).abs().amax(1, keepdim=True)
    inverse = torch.where(top > 0, top.reciprocal() * E4M3_MAX, torch.zeros_like(top))
    y = (x.view(-1, QBLOCK).abs() * inverse).clamp_(max=E4M3_MAX).reshape(-1)
    exponent = (y.view(torch.int32) >> 23).clamp_(min=121)
    steps = torch.floor(y * ((257 - exponent) << 23).view(torch.float32) + random.float() * 2.0 ** -16)
    codes = ((exponent - 121) << 3) + steps.int()
    if at_least_one:
        codes = torch.where(x > 0, codes.clamp(min=1), codes)
    codes = codes | ((x < 0).int() << 7)
    return codes.to(torch.uint8).view(torch.float8_e4m3fn), (top * (1 / E4M3_MAX)).reshape(-1)


def _adamw(st):
    t = st["step"]
    b1, b2 = st["beta1"], st["beta2"]
    wide = st["case"]["state"] == 32
    g = st["grad"].float()
    if wide:
        m, v = st["m"], st["v"]
    else:
        m = (st["m"].float().view(-1, QBLOCK) * st["m_scale"][:, None]).reshape(-1)
        v = (st["v"].float().view(-1, QBLOCK) * st["v_scale"][:, None]).reshape(-1).square()
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * (1 - b2) * g
    root = torch.sqrt(v)
    den = root * (1 / math.sqrt(1 - b2 ** t)) + st["eps"]
    weight = st["param"].float() if st["master"] is None else st["master"]
    weight = weight * (1 - st["lr"] * st["decay"]) - m / den * (st["lr"] / (1 - b1 ** t))
    units = torch.arange(g.numel() // 8, device=g.device)
    random = None if wide and st["case"]["param"] != "bf16" else _random16(units, 2, st["seed"] + t)
    if wide:
        st["m"], st["v"] = m, v
    else:
        swapped = (random & 0xFF) << 8 | random >> 8
        st["m"], st["m_scale"] = _to_e4m3(m, swapped, False)
        st["v"], st["v_scale"] = _to_e4m3(root, swapped, True)
    if st["case"]["param"] == "bf16":
        bits = (weight.view(torch.int32) + random.int()) & -65536
        st["param"] = bits.view(torch.float32).to(torch.bfloat16)
    else:
        st["param"] = weight.to(st["param"].dtype)
        st["master"] = weight if st["master"] is not None else None


def _adamw_answer(st):
    return {k: st[k] for k in ("param", "master", "m", "v", "m_scale", "v_scale") if st[k] is not None}


def run(state):
    st, op = state, state["case"]["op"]
    if not own:
        if op == "gn_fwd":
            return _gn_forward(st)
        if op == "gn_bwd":
            return _gn_backward(st)
        if op == "embed":
            return (st["weight"][st["ids"]].float() * st["scale"]).to(st["weight"].dtype)
        if op == "embed_grad":
            return _embed_grad(st)
        _adamw(st)
        st["step"] += 1
        return _adamw_answer(st)
    from paper_2203_10991_b200 import binding
    if op == "gn_fwd":
        return binding.mvue_group_norm_act(st["x"], st["g"], st["weight"], st["bias"], eps=st["eps"], act=st["act"])
    if op == "gn_bwd":
        return binding.mvue_group_norm_act_backward(st["dy"], st["x"], st["mean"], st["rstd"], st["g"], st["weight"], st["bias"], act=st["act"])
    if op == "embed":
        return binding.mvue_embedding(st["ids"], st["weight"], scale=st["scale"])
    if op == "embed_grad":
        return binding.mvue_embedding_grad(st["ids"], st["dy"], st["v"], scale=st["scale"], padding_idx=st["padding"])
    st["plan"].step(step=st["step"], lr=st["lr"], beta1=st["beta1"], beta2=st["beta2"], eps=st["eps"], weight_decay=st["decay"],
                    seed=st["seed"] + st["step"], stochastic_rounding=True)
    st["step"] += 1
    return _adamw_answer(st)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _exact_gn(st):
    x = st["x"].double()
    n, s, c = x.shape
    group = torch.arange(c, device=x.device) // (c // st["g"])                 # the group of each channel
    w, b = st["weight"].double(), st["bias"].double()

    def over_groups(per_channel):                                              # [n, c] sums to [n, c] means over each group
        sums = torch.zeros((n, st["g"]), dtype=torch.float64, device=x.device).index_add_(1, group, per_channel)
        return sums / (s * (c // st["g"]))

    if st["case"]["op"] == "gn_fwd":
        mean = over_groups(x.sum(1))
        x = x - mean[:, group][:, None]
        rstd = (over_groups((x * x).sum(1)) + st["eps"]) ** -0.5
    else:
        mean, rstd = st["mean"].double(), st["rstd"].double()
        x = x - mean[:, group][:, None]
    x = x * rstd[:, group][:, None]
    z = x * w + b
    cdf = {"silu": torch.sigmoid, "gelu": torch.special.ndtr, "relu": lambda u: (u > 0).double(), "none": torch.ones_like}[st["act"]](z)
    if st["case"]["op"] == "gn_fwd":
        return z * cdf, mean, rstd
    slope = {"silu": lambda u: cdf * (1 - cdf), "gelu": lambda u: torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)}.get(st["act"])
    dz = st["dy"].double() * (cdf + z * slope(z) if slope else cdf)
    along = (dz * x).sum(1)
    plain = dz.sum(1)
    dx = rstd[:, group][:, None] * (w * dz - over_groups(plain * w)[:, group][:, None] - x * over_groups(along * w)[:, group][:, None])
    return dx, along.sum(0), plain.sum(0)


def _exact_adamw(st):
    lr, b1, b2, t = st["lr"], st["beta1"], st["beta2"], st["step"]
    g, m, v = st["grad"].double(), st["m"].double(), st["v"].double()
    if st["m_scale"] is not None:
        m = m * st["m_scale"].double().repeat_interleave(QBLOCK)
        v = (v * st["v_scale"].double().repeat_interleave(QBLOCK)) ** 2
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g ** 2
    weight = (st["param"] if st["master"] is None else st["master"]).double()
    weight = weight - lr * (st["decay"] * weight + (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)) ** 0.5 + st["eps"]))
    said = {"param": weight}
    if st["master"] is not None:
        said["master"] = weight
    if st["m_scale"] is None:
        return {**said, "m": m, "v": v}
    # the codes are rounded by chance: what they stand for is the value over its block's scale
    for name, x in (("m", m), ("v", v ** 0.5)):
        scale = x.abs().reshape(-1, QBLOCK).amax(1) / E4M3_MAX
        said[name] = x / scale.repeat_interleave(QBLOCK).clamp(min=1e-300)
        said[name + "_scale"] = scale
    return said


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    op = case["op"]
    if op in ("gn_fwd", "gn_bwd"):
        return _exact_gn(st)
    if op == "adamw":
        return _exact_adamw(st)
    if op == "embed":
        return st["weight"].double().index_select(0, st["ids"]) * st["scale"]
    keep = st["ids"] != st["padding"]
    into = torch.zeros((st["v"], case["d"]), dtype=torch.float64, device="cuda")
    return into.index_add_(0, st["ids"][keep], st["dy"][keep].double()) * st["scale"]
