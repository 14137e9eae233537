"""Cases for the operators that a layer's own arithmetic needs beside the pruned products: layer norm and its backward pass,
the quantiser and the dense products in 8-bit floating point (e4m3) with a power-of-two scale for each block of 128, and the
Muon step, which orthogonalises the update of a weight matrix.

Each operator in two forms: the library's (`own` true) and a plain one of elementary torch operations in binary32.
`exact` states the same definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 128                      # elements along the reduction axis that share a scale
E4M3_MAX = 448.0
POLYNOMIAL = (3.4445, -4.7750, 2.0315)     # s -> 3.4445 s - 4.7750 s^3 + 2.0315 s^5 on the singular values


def listed():
    return [
        # one token for each of eight sequences, the width of the large feed-forward workload: latency
        {"name": "ln_fwd_8", "op": "ln_fwd", "rows": 8, "cols": 4096, "dtype": "bf16", "affine": "f32"},
        # all tokens of the large feed-forward workload
        {"name": "ln_fwd_16k", "op": "ln_fwd", "rows": 16384, "cols": 4096, "dtype": "bf16", "affine": "f32"},
        # the token count and width of the stack of twelve layers
        {"name": "ln_bwd_32k", "op": "ln_bwd", "rows": 32768, "cols": 1024, "dtype": "bf16", "affine": "f32"},
        # full precision, an odd number of odd rows
        {"name": "ln_bwd_odd_f32", "op": "ln_bwd", "rows": 4097, "cols": 1111, "dtype": "f32", "affine": "f32"},
        # the neural gradient of the large feed-forward workload, rounded without bias
        {"name": "quant_gradient", "op": "quant", "rows": 16384, "cols": 14336, "block_rows": 1, "stochastic": True, "dtype": "bf16"},
        # the weights of that layer, one scale for 128 x 128, once per step
        {"name": "quant_weights", "op": "quant", "rows": 14336, "cols": 4096, "block_rows": 128, "stochastic": False, "dtype": "bf16"},
        # eight tokens against those weights: what counts is how fast the weights stream
        {"name": "fwd_8", "op": "gemm", "t": 8, "out": 14336, "inp": 4096, "way": "forward", "dtype": "bf16"},
        # the forward product of the large feed-forward layer
        {"name": "fwd_ffn", "op": "gemm", "t": 16384, "out": 14336, "inp": 4096, "way": "forward", "dtype": "bf16"},
        # the backward product of a layer of the stack
        {"name": "bwd_stack", "op": "gemm", "t": 32768, "out": 4096, "inp": 1024, "way": "backward", "dtype": "bf16"},
        # odd extents, full precision out
        {"name": "bwd_odd_f32", "op": "gemm", "t": 1000, "out": 1111, "inp": 777, "way": "backward", "dtype": "f32"},
        # one small square matrix, orthogonalised alone: fifteen dependent products, latency
        {"name": "ortho_256", "op": "ortho", "tensors": 1, "rows": 256, "cols": 256, "grad": "f32"},
        # the weights of the stack of twelve layers
        {"name": "muon_stack", "op": "muon", "tensors": 24, "rows": 4096, "cols": 1024, "stochastic": True, "grad": "f32"},
    ]


def _spread(rng, low, high):
    """A whole number spread over the logarithm of [low, high]."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "quant", "gemm", "gemm", "muon", "ortho"])
    if op in ("ln_fwd", "ln_bwd"):
        rows, cols = _spread(rng, 1, 32768), rng.choice([_spread(rng, 17, 16384), 768, 1024, 4096])
        while rows * cols > 16384 * 4096:
            rows //= 2
        return {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "bf16", "f32"]), "affine": rng.choice(["f32", "bf16"])}
    if op == "quant":
        rows, cols = _spread(rng, 1, 32768), rng.choice([_spread(rng, 17, 14336), 1024, 4096])
        while rows * cols > 16384 * 14336:
            rows //= 2
        return {"op": op, "rows": rows, "cols": cols, "block_rows": rng.choice([1, 128]), "stochastic": rng.random() < 0.5,
                "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "gemm":
        t = _spread(rng, 1, 32768)
        out, inp = (rng.choice([_spread(rng, 17, 14336), 1024, 4096]) for _ in range(2))
        while t * out * inp > 16384 * 14336 * 4096:
            t //= 2
        return {"op": op, "t": t, "out": out, "inp": inp, "way": rng.choice(["forward", "backward"]), "dtype": rng.choice(["bf16", "bf16", "f32"])}
    tensors, rows, cols = _spread(rng, 1, 24), _spread(rng, 16, 4096), _spread(rng, 16, 4096)
    while tensors > 1 and tensors * _muon_flops(rows, cols) > 24 * _muon_flops(4096, 1024):
        tensors //= 2
    case = {"op": op, "tensors": tensors, "rows": rows, "cols": cols, "grad": rng.choice(["f32", "bf16"])}
    return case if op == "ortho" else {**case, "stochastic": rng.random() < 0.5}


def _blocks(n):
    return -(-n // BLOCK)


def _muon_flops(rows, cols):
    """Five times A = X X^T, A A (both symmetric: half of the entries) and B X."""
    m, n = min(rows, cols), max(rows, cols)
    return 5 * (m * m * n + m * m * m + 2 * m * m * n)


def work(case):
    op, esize = case["op"], {"bf16": 2, "f32": 4}.get(case.get("dtype"), 0)
    if op in ("ln_fwd", "ln_bwd"):
        e = case["rows"] * case["cols"]
        return {"bytes": e * esize * (2 if op == "ln_fwd" else 3) + 8 * case["rows"], "flops": e * (8 if op == "ln_fwd" else 14)}
    if op == "quant":
        e = case["rows"] * case["cols"]
        scales = _blocks(case["cols"]) * (case["rows"] if case["block_rows"] == 1 else _blocks(case["rows"]))
        return {"bytes": e * (esize + 1) + scales, "flops": 4 * e}
    if op == "gemm":
        t, o, i = case["t"], case["out"], case["inp"]
        k, n = (i, o) if case["way"] == "forward" else (o, i)
        return {"bytes": t * k + o * i + t * n * esize + t * _blocks(k) + _blocks(o) * _blocks(i), "flops": 2 * t * o * i}
    e = case["tensors"] * case["rows"] * case["cols"]
    return {"bytes": e * ((2 if op == "ortho" else 8 + 4) + {"f32": 4, "bf16": 2}[case["grad"]]), "flops": case["tensors"] * _muon_flops(case["rows"], case["cols"])}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _prepare_ln(case, seed):
    gen, dt = _generator(seed), DTYPES[case["dtype"]]
    rows, cols = case["rows"], case["cols"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    # tokens have means and widths of their own, a few channels stand out
    x = normal(rows, cols) * (0.5 + torch.rand((rows, 1), generator=gen, device="cuda")) + 0.5 * normal(rows, 1)
    x[:, torch.randperm(cols, generator=gen, device="cuda")[: cols // 256]] *= 8
    st = {"case": case, "x": x.to(dt), "eps": 1e-5, "weight": (1.0 + 0.2 * normal(cols)).to(DTYPES[case["affine"]]),
          "bias": (0.2 * normal(cols)).to(DTYPES[case["affine"]])}
    if case["op"] == "ln_bwd":
        st["dy"] = (1e-3 * normal(rows, cols)).to(dt)
        # the statistics that the forward pass left
        x = st["x"].float()
        st["mean"] = x.mean(1)
        st["rstd"] = ((x - st["mean"][:, None]).square().mean(1) + st["eps"]).rsqrt()
    return st


def _prepare_quant(case, seed):
    gen = _generator(seed)
    x = torch.randn((case["rows"], case["cols"]), generator=gen, device="cuda")
    if case["block_rows"] == 1:
        # a neural gradient: tokens of very different size, heavy tails
        x = x * torch.exp(torch.randn((case["rows"], 1), generator=gen, device="cuda")) * x.abs() * 1e-3
    else:
        x = 0.02 * x
    return {"case": case, "x": x.to(DTYPES[case["dtype"]]), "block_rows": case["block_rows"],
            "seed": seed * 1_000_003 + 17 if case["stochastic"] else None}


def _pitched(codes):
    """The same codes with rows that start on 16-byte boundaries, as the quantiser leaves them."""
    rows, cols = codes.shape
    wide = torch.zeros((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=codes.device)
    wide[:, :cols] = codes.view(torch.uint8)
    return wide.view(torch.float8_e4m3fn)[:, :cols]


def _prepare_gemm(case, seed):
    gen = _generator(seed)
    t, o, i = case["t"], case["out"], case["inp"]
    forward = case["way"] == "forward"
    k = i if forward else o
    # activations behind a norm, or a gradient with tokens of very different size; weights of a trained layer
    a = torch.randn((t, k), generator=gen, device="cuda")
    if not forward:
        a *= 1e-3 * torch.exp(torch.randn((t, 1), generator=gen, device="cuda"))
    w = torch.randn((o, i), generator=gen, device="cuda") * (i ** -0.5)
    a, a_scales = _quantize(a, 1, None)
    w, w_scales = _quantize(w, BLOCK, None)
    return {"case": case, "a": _pitched(a), "a_scales": a_scales, "w": _pitched(w), "w_scales": w_scales, "forward": forward,
            "dtype": DTYPES[case["dtype"]]}


def _prepare_muon(case, seed):
    gen = _generator(seed)
    shape = (case["tensors"], case["rows"], case["cols"])

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    # gradients of a layer: a few directions that many examples share, and noise
    r = max(1, min(case["rows"], case["cols"]) // 16)
    grad = 1e-3 * (normal(*shape) + normal(shape[0], shape[1], r) @ normal(shape[0], r, shape[2]) * r ** -0.5)
    if case["op"] == "ortho":
        return {"case": case, "x": grad.to(DTYPES[case["grad"]]), "steps": 5}
    st = {"case": case, "param": (0.02 * normal(*shape)).to(torch.bfloat16), "m": 0.3e-3 * normal(*shape) + 0.7 * grad,
          "grad": grad.to(DTYPES[case["grad"]]), "lr": 1e-3, "momentum": 0.95, "decay": 0.1, "steps": 5,
          "step": 100, "seed": seed * 1_000_003 + 17}
    if own:
        # the optimiser object that a program makes once beside its weights: the list of its matrices and gradient buffers
        from paper_2203_10991_b200 import optim
        st["plan"] = optim.MuonPlan(list(st["param"]), list(st["m"]), grads=list(st["grad"]))
    return st


def prepare(case, seed):
    return {"ln_fwd": _prepare_ln, "ln_bwd": _prepare_ln, "quant": _prepare_quant, "gemm": _prepare_gemm, "muon": _prepare_muon,
            "ortho": _prepare_muon}[case["op"]](case, seed)


# ---- the operators in plain form -------------------------------------------------------------------------------------

def _ln_forward(st):
    x = st["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt(d.square().mean(1) + st["eps"])
    return (d * rstd[:, None] * st["weight"].float() + st["bias"].float()).to(st["x"].dtype), mean, rstd


def _ln_backward(st):
    xh = (st["x"].float() - st["mean"][:, None]) * st["rstd"][:, None]
    dy = st["dy"].float()
    g = dy * st["weight"].float()
    dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * st["rstd"][:, None]
    return dx.to(st["x"].dtype), (dy * xh).sum(0), dy.sum(0)


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
    return torch.stack([words & 0xFFFF, words >> 16], 2)


def _per_element(scales, rows, cols, block_rows):
    """The values of scales (exponent bytes) spread over the elements of a [rows, cols] matrix."""
    values = torch.exp2(scales.float() - 127)
    if block_rows == 1:
        return values.T.repeat_interleave(BLOCK, 1)[:, :cols]
    return values.repeat_interleave(BLOCK, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def _exponents(x, block_rows):
    """The exponent byte of each block's scale: the least power of two (from 2^-126) that brings its largest magnitude to 448 or less."""
    rows, cols = x.shape
    wide = torch.zeros((-(-rows // block_rows) * block_rows, _blocks(cols) * BLOCK), device=x.device)
    wide[:rows, :cols] = x.abs()
    top = wide.view(-1, block_rows, _blocks(cols), BLOCK).amax((1, 3))
    bits = top.contiguous().view(torch.int32)
    # 448 = 1.75 * 2^8: one binade more where the fraction is above 0.75
    scales = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000)).clamp_(min=1).to(torch.uint8)
    return scales.T.contiguous() if block_rows == 1 else scales


def _quantize(x, block_rows, seed):
    """(codes, scales): e4m3 of the elements over their block's scale, to the nearest (ties to even) or, with a seed, to one
    of the two neighbours with the probability of the place between them."""
    x = x.float()
    rows, cols = x.shape
    scales = _exponents(x, block_rows)
    y = x * torch.exp2(127 - _exponent_of_each(scales, rows, cols, block_rows))
    if seed is None:
        return y.to(torch.float8_e4m3fn), scales
    units = -(-cols // 8)                                     # eight neighbours of a row share a generator call
    random = _random16(torch.arange(rows * units, device=x.device), 3, seed).view(rows, units * 8)[:, :cols]
    exponent = (y.abs().view(torch.int32) >> 23).clamp_(min=121)
    steps = torch.floor(y.abs() * ((257 - exponent) << 23).view(torch.float32) + random.float() * 2.0 ** -16)
    codes = ((exponent - 121) << 3) + steps.int() | ((y.view(torch.int32) >> 31) & 0x80)
    return codes.to(torch.uint8).view(torch.float8_e4m3fn), scales


def _exponent_of_each(scales, rows, cols, block_rows):
    e = scales.float()
    if block_rows == 1:
        return e.T.repeat_interleave(BLOCK, 1)[:, :cols]
    return e.repeat_interleave(BLOCK, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def _gemm(st):
    a = st["a"].float() * _per_element(st["a_scales"], *st["a"].shape, 1)
    w = st["w"].float() * _per_element(st["w_scales"], *st["w"].shape, BLOCK)
    return (a @ (w.T if st["forward"] else w)).to(st["dtype"])


def _orthogonalize(x, steps):
    a, b, c = POLYNOMIAL
    flip = x.shape[1] > x.shape[2]
    if flip:
        x = x.transpose(1, 2)
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for _ in range(steps):
        s = x @ x.transpose(1, 2)
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.transpose(1, 2) if flip else x


def _muon(st):
    g = st["grad"].float()
    st["m"] = st["m"] * st["momentum"] + g * (1 - st["momentum"])
    x = st["m"] * st["momentum"] + g * (1 - st["momentum"])            # Nesterov's look ahead
    rows, cols = x.shape[1:]
    x = _orthogonalize(x, st["steps"])
    weight = st["param"].float() * (1 - st["lr"] * st["decay"]) - x * (st["lr"] * 0.2 * math.sqrt(max(rows, cols)))
    if st["case"]["stochastic"]:
        n = rows * cols
        padded = -(-n // 256) * 256                                    # each matrix counts up to a multiple of 256 elements
        units = torch.arange(st["case"]["tensors"] * padded // 8, device=g.device)
        random = _random16(units, 2, st["seed"] + st["step"]).view(-1, padded)[:, :n].reshape(weight.shape)
        bits = (weight.view(torch.int32) + random.int()) & -65536
        weight = bits.view(torch.float32)
    st["param"] = weight.to(torch.bfloat16)


def run(state):
    st, op = state, state["case"]["op"]
    if not own:
        if op == "ln_fwd":
            return _ln_forward(st)
        if op == "ln_bwd":
            return _ln_backward(st)
        if op == "quant":
            return _quantize(st["x"], st["block_rows"], st["seed"])
        if op == "gemm":
            return _gemm(st)
        if op == "ortho":
            return _orthogonalize(st["x"].float(), st["steps"]).to(torch.bfloat16).contiguous()
        _muon(st)
        st["step"] += 1
        return st["param"], st["m"]
    from paper_2203_10991_b200 import binding
    if op == "ln_fwd":
        return binding.mvue_layer_norm(st["x"], st["weight"], st["bias"], eps=st["eps"])
    if op == "ln_bwd":
        return binding.mvue_layer_norm_backward(st["dy"], st["x"], st["mean"], st["rstd"], st["weight"])
    if op == "quant":
        return binding.mvue_quantize_e4m3(st["x"], st["block_rows"], seed=st["seed"])
    if op == "gemm":
        product = binding.mvue_scaled_forward_gemm if st["forward"] else binding.mvue_scaled_backward_gemm
        return product(st["a"], st["a_scales"], st["w"], st["w_scales"], out_dtype=st["dtype"])
    if op == "ortho":
        return binding.mvue_orthogonalize(st["x"], steps=st["steps"], out_dtype=torch.bfloat16)
    st["plan"].step(lr=st["lr"], momentum=st["momentum"], nesterov=True, weight_decay=st["decay"], ns_steps=st["steps"], scale="rms",
                    stochastic_rounding=st["case"]["stochastic"], seed=st["seed"] + st["step"])
    st["step"] += 1
    return st["param"], st["m"]


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _exact_ln(st):
    x, w = st["x"].double(), st["weight"].double()
    if st["case"]["op"] == "ln_fwd":
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + st["eps"]) ** -0.5
        return torch.addcmul(st["bias"].double(), (x - mean[:, None]) * rstd[:, None], w), mean, rstd
    dy, rstd = st["dy"].double(), st["rstd"].double()[:, None]
    x.sub_(st["mean"].double()[:, None]).mul_(rstd)
    along = torch.einsum("rc,rc,c->r", dy, x, w)[:, None]
    plain = (dy @ w)[:, None]
    n = x.shape[1]
    return rstd * (w * dy - (plain + x * along) / n), torch.einsum("rc,rc->c", dy, x), torch.einsum("rc->c", dy)


def _exact_quant(st):
    x = st["x"].double()
    rows, cols = x.shape
    r, c = torch.arange(rows, device=x.device) // st["block_rows"], torch.arange(cols, device=x.device) // BLOCK
    by_cols = torch.zeros((rows, _blocks(cols)), dtype=torch.float64, device=x.device).index_reduce_(1, c, x.abs(), "amax")
    top = torch.zeros((int(r[-1]) + 1, _blocks(cols)), dtype=torch.float64, device=x.device).index_reduce_(0, r, by_cols, "amax")
    _, e = torch.frexp(top / E4M3_MAX)                        # top / 448 = f 2^e, 0.5 <= f < 1
    e = torch.where(top / E4M3_MAX == torch.exp2((e - 1).double()), e - 1, e).clamp(min=-126)
    values = torch.exp2(-e.double())[r][:, c]
    return x * values, ((e + 127).T if st["block_rows"] == 1 else e + 127).to(torch.uint8)


def _exact_gemm(st):
    t, k = st["a"].shape
    index = torch.arange(k, device="cuda") // BLOCK
    a = torch.ldexp(st["a"].double(), st["a_scales"].int()[index].T - 127)
    o, i = (torch.arange(n, device="cuda") // BLOCK for n in st["w"].shape)
    w = torch.ldexp(st["w"].double(), st["w_scales"].int()[o][:, i] - 127)
    return torch.einsum("tk,nk->tn" if st["forward"] else "tk,kn->tn", a, w)


def _exact_ortho(u, steps):
    wide = u.shape[1] <= u.shape[2]
    u = u / (torch.linalg.matrix_norm(u, keepdim=True) + 1e-7)
    for _ in range(steps):
        # the odd polynomial of degree five from the left or from the right, whichever Gram matrix is the smaller
        gram = torch.bmm(u, u.mT) if wide else torch.bmm(u.mT, u)
        series = torch.baddbmm(gram, gram, gram, beta=POLYNOMIAL[1], alpha=POLYNOMIAL[2])
        u = POLYNOMIAL[0] * u + (torch.bmm(series, u) if wide else torch.bmm(u, series))
    return u


def _exact_muon(st):
    if st["case"]["op"] == "ortho":
        return _exact_ortho(st["x"].double(), st["steps"])
    mu, lr = st["momentum"], st["lr"]
    g = st["grad"].double()
    m = mu * st["m"].double() + (1 - mu) * g
    u = _exact_ortho(torch.lerp(g, m, mu), st["steps"])
    weight = st["param"].double()
    return weight - lr * (st["decay"] * weight + 0.2 * max(u.shape[1:]) ** 0.5 * u), m


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    return {"ln_fwd": _exact_ln, "ln_bwd": _exact_ln, "quant": _exact_quant, "gemm": _exact_gemm, "muon": _exact_muon, "ortho": _exact_muon}[case["op"]](st)
