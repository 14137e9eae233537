"""Layer norm, e4m3 codes and the Muon step in 64 bits (or whole numbers), and how far binary32 arithmetic may be from them.

The bounds are first-order: U = 2^-24 per rounding, sums of n terms in any order within their depth of additions times U times the
sum of magnitudes."""
import numpy as np
import torch

U = 2.0 ** -24
HALF_STEP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}       # of the one rounding to the output type (fp32: counted in U)
DEPTH = 100                     # additions that an element of a row's sum goes through at most: 32 in a thread, a warp's and a block's joins, or
                                # one in 1024 of up to 2^15 elements and the joins


def layer_norm(x, w, b, eps):
    """(y, mean, rstd) in 64 bits and bounds of their errors."""
    x = x.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros_like(w) if b is None else b.double()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    var = d.square().mean(-1, keepdim=True)
    rstd = (var + eps).rsqrt()
    xh = d * rstd
    y = xh * w + b
    top = x.abs().amax(-1, keepdim=True)
    d_mean = DEPTH * U * x.abs().mean(-1, keepdim=True) + 4 * U * top         # a thread's own mean is added and taken away again
    # the variance about a mean that is off by d_mean is off by its square and the roundings; each difference is off by 2 U top + d_mean
    d_d = d_mean + 4 * U * top
    d_var = 2 * d_d * d.abs().mean(-1, keepdim=True) + d_d.square() + (DEPTH + 4) * U * var
    d_rstd = rstd * (0.5 * d_var / (var + eps) + 6 * U)                      # rsqrtf: 2 units in the last place
    d_y = w.abs() * (rstd * d_d + d.abs() * d_rstd) + 4 * U * (xh * w).abs() + 2 * U * (b.abs() + y.abs())
    return (y, mean.squeeze(-1), rstd.squeeze(-1)), (d_y, d_mean.squeeze(-1), d_rstd.squeeze(-1))


def layer_norm_backward(dy, x, mean, rstd, w):
    """(dx, dw, db) in 64 bits for the given statistics, and bounds of their errors."""
    cols = x.shape[-1]
    x, dy = x.double().reshape(-1, cols), dy.double().reshape(-1, cols)
    w = torch.ones(cols, dtype=torch.float64, device=x.device) if w is None else w.double()
    mean, rstd = mean.double().reshape(-1, 1), rstd.double().reshape(-1, 1)
    xh = (x - mean) * rstd
    g = dy * w
    m0, m1 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = rstd * (g - m0 - xh * m1)
    e0 = (DEPTH + 4) * U * g.abs().mean(1, keepdim=True)
    e1 = (DEPTH + 8) * U * (g * xh).abs().mean(1, keepdim=True)
    d_dx = rstd * (e0 + xh.abs() * e1 + 8 * U * (g.abs() + m0.abs() + (xh * m1).abs()))
    rows = x.shape[0]
    deep = (rows // 16 + DEPTH) * U                                          # a thread's rows one after another, then the joins
    return (dx, (dy * xh).sum(0), dy.sum(0)), (d_dx, (deep + 6 * U) * (dy * xh).abs().sum(0), deep * dy.abs().sum(0))


# ---- e4m3 ------------------------------------------------------------------------------------------------------------

def philox_halves(units, stream, seed):
    """Eight 16-bit numbers for each generator call (unit): Philox4x32-10, counter (low, high, stream, 0)."""
    mask = np.uint64(0xFFFFFFFF)
    units = np.asarray(units, dtype=np.uint64)
    c = [units & mask, units >> np.uint64(32), np.full_like(units, stream), np.zeros_like(units)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & mask, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & mask]
        k0, k1 = k0 + 0x9E3779B9 & 0xFFFFFFFF, k1 + 0xBB67AE85 & 0xFFFFFFFF
    return np.stack([half for w in c for half in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 1).astype(np.int64)


def quantize(x, block_rows, seed=None):
    """(codes uint8, scales uint8) of a float32 array [rows, cols], element for element as the definition says."""
    x = np.asarray(x, dtype=np.float32)
    rows, cols = x.shape
    blocks, high = -(-cols // 128), -(-rows // block_rows)
    finite = np.isfinite(x)
    wide = np.zeros((high * block_rows, blocks * 128))
    wide[:rows, :cols] = np.where(finite, np.abs(x), 0)
    top = wide.reshape(high, block_rows, blocks, 128).max((1, 3))
    e = np.ones(top.shape, dtype=np.int64)
    for byte in range(2, 255):                                               # the least byte that brings the top to 448 or less
        e[top > 448.0 * 2.0 ** (byte - 1 - 127)] = byte
    spread = np.repeat(np.repeat(e, block_rows, 0)[:rows], 128, 1)[:, :cols]
    z = np.where(finite, np.abs(x), 0).astype(np.float64) * 2.0 ** (127.0 - spread)
    with np.errstate(divide="ignore"):
        binade = np.maximum(np.floor(np.log2(z)), -6).astype(np.int64)       # exact: z has 24 bits
    over = z >= 2.0 ** (binade + 1)                                          # (log2 of a number just below a power of two)
    binade = np.where(over, binade + 1, np.where((z < 2.0 ** binade) & (binade > -6), binade - 1, binade))
    steps = z * 2.0 ** (3.0 - binade)                                        # in units of the distance of two codes, 8 .. 16 above 2^-6
    if seed is None:
        whole = np.rint(steps).astype(np.int64)                              # ties to even
    else:
        units = -(-cols // 8)
        random = philox_halves(np.arange(rows * units), 3, seed).reshape(rows, units * 8)[:, :cols]
        whole = (np.rint(steps * 2.0 ** 20).astype(np.int64) + (random << 4)) >> 20
    codes = (binade + 6) * 8 + whole                                         # a carry into the next binade is the next code
    codes = np.where(finite, codes, 0x7F) | np.where(np.signbit(x), 0x80, 0)
    return codes.astype(np.uint8), (e.T if block_rows == 1 else e).astype(np.uint8)


def dequantize(codes, scales, block_rows):
    """The values in 64 bits of codes [rows, cols] and their scales (torch tensors)."""
    rows, cols = codes.shape
    e = scales.double().T if block_rows == 1 else scales.double().repeat_interleave(128, 0)[:rows]
    return codes.view(torch.float8_e4m3fn).double() * torch.exp2(e.repeat_interleave(128, 1)[:, :cols] - 127)


# ---- Muon ------------------------------------------------------------------------------------------------------------
A, B, C = 3.4445, -4.7750, 2.0315


def orthogonalize(x, steps=5):
    """The definition in 64 bits."""
    x = x.double()
    flip = x.shape[-2] > x.shape[-1]
    x = x.mT if flip else x
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + 1e-7)
    for _ in range(steps):
        s = x @ x.mT
        x = A * x + (B * s + C * (s @ s)) @ x
    return x.mT if flip else x


def orthogonalize_rounded(x, steps=5):
    """The same with the binary16 roundings of the operands (in the power-of-two scale S of the entries, S = 2^round(log2(n) / 2)), sums
    in 64 bits: X, A and a I + b A + c A A rounded once each step; what X loses is added to the product, a times it, in all steps but
    the last two."""
    x = x.double()
    flip = x.shape[-2] > x.shape[-1]
    x = x.mT if flip else x
    scale = 2.0 ** round(0.5 * np.log2(x.shape[-1]))
    h = lambda t: (t * scale).to(torch.float16).double() / scale             # noqa: E731
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + 1e-7)
    for k in range(steps):
        r = h(x)
        s = h(r @ r.mT)
        b = h(A * torch.eye(s.shape[-1], dtype=s.dtype, device=s.device) + B * s + C * (s @ s))
        x = b @ r + (A * (x - r) if k < steps - 2 else 0)
    return h(x).mT if flip else h(x)
