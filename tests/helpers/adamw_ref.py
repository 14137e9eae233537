"""Plain AdamW steps for the tests: in 64 bits from the formulas, and the 8-bit states' codes in numpy binary32."""
import numpy as np

from oracle import philox_py

BLOCK = 256
F = np.float32


def random16(first_unit: int, units: int, seed: int) -> np.ndarray:
    """Eight 16-bit numbers for each unit (low halves first), by the big-integer generator."""
    out = np.empty((units, 8), np.uint32)
    key = (seed & 0xFFFFFFFF, seed >> 32)
    for i in range(units):
        u = first_unit + i
        words = philox_py.philox4x32((u & 0xFFFFFFFF, u >> 32, 2, 0), key)
        for j, w in enumerate(words):
            out[i, 2 * j], out[i, 2 * j + 1] = w & 0xFFFF, w >> 16
    return out.reshape(-1)


def e4m3_values() -> np.ndarray:
    """The 256 values of the 8-bit format, from its definition (no infinities; 0x7F and 0xFF are not used here)."""
    code = np.arange(256)
    e, f = (code >> 3) & 15, code & 7
    mag = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    return np.where(code & 128, -mag, mag)


def scale_of(top: np.ndarray):
    """(scale, factor to codes) of blocks whose largest magnitudes are `top`."""
    with np.errstate(divide="ignore", over="ignore"):
        factor = F(448) * (F(1) / top)
    factor = np.where((top >= F(2.0 ** -110)) & np.isfinite(top), factor, F(0)).astype(F)
    scale = np.where(top >= F(2.0 ** -110), top * (F(1) / F(448)), F(0)).astype(F)
    return np.where(np.isfinite(top), scale, F(np.nan)).astype(F), factor


def quantise(x: np.ndarray, random: np.ndarray, floor_one: bool):
    """codes, scales of fp32 x (any length): each block by its largest magnitude, rounded up where the fraction of a step
    plus random / 2^16 reaches one.  In 64 bits from the binary32 product on: nothing is rounded there."""
    n = x.size
    pad = -n % BLOCK
    xp = np.pad(x, (0, pad)).reshape(-1, BLOCK)
    scale, factor = scale_of(np.abs(xp).max(1))
    y = np.minimum((np.abs(xp) * factor[:, None]).astype(F), F(448)).astype(np.float64).reshape(-1)[:n]
    e = np.maximum(np.floor(np.log2(np.maximum(y, 1e-300))), -6)
    k = np.floor(y / 2.0 ** (e - 3) + random / 65536.0)
    code = (8 * (e + 6) + k).astype(np.int64)
    if floor_one:
        code = np.where(x > 0, np.maximum(code, 1), code)
    return (code | np.where(x < 0, 128, 0)).astype(np.uint8), scale


def moments32(g, m, v, beta1, beta2, grad_scale=1.0):
    """m', v' in binary32, each operation rounded on its own (numpy arrays of float32)."""
    g = g * F(grad_scale)
    return F(beta1) * m + F(1 - beta1) * g, F(beta2) * v + (F(1 - beta2) * g) * g


def step64(p, g, m, v, *, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    """(p', m', v') in 64 bits."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = g * grad_scale
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    with np.errstate(invalid="ignore", divide="ignore"):
        upd = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return p - lr * weight_decay * p - lr * upd, m, v
