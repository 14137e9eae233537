"""The AdamW step with 8-bit states as the header defines it, in torch binary32 on the device (large tensors): every
operation rounded on its own, the root correctly rounded by way of 64 bits."""
import torch

BLOCK = 256


def random16(units: int, seed: int, device) -> torch.Tensor:
    """Eight 16-bit numbers for each of the units 0 .. units - 1, low halves first (int32)."""
    low = 0xFFFFFFFF
    u = torch.arange(units, device=device)
    c0, c1, c2, c3 = u & low, u >> 32, torch.full_like(u, 2), torch.zeros_like(u)
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1).int()


def quantise(x: torch.Tensor, random: torch.Tensor, floor_one: bool):
    """(codes uint8, scales) of fp32 x, whole blocks; `random` 16-bit numbers."""
    top = x.view(-1, BLOCK).abs().amax(1, keepdim=True)
    large = top >= 2.0 ** -110
    factor = torch.where(large, top.reciprocal() * 448.0, 0.0)
    y = (x.view(-1, BLOCK).abs() * factor).clamp_(max=448.0).reshape(-1)
    e = (y.view(torch.int32) >> 23).clamp_(min=121)                   # of the power of two, 2^-6 at least
    # the product by a power of two is exact; the sum is rounded to binary32 (below 2^-6 it may have more digits)
    steps = torch.floor(y * ((257 - e) << 23).view(torch.float32) + random.float() * 2.0 ** -16)
    codes = ((e - 121) << 3) + steps.int()
    if floor_one:
        codes = torch.where(x > 0, codes.clamp(min=1), codes)
    return (codes | ((x < 0).int() << 7)).to(torch.uint8), torch.where(large, top * (1.0 / 448.0), 0.0).reshape(-1)


class States:
    """Codes and scales of m and sqrt(v) of one tensor of whole blocks, zero at first."""

    def __init__(self, n: int, device):
        self.m, self.v = (torch.zeros(n, dtype=torch.uint8, device=device) for _ in range(2))
        self.ms, self.vs = (torch.zeros(n // BLOCK, device=device) for _ in range(2))

    @staticmethod
    def _values(codes, scales):
        return (codes.view(torch.float8_e4m3fn).float().view(-1, BLOCK) * scales[:, None]).reshape(-1)

    def step(self, g: torch.Tensor, beta1: float, beta2: float, seed: int):
        """The new moments (binary32, before they are rounded to codes)."""
        m, root = self._values(self.m, self.ms), self._values(self.v, self.vs)
        m = m * beta1 + g * (1 - beta1)
        v = (root * root) * beta2 + (g * (1 - beta2)) * g
        root = v.double().sqrt().float()
        r = random16(g.numel() // 8, seed, g.device)
        r = (r & 255) << 8 | r >> 8
        (self.m, self.ms), (self.v, self.vs) = quantise(m, r, False), quantise(root, r, True)
        return m, v
