"""Plain forms, in 64 bits on the CPU, of dropout, the linear layer and its gradient, with the
magnitudes that tolerances are made of."""
import math

import numpy as np

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85


def philox(counter, key):
    """Philox4x32-10 (Salmon et al. 2011): arrays of 4 counter words, 2 key words -> 4 words."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(v, np.uint64) for v in counter]
    k0, k1 = key
    for _ in range(10):
        a, b = c[0] * np.uint64(M0), c[2] * np.uint64(M1)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + W0) & 0xFFFFFFFF, (k1 + W1) & 0xFFFFFFFF
    return c


def limit(p):
    return math.floor(float(np.float32(p)) * 65536 + 0.5)


def factors(rows, cols, p, seed, draw):
    """What dropout multiplies each element by, float64 [rows, cols]."""
    groups = -(-cols // 8)
    c, r = np.meshgrid(np.arange(groups), np.arange(rows))
    words = philox([c, r, np.full_like(c, draw & 0xFFFFFFFF), np.full_like(c, draw >> 32)],
                   (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.empty((rows, groups, 8), np.uint64)
    for e in range(8):
        bits[:, :, e] = (words[e // 2] >> np.uint64(16 * (e % 2))) & np.uint64(0xFFFF)
    t = limit(p)
    scale = 65536.0 / (65536 - t) if t < 65536 else 0.0
    return np.where(bits.reshape(rows, groups * 8)[:, :cols] >= t, scale, 0.0)


def activate(torch, act, z):
    """act(z) and its slope."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if act == "gelu":
        cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "tanh":
        return torch.tanh(z), 1 / torch.cosh(z) ** 2
    s = torch.sigmoid(z)
    return (z * s, s + z * s * torch.sigmoid(-z)) if act == "silu" else (s, s * torch.sigmoid(-z))


HALF = {"float32": 2.0**-24, "bfloat16": 2.0**-8, "float16": 2.0**-11}
# half of the smallest subnormal
FLOOR = {"float32": 0.0, "bfloat16": 0.0, "float16": 2.0**-25}
# activations and slopes: relative to the largest factor in them.  The fit of the normal
# distribution is 7.3e-7 off, exponentials and quotients a few units of 2^-24; 16-bit types leave
# the exponent's rounding in, |v| 2^-24 of exp(v)
FUNCTION = {"float32": 2.0**-20, "bfloat16": 2.0**-16, "float16": 2.0**-16}
UNIT = 2.0**-24
