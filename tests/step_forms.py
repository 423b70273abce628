"""Plain 64-bit forms of the layer norm, the gradients' norm and the optimizer's step for the tests: torch on the CPU, written from
the formulas in include/aq_b200.h, without this library's code."""
import math

import torch

F64 = torch.float64
BLOCK = 256


def layer_norm(s, w, b, eps):
    """(y, mean, rstd) of binary64 rows."""
    mean = s.mean(1)
    rstd = 1 / torch.sqrt((s - mean[:, None]).square().mean(1) + eps)
    n = (s - mean[:, None]) * rstd[:, None]
    return n * w + b, mean, rstd


def layer_norm_grad(dy, dsum, s, w, mean, rstd):
    """(dx, dw, db)."""
    n, g = (s - mean[:, None]) * rstd[:, None], dy * w
    dx = rstd[:, None] * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    return (dx if dsum is None else dx + dsum), (dy * n).sum(0), dy.sum(0)


def clip(grads, inv_scale, max_norm):
    """(norm, factor)."""
    norm = inv_scale * math.sqrt(sum(g.double().square().sum().item() for g in grads))
    if not math.isfinite(norm):
        return norm, math.nan
    return norm, inv_scale * (min(1.0, max_norm / (norm + 1e-6)) if max_norm > 0 else 1.0)


def adamw(p, g, m, v, lr, decay, step, beta1=0.9, beta2=0.999, eps=1e-8):
    """(p, m, v) after a step."""
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    return p - lr * decay * p - lr * (m / (1 - beta1 ** step)) / (torch.sqrt(v / (1 - beta2 ** step)) + eps), m, v


def moments32(g, m, v, factor=1.0, beta1=0.9, beta2=0.999):
    """m and v of binary32 tensors after a step, every product and sum rounded to binary32."""
    f = lambda x: torch.tensor(x, dtype=torch.float32)  # noqa: E731
    g = g * f(factor)
    return m * f(beta1) + g * f(1 - beta1), v * f(beta2) + (g * g) * f(1 - beta2)


def random(n, step, begin=0):
    """(for m, for v): the whole numbers below 65536 of elements begin, begin + 1 ... at a step."""
    a, b, m = 0xBB67AE85, 0x9E3779B9, 1 << 32
    k = step * b % m
    k = (k ^ (k >> 16)) * a % m
    k = (k ^ (k >> 15)) * b % m
    k ^= k >> 16
    i = (torch.arange(begin, begin + n, dtype=torch.int64) + k) & (m - 1)
    u = torch.tensor([0], dtype=torch.int64)
    for factor, shift in ((a, 15), (b, 16)):                # products mod 2^32 from 16-bit halves, which stay small
        i = ((i & 0xFFFF) * factor + (((i >> 16) * (factor & 0xFFFF)) << 16)) & (m - 1)
        u = i = i ^ (i >> shift)
    return (u % 65536).double(), (u // 65536).double()


FORMATS = {"e4m3": (3, -6, 8), "e5m2": (2, -14, 15)}        # bits of the mantissa, smallest and largest exponent


def block_scales(x, kind):
    """Scale of every block of magnitudes x: the smallest power of two (not below 2^-126) that keeps the largest in range."""
    out = []
    for largest in [c.max().item() for c in x.split(BLOCK)]:
        k = -126
        if largest > 0:
            part, e = math.frexp(largest)                   # part in [1/2, 1)
            k = max(-126, e - 1 - FORMATS[kind][2] + (part > 0.875))
        out.append(2.0 ** k)
    return torch.tensor(out, dtype=F64)


def store8(x, random, kind):
    """(values in units of the scale, scales) that a binary32 moment is stored as."""
    bits, low, top = FORMATS[kind]
    mag = x.double().abs()
    scale = block_scales(mag, kind)
    z = mag / scale.repeat_interleave(BLOCK)[:x.numel()]
    step = torch.ldexp(torch.ones_like(z), (torch.frexp(z)[1] - 1).clamp(min=low) - bits)
    z = torch.floor(z / step + random / 65536) * step
    z = z.clamp(max=1.75 * 2.0 ** top)
    if kind == "e5m2":
        z = torch.where((z == 0) & (mag > 0), 2.0 ** -16, z)
    return torch.where(x < 0, -z, z), scale
