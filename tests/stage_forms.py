"""Plain 64-bit forms of the stage operators for the tests: torch on the CPU in binary64, written from the formulas in
include/aq_b200.h, without this library's code."""
import math

import torch

F64 = torch.float64
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
UNIT = {"fp16": 2.0 ** -11, "bf16": 2.0 ** -8, "fp32": 2.0 ** -24}      # one rounding to nearest: |error| <= UNIT |x| (bf16: 8 bits)
TINY = {"fp16": 2.0 ** -25, "bf16": 2.0 ** -134, "fp32": 2.0 ** -150}   # ... and below the normal range


def logprobs(x, targets, scale, k):
    """(logprob, entropy, lse, top ids, top logprobs) of one row of binary64 logits; `scale` as binary64."""
    v = x.numel()
    z = x * scale
    m = z.max().item()
    if m == -math.inf:
        return (-math.inf if targets >= 0 else 0.0), 0.0, -math.inf, torch.arange(k), torch.full((k,), -math.inf, dtype=F64)
    e = torch.exp(z - m)
    s = e.sum()
    lp = z - m - torch.log(s)
    p = e / s
    entropy = -(p * torch.where(p > 0, lp, torch.zeros_like(lp))).sum().item()
    order = torch.sort(x + 0.0, descending=True, stable=True).indices[:k]
    return (lp[targets].item() if 0 <= targets < v else 0.0), entropy, m + math.log(s.item()), order, lp[order]


def logprobs_grad(x, target, scale, gl, gh):
    """Gradient of gl * logprob + gh * entropy by the formula."""
    z = x * scale
    if z.max().item() == -math.inf:
        return torch.zeros_like(x)
    lp = torch.log_softmax(z, 0)
    p = lp.exp()
    lp = torch.where(p > 0, lp, torch.zeros_like(lp))
    h = -(p * lp).sum()
    g = -gh * p * (lp + h)
    if 0 <= target < x.numel():
        g = g - gl * p
        g[target] += gl
    return g * scale


def act(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return 0.5 * g * torch.erfc(-g / math.sqrt(2.0))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def act_grad(name, g):
    g = g.clone().requires_grad_(True)
    return torch.autograd.grad(act(name, g).sum(), g)[0]


def ffn(x, wg, wu, name):
    g, u = x @ wg.T, x @ wu.T
    return act(name, g) * u, g, u


def ffn_grad(dh, x, wg, wu, g, u, name):
    dg, du = dh * u * act_grad(name, g), dh * act(name, g)
    return dg, du, dg @ wg + du @ wu, dg.T @ x, du.T @ x


def qk(x, w, eps, cos_sin, positions, rot, interleaved):
    """x [rows, heads, head_dim]; differentiable."""
    y = w * x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if rot == 0:
        return y
    f = cos_sin[positions]
    cos, sin = f[:, None, :rot // 2], f[:, None, rot // 2:]
    if interleaved:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([r, y[..., rot:]], -1)
