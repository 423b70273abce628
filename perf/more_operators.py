"""Layer norm and the optimizer's step of a pipeline stage: cases, plain forms and 64-bit values.

The models whose boundaries the codec serves normalise the residual stream with layer norms, and every visit of a
macro-batch ends in one step of the optimizer over all of the stage's tensors.  Four operators:

  norm / norm_grad   s = x + residual, y = (s - mean) rstd w + b; dx with the skip path's gradient, dw, db
  clip               the 2-norm of many tensors' gradients and the factor that unscales and clips them
  adamw              one AdamW step over many tensors, with the moments in 32 bits or in 8

`run` computes them with elementary torch operations in binary32 (`own` false) or by the library's calls (`own`
true); `exact` gives the same outputs in binary64 from the definitions.

The moments in 8 bits: m in e4m3, v in e5m2, each block of 256 elements of a tensor with a power of two as its scale,
the smallest that keeps the block's largest magnitude in range.  v moves by a thousandth of its value per step, far
less than half a step of any 8-bit format, so roundings are random, by 16-bit numbers that element i of a tensor has at
step t: the value goes up where its place between two neighbours and the number add up to one or more.  The numbers are
the halves of a hash of i and t (`_random`).  A v that is not zero does not become zero.
"""
import math

import torch

own = False

T = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"fp16": 2, "bf16": 2, "fp32": 4}
EPS_NORM, EPS_ADAM, BETA1, BETA2 = 1e-5, 1e-8, 0.9, 0.999
BLOCK = 256
ROOT3, GOLDEN = 0xBB67AE85, 0x9E3779B9      # the fractions of the square root of 3 and of the golden ratio, times 2^32


# ---- cases ------------------------------------------------------------------------------------------------

def listed():
    return [
        # decoding through a stage: the norm of one new token, GPT2-1.5B-shaped hidden size
        dict(name="norm one token", op="norm", rows=1, hidden=1600, pad=0, dtype="fp16", residual=True, affine=True),
        # one ragged sequence on a DeBERTa-1.5B-shaped stage, without a residual (its first norm)
        dict(name="norm sequence", op="norm", rows=1000, hidden=1536, pad=0, dtype="bf16", residual=False, affine=True),
        # the codec's macro-batch of 32 sequences of 1024, GPT2-1.5B-shaped
        dict(name="norm macro-batch", op="norm", rows=32768, hidden=1600, pad=0, dtype="fp16", residual=True, affine=True),
        # the backward pass of the small boundary's hidden size, a ragged number of rows
        dict(name="norm gradient small", op="norm_grad", rows=509, hidden=768, pad=0, dtype="bf16", residual=False, affine=True),
        # binary32 rows of an odd length, as a head of its own on top of the last stage has them
        dict(name="norm gradient odd", op="norm_grad", rows=4096, hidden=1021, pad=3, dtype="fp32", residual=True, affine=True),
        # the backward pass of the macro-batch, with the gradient that comes along the residual stream
        dict(name="norm gradient macro-batch", op="norm_grad", rows=32768, hidden=1600, pad=0, dtype="fp16", residual=True, affine=True),
        # the vectors of a stage's layer norms alone: the smallest call
        dict(name="clip vectors", op="clip", set="vectors", hidden=768, layers=2, packed=False, dtype="bf16", grads="fp32", scale=1.0),
        # every gradient of twelve GPT2-1.5B-shaped layers, scaled for fp16
        dict(name="clip stage", op="clip", set="layers", hidden=1600, layers=12, packed=False, dtype="fp16", grads="fp16", scale=1024.0),
        # fine-tuning nothing but the norms: many short vectors in binary32
        dict(name="adamw vectors", op="adamw", bits=32, set="vectors", hidden=768, layers=12, packed=False, dtype="fp32", grads="fp32",
             master=False, clip=False, clock=False),
        # a stage of six GPT2-1.5B-shaped layers: fp16 weights with binary32 copies and moments, clipped
        dict(name="adamw stage", op="adamw", bits=32, set="layers", hidden=1600, layers=6, packed=False, dtype="fp16", grads="fp16",
             master=True, clip=True, clock=False),
        # tensors of any length directly behind one another, as adapters and heads kept in one buffer are
        dict(name="adamw 8 bits odd", op="adamw", bits=8, set="odd", hidden=1021, layers=24, packed=True, dtype="bf16", grads="bf16",
             master=False, clip=True, clock=True),
        # the stage of twelve layers whose moments would not fit beside the codec's messages in 32 bits
        dict(name="adamw 8 bits stage", op="adamw", bits=8, set="layers", hidden=1600, layers=12, packed=False, dtype="bf16", grads="bf16",
             master=False, clip=True, clock=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "norm", "norm_grad", "clip", "adamw", "adamw", "adamw"])
    dtype = rng.choice(["fp16", "bf16", "fp32"])
    if op in ("norm", "norm_grad"):
        hidden = _log(rng, 16, 12000)
        if rng.random() < 0.6:
            hidden = (hidden + 7) // 8 * 8
        rows = _log(rng, 1, min(32768, 32768 * 1600 // (2 if dtype == "fp32" else 1) // hidden))
        return dict(op=op, rows=rows, hidden=hidden, pad=rng.choice([0, 0, 0, 8, 3]), dtype=dtype, residual=rng.random() < 0.6,
                    affine=rng.random() < 0.8)
    c = dict(op=op, set=rng.choice(["vectors", "layers", "layers", "odd"]), hidden=8 * _log(rng, 16, 256), layers=_log(rng, 1, 12),
             packed=rng.random() < 0.3, dtype=dtype, grads=rng.choice([dtype, dtype, "fp32"]))
    if c["set"] == "odd":
        c["hidden"], c["layers"] = _log(rng, 100, 4000), _log(rng, 1, 64)
    while _count(c) > 200e6:
        c["layers"] //= 2
    if op == "clip":
        return dict(c, scale=rng.choice([1.0, 128.0]))
    return dict(c, bits=rng.choice([32, 8, 8]), master=dtype != "fp32" and rng.random() < 0.4, clip=rng.random() < 0.6, clock=rng.random() < 0.4)


def _sizes(c):
    """[(elements, weight decay)] of the case's tensors."""
    d, out = c["hidden"], []
    for i in range(c["layers"]):
        if c["set"] == "layers":       # qkv and output projections, the gated feed-forward's three, two layer norms, query and key norms
            out += [(n, 0.01) for n in (3 * d * d, d * d, 4 * d * d, 4 * d * d, 4 * d * d)] + [(d, 0.0)] * 4 + [(64, 0.0)] * 2
        elif c["set"] == "vectors":
            out += [(d, 0.0)] * 4
        else:                          # lengths without a pattern, from one element to d^2
            out += [(1 + (i * 7919 + 13) % (3 * d), 0.0), (1 + (d * d * (i + 1)) // c["layers"], 0.1), (i % 5 + 1, 0.01)]
    return out


def _count(c):
    return sum(n for n, _ in _sizes(c))


def _places(c):
    """[(begin, elements, first block, blocks, weight decay)] of the tensors in the case's buffers, and the buffers' elements and blocks."""
    at = block = 0
    out = []
    for n, decay in _sizes(c):
        out.append((at, n, block, -(-n // BLOCK), decay))
        block += -(-n // BLOCK)
        at = at + n if c["packed"] else -(-(at + n) // BLOCK) * BLOCK
    return out, at, block


# ---- inputs -----------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _gradient(g, *shape):
    """Small with a few large entries, as gradients are."""
    x = 1e-3 * _normal(g, *shape)
    return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.01, 100 * x, x)


def _rows(c, x=None):
    """[rows, hidden] inside rows of hidden + pad elements, holding x."""
    buf = torch.zeros((c["rows"], c["hidden"] + c["pad"]), dtype=T[c["dtype"]], device="cuda")
    view = buf[:, :c["hidden"]]
    if x is not None:
        view.copy_(x)
    return view


def prepare(case, seed):
    c, g = case, _gen(seed)
    t = T[c["dtype"]]
    s = {"case": c}
    if c["op"] in ("norm", "norm_grad"):
        rows, d = c["rows"], c["hidden"]
        # a residual stream: some columns stand far out in every row, and a row's mean is not zero
        far = torch.where(torch.rand((d,), generator=g, device="cuda") < 0.005, 30.0, 1.0)
        x = _rows(c, _normal(g, rows, d) * far + 0.5 * _normal(g, rows, 1))
        s["w"], s["b"] = ((1 + 0.2 * _normal(g, d)).to(t), (0.1 * _normal(g, d)).to(t)) if c["affine"] else (None, None)
        s["mean"], s["rstd"] = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        if c["op"] == "norm":
            s["x"], s["y"] = x, _rows(c)
            s["residual"], s["sum"] = (_rows(c, 3 * _normal(g, rows, d)), _rows(c)) if c["residual"] else (None, None)
        else:
            s["s"], s["dy"], s["dx"] = x, _rows(c, _gradient(g, rows, d)), _rows(c)
            s["dsum"] = _rows(c, _gradient(g, rows, d)) if c["residual"] else None
            s["mean"], s["rstd"] = _statistics(x.float())        # as the forward call left them
            s["dw"], s["db"] = (torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")) if c["affine"] else (None, None)
        return s
    places, n, blocks = _places(c)
    step = int(torch.randint(1, 5000, (1,), generator=g, device="cuda")) if c["op"] == "adamw" else 0
    s.update(places=places, grad=(_gradient(g, n) * c.get("scale", 1.0)).to(T[c["grads"]]))
    if c["op"] == "clip":
        s.update(norm=torch.zeros(1, device="cuda"), factor=torch.zeros(1, device="cuda"), step=torch.zeros(1, dtype=torch.int64, device="cuda"))
        return s
    param = 0.05 * _normal(g, n)
    s.update(param=param.to(t), master=param if c["master"] else None)
    s.update(lr=1e-4, step=step, factor=torch.rand(1, generator=g, device="cuda") if c["clip"] else None)
    s["clock"] = (torch.tensor([s["lr"]], device="cuda"), torch.tensor([step], device="cuda")) if c["clock"] else None
    m, v = 3e-4 * _normal(g, n), (1e-3 * _normal(g, n)).square() + 1e-7
    if c["bits"] == 32:
        s.update(m=m, v=v)
    else:
        s.update(m=torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda"), v=torch.zeros(n, dtype=torch.float8_e5m2, device="cuda"),
                 m_scale=torch.zeros(blocks, device="cuda"), v_scale=torch.zeros(blocks, device="cuda"))
        for place in places:
            _store(s, place, m[place[0]:place[0] + place[1]], v[place[0]:place[0] + place[1]], step - 1)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------

def run(state):
    return (_library if own else _plain)[state["case"]["op"]](state)


def _statistics(x):
    mean = x.mean(1)
    return mean, torch.rsqrt((x - mean[:, None]).square().mean(1) + EPS_NORM)


def _outputs(s, *names):
    return {n: s[n] for n in names if s.get(n) is not None}


def _plain_norm(s):
    x, t = s["x"], s["x"].dtype
    if s["residual"] is not None:
        s["sum"].copy_((x.float() + s["residual"].float()).to(t))
        x = s["sum"]
    x = x.float()
    mean, rstd = _statistics(x)
    y = (x - mean[:, None]) * rstd[:, None]
    if s["w"] is not None:
        y = y * s["w"].float() + s["b"].float()
    s["y"].copy_(y.to(t))
    s["mean"].copy_(mean)
    s["rstd"].copy_(rstd)
    return _outputs(s, "y", "sum", "mean", "rstd")


def _plain_norm_grad(s):
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    n = (s["s"].float() - s["mean"][:, None]) * rstd
    if s["w"] is not None:
        s["db"].copy_(dy.sum(0))
        s["dw"].copy_((dy * n).sum(0))
        dy = dy * s["w"].float()
    dx = rstd * (dy - dy.mean(1, keepdim=True) - n * (dy * n).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    s["dx"].copy_(dx.to(s["dx"].dtype))
    return _outputs(s, "dx", "dw", "db")


def _parts(s, name):
    """The tensors of one of the case's buffers."""
    return [s[name][at:at + n] for at, n, *_ in s["places"]]


def _plain_clip(s):
    # squares in 64 bits: the sum is over up to a billion of them
    total = torch.stack([x.double().square().sum() for x in _parts(s, "grad")]).sum()
    inverse = 1 / s["case"]["scale"]
    norm = total.sqrt() * inverse
    factor = torch.where(norm.isfinite(), inverse * (1 / (norm + 1e-6)).clamp(max=1.0), math.nan)
    s["norm"].copy_(norm)
    s["factor"].copy_(factor)
    s["step"].add_(norm.isfinite())
    return _outputs(s, "norm", "factor", "step")


def _random(n, step):
    """16-bit numbers for m and v; all arithmetic mod 2^32."""
    k = (step * GOLDEN) & 0xFFFFFFFF
    k = ((k ^ (k >> 16)) * ROOT3) & 0xFFFFFFFF
    k = ((k ^ (k >> 15)) * GOLDEN) & 0xFFFFFFFF
    k = k ^ (k >> 16)
    u = ((torch.arange(n, device="cuda") + k) * ROOT3) & 0xFFFFFFFF
    u = ((u ^ (u >> 15)) * GOLDEN) & 0xFFFFFFFF
    u = u ^ (u >> 16)
    return (u & 0xFFFF).int(), (u >> 16).int()


def _blocks(x):
    """A tensor in rows of BLOCK elements, filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def _encode(x, random, mantissa, bias, top):
    """(codes, scales) of x >= 0 in the format with so many mantissa bits; `top`: its largest exponent."""
    drop = 23 - mantissa
    # 1.75 * 2^top is the largest value of either format: 1.75 and less of an octave stay in it
    largest = _blocks(x).amax(1).view(torch.int32)
    k = (((largest + (1 << 21) - 1) >> 23) - 127 - top).clamp(min=-126)
    # scaled so that the format's exponents are binary32's smallest, its subnormal numbers among them
    y = (_blocks(x) * ((127 - k) << 23).view(torch.float32)[:, None]).flatten()[:x.numel()] * 2.0 ** (bias - 127)
    return (y.view(torch.int32) + (random << (drop - 16))) >> drop, ((127 + k) << 23).view(torch.float32)


def _store(s, place, m, v, step):
    """A tensor's moments into the case's buffers."""
    at, n, block, blocks, _ = place
    um, uv = _random(n, step)
    code, s["m_scale"][block:block + blocks] = _encode(m.abs(), um, 3, 7, 8)
    code = code | ((m.view(torch.int32) >> 31) & 0x80)
    s["m"][at:at + n].view(torch.uint8).copy_(code)
    code, s["v_scale"][block:block + blocks] = _encode(v, uv, 2, 15, 15)
    code = torch.maximum(code, (v > 0).int())
    s["v"][at:at + n].view(torch.uint8).copy_(code)


def _load(s, name, place, real):
    at, n, block, blocks, _ = place
    x = s[name][at:at + n].to(real)
    if s["case"]["bits"] == 8:
        x = (_blocks(x) * s[name + "_scale"][block:block + blocks, None].to(real)).flatten()[:n]
    return x


def _clock(s, real):
    """(learning rate, 1 - beta1^t, 1 - beta2^t), numbers or tensors."""
    if s["clock"] is None:
        return s["lr"], 1 - BETA1 ** s["step"], 1 - BETA2 ** s["step"]
    lr, step = s["clock"]
    return lr.to(real), (1 - BETA1 ** step.double()).to(real), (1 - BETA2 ** step.double()).to(real)


def _plain_adamw_tensor(s, place, lr, c1, c2):
    at, n, *_, decay = place
    g = s["grad"][at:at + n].float()
    if s["factor"] is not None:
        g = g * s["factor"]
    m, v = _load(s, "m", place, torch.float32), _load(s, "v", place, torch.float32)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    p = (s["param"] if s["master"] is None else s["master"])[at:at + n]
    new = p.float() * (1 - lr * decay) - lr / c1 * (m / ((v / c2).sqrt() + EPS_ADAM))
    if s["case"]["bits"] == 32:
        s["m"][at:at + n], s["v"][at:at + n] = m, v
    else:
        _store(s, place, m, v, s["step"] if s["clock"] is None else s["clock"][1])
    if s["master"] is not None:
        s["master"][at:at + n] = new
    s["param"][at:at + n] = new.to(s["param"].dtype)


def _plain_adamw(s):
    now = _clock(s, torch.float32)
    [_plain_adamw_tensor(s, place, *now) for place in s["places"]]
    return _outputs(s, "param", "master", "m", "v", "m_scale", "v_scale")


_plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "clip": _plain_clip, "adamw": _plain_adamw}


# ---- the library's calls ----------------------------------------------------------------------------------

_stages = {}


def _stage(dtype):
    """The stage handle of an element type, made once as a program does."""
    import paper_2206_01299_b200 as aq
    if dtype not in _stages:
        st = aq.aq_stage_create()
        aq.aq_stage_configure(st, aq.AQ_DTYPE, {"fp16": aq.AQ_FP16, "bf16": aq.AQ_BF16, "fp32": aq.AQ_FP32}[dtype])
        _stages[dtype] = st
    return aq, _stages[dtype]


def _library_norm(s):
    c = s["case"]
    aq, st = _stage(c["dtype"])
    ld = c["hidden"] + c["pad"]
    aq.aq_layer_norm(st, s["x"], ld, s["residual"], ld, s["w"], s["b"], EPS_NORM, c["rows"], c["hidden"], s["sum"], ld, s["y"], ld,
                     s["mean"], s["rstd"])
    return _outputs(s, "y", "sum", "mean", "rstd")


def _library_norm_grad(s):
    c = s["case"]
    aq, st = _stage(c["dtype"])
    ld = c["hidden"] + c["pad"]
    aq.aq_layer_norm_grad(st, s["dy"], ld, s["dsum"], ld, s["s"], ld, s["w"], s["mean"], s["rstd"], c["rows"], c["hidden"], s["dx"], ld,
                          s["dw"], s["db"])
    return _outputs(s, "dx", "dw", "db")


def _table(aq, st, s):
    """The tensors' addresses, which a program lays out once, as its tensors keep their places from step to step."""
    if "table" not in s:
        if s["case"]["op"] == "clip":
            s["table"] = aq.aq_adam_table(st, grads=_parts(s, "grad"))
        else:
            scales = {}
            if s["case"]["bits"] == 8:
                scales = {n: [s[n][block:block + blocks] for _, _, block, blocks, _ in s["places"]] for n in ("m_scale", "v_scale")}
            s["table"] = aq.aq_adam_table(st, params=_parts(s, "param"), masters=None if s["master"] is None else _parts(s, "master"),
                                          grads=_parts(s, "grad"), m=_parts(s, "m"), v=_parts(s, "v"),
                                          weight_decay=[decay for *_, decay in s["places"]], **scales)
    return s["table"]


def _library_clip(s):
    aq, st = _stage(s["case"]["dtype"])
    aq.aq_grad_norm(st, _table(aq, st, s), len(s["places"]), 1 / s["case"]["scale"], 1.0, s["norm"], s["factor"], s["step"])
    return _outputs(s, "norm", "factor", "step")


def _library_adamw(s):
    aq, st = _stage(s["case"]["dtype"])
    if "config" not in s:
        s["config"] = aq.AdamwConfig(beta1=BETA1, beta2=BETA2, eps=EPS_ADAM, lr=s["lr"], step=s["step"], state_bits=s["case"]["bits"])
    lr, step = s["clock"] or (None, None)
    aq.aq_adamw(st, s["config"], _table(aq, st, s), len(s["places"]), s["factor"], lr, step)
    return _outputs(s, "param", "master", "m", "v", "m_scale", "v_scale")


_library = {"norm": _library_norm, "norm_grad": _library_norm_grad, "clip": _library_clip, "adamw": _library_adamw}


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] in ("norm", "norm_grad"):
        n, size, d = c["rows"] * c["hidden"], SIZE[c["dtype"]], c["hidden"]
        if c["op"] == "norm":
            return {"bytes": n * size * (4 if c["residual"] else 2) + 8 * c["rows"] + (2 * d * size if c["affine"] else 0), "flops": 8 * n}
        return {"bytes": n * size * (4 if c["residual"] else 3) + 8 * c["rows"] + (d * (size + 8) if c["affine"] else 0), "flops": 14 * n}
    n, g = _count(c), SIZE[c["grads"]]
    if c["op"] == "clip":
        return {"bytes": n * g + 16, "flops": 2 * n}
    weight = SIZE[c["dtype"]] + 8 if c["master"] else 2 * SIZE[c["dtype"]]
    moments = 16 if c["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (weight + g + moments), "flops": 16 * n}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def _round(x, random, mantissa, lowest, top):
    """Values of x >= 0 in blocks' scaled 8-bit format, and the scales: magnitudes and steps by exponents, no bit patterns."""
    rows = _blocks(x)
    largest = rows.amax(1)
    part, e = torch.frexp(largest)                            # largest = part 2^e, part in [1/2, 1)
    k = torch.where(largest > 0, e - 1 + (part > 0.875).int() - top, -126).clamp(min=-126)
    scale = torch.pow(2.0, k.double())
    z = rows / scale[:, None]
    step = torch.pow(2.0, (torch.frexp(z)[1] - 1).clamp(min=lowest).double() - mantissa)
    up = _blocks(random).double() / 65536
    z = (torch.floor(z / step + up) * step).clamp(max=1.75 * 2.0 ** top)
    return z.flatten()[:x.numel()], scale


def _exact_adamw_tensor(s, place, out):
    c, f64 = s["case"], torch.float64
    at, n, block, blocks, decay = place
    here = slice(at, at + n)
    g = s["grad"][here].to(f64) * (1.0 if s["factor"] is None else s["factor"].to(f64))
    m, v = _load(s, "m", place, f64), _load(s, "v", place, f64)
    m, v = torch.lerp(m, g, 1 - BETA1), torch.lerp(v, g ** 2, 1 - BETA2)
    lr = s["lr"] if s["clock"] is None else float(s["clock"][0])
    p = (s["param"] if s["master"] is None else s["master"])[here].to(f64)
    mhat, vhat = m / (1 - BETA1 ** s["step"]), v / (1 - BETA2 ** s["step"])
    p = p - lr * decay * p - lr * mhat / (torch.sqrt(vhat) + EPS_ADAM)
    out["param"][here] = p
    if s["master"] is not None:
        out["master"][here] = p
    if c["bits"] == 32:
        out["m"][here], out["v"][here] = m, v
        return
    um, uv = _random(n, s["step"])
    z, out["m_scale"][block:block + blocks] = _round(m.abs(), um, 3, -6, 8)
    out["m"][here] = torch.where(m < 0, -z, z)
    z, out["v_scale"][block:block + blocks] = _round(v, uv, 2, -14, 15)
    out["v"][here] = torch.where((z == 0) & (v > 0), 2.0 ** -16, z)


def exact(case, seed):
    """What run() returns, from the definitions in binary64: torch's layer norm and its differentiation, moments by interpolation."""
    s = prepare(case, seed)
    c, f64 = case, torch.float64
    if c["op"] in ("norm", "norm_grad"):
        shape = (c["hidden"],)
        w, b = (None if s[n] is None else s[n].to(f64).requires_grad_(True) for n in ("w", "b"))
        x = s["x" if c["op"] == "norm" else "s"].to(f64)
        if c["op"] == "norm":
            out = {}
            if s["residual"] is not None:
                x = (x + s["residual"].to(f64)).to(s["x"].dtype).to(f64)          # the stored sum is what is normalised
                out["sum"] = x
            var, mean = torch.var_mean(x, 1, correction=0)
            y = torch.nn.functional.layer_norm(x, shape, w, b, EPS_NORM).detach()
            return dict(out, y=y, mean=mean, rstd=(var + EPS_NORM) ** -0.5)
        x.requires_grad_(True)
        y = torch.nn.functional.layer_norm(x, shape, w, b, EPS_NORM)
        got = torch.autograd.grad(y, [x] if w is None else [x, w, b], s["dy"].to(f64))
        dx = got[0] if s["dsum"] is None else got[0] + s["dsum"].to(f64)
        return dict(dx=dx) if w is None else dict(dx=dx, dw=got[1], db=got[2])
    if c["op"] == "clip":
        norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(x, dtype=f64) for x in _parts(s, "grad")])) / c["scale"]
        return dict(norm=norm[None], factor=(torch.minimum(torch.ones_like(norm), 1 / (norm + 1e-6)) / c["scale"])[None], step=None)
    names = ["param", "m", "v"] + (["master"] if s["master"] is not None else []) + (["m_scale", "v_scale"] if c["bits"] == 8 else [])
    out = {n: torch.zeros(s[n].shape, dtype=f64, device="cuda") for n in names}
    if not c["packed"]:                                       # what lies between the tensors stays as it was
        for n in names[:4]:
            if not n.endswith("scale"):
                out[n].copy_(s[n].to(f64))
    for place in s["places"]:
        _exact_adamw_tensor(s, place, out)
    return out
