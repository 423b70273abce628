"""The operators of a pipeline stage's own work beside the boundary codec: cases, plain forms and 64-bit values.

Between two boundaries a stage of a language model normalises and rotates the queries and keys of its
attention layers, runs gated feed-forward blocks, and, on the last stage, turns logits into the loss.  Three
operators, each with its backward direction:

  logprob / logprob_grad   log probabilities of given tokens with entropy and top alternatives; d logits
  ffn / ffn_grad           h = act(x Wg^T) * (x Wu^T); dx, dWg, dWu
  qk / qk_grad             RMS norm of every query and key head with the position rotation; dq, dk, dwq, dwk

`run` computes them with elementary torch operations in binary32 (`own` false) or by the library's calls
(`own` true); `exact` gives the same outputs in binary64 from the definitions.
"""
import math

import torch

own = False

T = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"fp16": 2, "bf16": 2, "fp32": 4}
LOWEST = {"fp16": -65504.0, "bf16": -3.3895313892515355e38, "fp32": -3.4028234663852886e38}
EPS = 1e-6


# ---- cases ------------------------------------------------------------------------------------------------

def listed():
    return [
        # sampling: the logits of one new token, unpadded GPT2 vocabulary, eight alternatives reported
        dict(name="logprob one token", op="logprob", rows=1, vocab=50257, pad=0, dtype="fp32", top_k=8, mask=0.1, scale=1.25),
        # one sequence of 1024 tokens; the odd vocabulary leaves every second row of fp16 logits off a word boundary
        dict(name="logprob sequence", op="logprob", rows=1024, vocab=50257, pad=0, dtype="fp16", top_k=4, mask=0.0, scale=1.0),
        # a macro-batch of eight sequences on the last stage, vocabulary padded by the model's head
        dict(name="logprob macro-batch", op="logprob", rows=8192, vocab=50304, pad=0, dtype="bf16", top_k=5, mask=0.02, scale=1.0),
        # the loss's gradient for half a macro-batch, with an entropy term; rows padded to 16 bytes
        dict(name="logprob gradient", op="logprob_grad", rows=4096, vocab=50257, pad=7, dtype="bf16", mask=0.02, scale=1.0),
        # decoding through a stage: one token, GPT2-1.5B-shaped hidden size
        dict(name="ffn one token", op="ffn", rows=1, hidden=1600, inner=6400, dtype="fp16", act="silu", save=False),
        # one ragged sequence on a DeBERTa-1.5B-shaped stage, kept for the backward pass
        dict(name="ffn sequence", op="ffn", rows=1000, hidden=1536, inner=4096, dtype="bf16", act="gelu", save=True),
        # a macro-batch of eight GPT2-1.5B-shaped sequences, kept for the backward pass
        dict(name="ffn macro-batch", op="ffn", rows=8192, hidden=1600, inner=6400, dtype="fp16", act="silu", save=True),
        # the backward pass of the small boundary's hidden size, a ragged number of rows
        dict(name="ffn gradient small", op="ffn_grad", rows=509, hidden=768, inner=2048, dtype="bf16", act="gelu_tanh"),
        # the backward pass of a macro-batch: the costliest call of a training step
        dict(name="ffn gradient macro-batch", op="ffn_grad", rows=8192, hidden=1600, inner=6400, dtype="fp16", act="silu"),
        # decoding: the queries and keys of one token, 25 heads of 64
        dict(name="qk one token", op="qk", rows=1, heads_q=25, heads_k=25, head_dim=64, rot=64, interleaved=False, dtype="fp16"),
        # a macro-batch of 32 sequences of 1024
        dict(name="qk macro-batch", op="qk", rows=32768, heads_q=25, heads_k=25, head_dim=64, rot=64, interleaved=False, dtype="fp16"),
        # the backward pass with shared key heads and a partial, interleaved rotation
        dict(name="qk gradient", op="qk_grad", rows=16384, heads_q=24, heads_k=8, head_dim=64, rot=32, interleaved=True, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprob", "logprob_grad", "ffn", "ffn_grad", "qk", "qk_grad"])
    if op in ("logprob", "logprob_grad"):
        dtype = rng.choice(["fp16", "bf16", "fp32"])
        vocab = _log(rng, 50, 130000)
        rows = _log(rng, 1, min(8192, max(1, 8192 * 50304 // (2 if dtype == "fp32" else 1) // vocab)))
        c = dict(op=op, rows=rows, vocab=vocab, pad=rng.choice([0, 0, 1, 8, -vocab % 8]), dtype=dtype,
                 mask=rng.choice([0.0, 0.02, 0.5]), scale=rng.choice([1.0, 0.7, 1.25]))
        if op == "logprob":
            c["top_k"] = rng.randint(0, 20)
        return c
    if op in ("ffn", "ffn_grad"):
        hidden, inner = 8 * _log(rng, 8, 256), 8 * _log(rng, 16, 800)
        c = dict(op=op, rows=_log(rng, 1, 8192), hidden=hidden, inner=inner, dtype=rng.choice(["fp16", "bf16"]),
                 act=rng.choice(["silu", "gelu", "gelu_tanh"]))
        while c["rows"] * hidden * inner > 8192 * 1600 * 6400:
            c["rows"] = c["rows"] // 2
        if op == "ffn":
            c["save"] = rng.choice([True, False])
        return c
    head_dim = 8 * rng.randint(4, 32)
    heads_k = rng.randint(1, 16)
    heads_q = heads_k * rng.choice([1, 1, 2, 3, 4])
    most = 32768 * 50 * 64 // ((heads_q + heads_k) * head_dim)
    return dict(op=op, rows=_log(rng, 1, max(1, min(32768, most))), heads_q=heads_q, heads_k=heads_k, head_dim=head_dim,
                rot=rng.choice([head_dim, head_dim, head_dim // 2, 16]), interleaved=rng.choice([False, True]),
                dtype=rng.choice(["fp16", "bf16"]))


# ---- inputs -----------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _gradient(g, *shape):
    """Small with a few large entries, as activation gradients are."""
    x = 1e-3 * _normal(g, *shape)
    return torch.where(torch.rand(shape, generator=g, device="cuda") < 0.01, 100 * x, x)


def _empty(shape, dtype):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _prepare_logits(c, g):
    rows, vocab, t = c["rows"], c["vocab"], T[c["dtype"]]
    buf = _empty((rows, vocab + c["pad"]), t)
    logits = buf[:, :vocab]
    step = max(1, (1 << 28) // vocab)                 # in pieces: the binary32 normals of a whole macro-batch are 3 GB
    targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    for r in range(0, rows, step):
        x = 2.5 * _normal(g, min(step, rows - r), vocab)
        # what a trained model sees: the right token stands out in most rows
        x[torch.arange(x.shape[0], device="cuda"), targets[r:r + step]] += 8 * torch.rand((x.shape[0],), generator=g, device="cuda")
        if c["mask"]:                                 # forbidden tokens: -inf in even rows, the type's lowest value in odd ones
            off = torch.rand(x.shape, generator=g, device="cuda") < c["mask"]
            off[torch.arange(x.shape[0], device="cuda"), targets[r:r + step]] = False
            lowest = torch.where((torch.arange(x.shape[0], device="cuda") % 2 == 0)[:, None], -math.inf, LOWEST[c["dtype"]])
            x = torch.where(off, lowest, x)
        logits[r:r + step] = x.to(t)
    if c["pad"]:
        buf[:, vocab:] = 1000.0                       # padding is not part of the row
    if rows > 8:
        targets[torch.arange(5, rows, 97, device="cuda")] = -1      # positions without a token to predict
        if c["mask"]:
            logits[rows // 2] = -math.inf             # a row whose mask leaves nothing
    s = dict(logits=logits, ld=vocab + c["pad"], targets=targets.int())
    s["lse"], s["entropy"] = _empty((rows,), torch.float32), _empty((rows,), torch.float32)
    return s


def prepare(case, seed):
    c, g = case, _gen(seed)
    t = T[c["dtype"]]
    s = {"case": c}
    if c["op"] in ("logprob", "logprob_grad"):
        s.update(_prepare_logits(c, g))
        rows, vocab = c["rows"], c["vocab"]
        if c["op"] == "logprob":
            k = min(c["top_k"], vocab)
            s.update(k=k, logprob=_empty((rows,), torch.float32), top_ids=_empty((rows, k), torch.int32), top_logprobs=_empty((rows, k), torch.float32))
        else:
            # what the forward call left: binary32 values of the row's statistics
            lse, entropy = _statistics(s["logits"], c["scale"], torch.float32)
            s["lse"], s["entropy"] = lse, entropy
            s["d_logprob"] = -(0.5 + torch.rand((rows,), generator=g, device="cuda")) / rows
            s["d_entropy"] = 0.01 * _normal(g, rows) / rows
            s["d_logits"] = torch.zeros((rows, s["ld"]), dtype=t, device="cuda")
    elif c["op"] in ("ffn", "ffn_grad"):
        rows, d, f = c["rows"], c["hidden"], c["inner"]
        s["x"] = _normal(g, rows, d).to(t)
        s["wg"], s["wu"] = (_normal(g, f, d) / math.sqrt(d)).to(t), (_normal(g, f, d) / math.sqrt(d)).to(t)
        if c["op"] == "ffn":
            s["h"] = _empty((rows, f), t)
            s["g"], s["u"] = (_empty((rows, f), t), _empty((rows, f), t)) if c["save"] else (None, None)
        else:
            s["dh"] = _gradient(g, rows, f).to(t)
            s["g"], s["u"] = (s["x"].float() @ s["wg"].float().T).to(t), (s["x"].float() @ s["wu"].float().T).to(t)
            s["dx"], s["dwg"], s["dwu"] = _empty((rows, d), t), _empty((f, d), t), _empty((f, d), t)
    else:
        rows, dh, nq, nk = c["rows"], c["head_dim"], c["heads_q"], c["heads_k"]
        wide = (nq + 2 * nk) * dh                     # queries, keys and values of a token side by side, as one projection leaves them
        qkv = (1.5 * _normal(g, rows, wide)).to(t)
        s["q"], s["k"] = qkv[:, :nq * dh], qkv[:, nq * dh:(nq + nk) * dh]
        s["wq"], s["wk"] = (1 + 0.2 * _normal(g, dh)).to(t), (1 + 0.2 * _normal(g, dh)).to(t)
        n_pos = 2048
        s["positions"] = (torch.arange(rows, device="cuda") % n_pos if rows > 1 else torch.randint(0, n_pos, (1,), generator=g, device="cuda")).int()
        angle = torch.arange(n_pos, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64) * 2 / c["rot"])[None, :]
        s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        if c["op"] == "qk":
            s["q_out"], s["k_out"] = _empty((rows, nq * dh), t), _empty((rows, nk * dh), t)
        else:
            s["dq_out"], s["dk_out"] = _gradient(g, rows, nq * dh).to(t), _gradient(g, rows, nk * dh).to(t)
            s["dqkv"] = torch.zeros((rows, wide), dtype=t, device="cuda")
            s["dwq"], s["dwk"] = _empty((dh,), torch.float32), _empty((dh,), torch.float32)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------

def run(state):
    return (_library if own else _plain)[state["case"]["op"]](state)


def _statistics(logits, scale, real):
    """Log of the sum and entropy of every row; a row without a finite logit has none: -inf and 0."""
    z = logits.to(real) * scale
    m = z.amax(1)
    m = torch.where(m == -math.inf, 0.0, m)
    z -= m[:, None]
    e = z.exp()
    total = e.sum(1)
    z[z == -math.inf] = 0.0
    mean = (e * z).sum(1)
    lse = total.log() + m
    entropy = torch.where(total > 0, total.log() - mean / total, 0.0)
    return lse, entropy


def _plain_logprob(s):
    c, logits, targets = s["case"], s["logits"], s["targets"].long()
    lse, entropy = _statistics(logits, c["scale"], torch.float32)
    out = dict(lse=lse, entropy=entropy)
    at = logits.gather(1, targets.clamp(min=0)[:, None])[:, 0].float() * c["scale"]
    out["logprob"] = torch.where(targets >= 0, torch.where(lse == -math.inf, -math.inf, at - lse), 0.0)
    if s["k"]:
        # one key a logit: its value's order above, the place from the right below, so that ties go to the lowest id
        bits = (logits.float() + 0.0).view(torch.int32)
        order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long()
        key = order * (1 << 32) + (0xFFFFFFFF - torch.arange(c["vocab"], device="cuda"))
        ids = 0xFFFFFFFF - (key.topk(s["k"], 1).values & 0xFFFFFFFF)
        top = logits.gather(1, ids).float() * c["scale"] - lse[:, None]
        out["top_ids"], out["top_logprobs"] = ids.int(), torch.where(lse[:, None] == -math.inf, -math.inf, top)
    return out


def _plain_logprob_grad(s):
    c, targets = s["case"], s["targets"].long()
    lp = s["logits"].float() * c["scale"] - torch.where(s["lse"] == -math.inf, 0.0, s["lse"])[:, None]
    p = lp.exp()
    lp[lp == -math.inf] = 0.0
    gl = torch.where(targets >= 0, s["d_logprob"], 0.0)
    d = -p * (gl[:, None] + s["d_entropy"][:, None] * (lp + s["entropy"][:, None]))
    d[torch.arange(d.shape[0], device="cuda"), targets.clamp(min=0)] += gl
    d *= c["scale"]
    d[s["lse"] == -math.inf] = 0.0
    return d.to(s["logits"].dtype)


def _act(name, g):
    """act(g) and act'(g)."""
    if name == "gelu":
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    if name == "silu":
        y, dy = g, 1.0
    else:
        y = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        dy = 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g * g)
    sig = torch.sigmoid(y)
    return g * sig, sig + g * sig * (1 - sig) * dy


def _ffn(s, real):
    x, wg, wu = s["x"].to(real), s["wg"].to(real), s["wu"].to(real)
    g, u = x @ wg.T, x @ wu.T
    return _act(s["case"]["act"], g)[0] * u, g, u


def _plain_ffn(s):
    t = s["x"].dtype
    h, g, u = _ffn(s, torch.float32)
    return dict(h=h.to(t), g=g.to(t), u=u.to(t)) if s["case"]["save"] else h.to(t)


def _ffn_grad(s, real):
    x, wg, wu, dh, g, u = (s[k].to(real) for k in ("x", "wg", "wu", "dh", "g", "u"))
    a, da = _act(s["case"]["act"], g)
    dg, du = dh * u * da, dh * a
    return dict(dx=dg @ wg + du @ wu, dwg=dg.T @ x, dwu=du.T @ x)


def _plain_ffn_grad(s):
    return {k: v.to(s["x"].dtype) for k, v in _ffn_grad(s, torch.float32).items()}


def _cos_sin(s, real):
    """The rotation's factors of each row, [rows, 1, rot / 2]."""
    cs, half = s["cos_sin"][s["positions"].long()].to(real), s["case"]["rot"] // 2
    return cs[:, None, :half], cs[:, None, half:]


def _split(c, y):
    """First and second members of the rotated pairs, and what is not rotated; y [rows, heads, head_dim]."""
    rot = c["rot"]
    if c["interleaved"]:
        return y[..., 0:rot:2], y[..., 1:rot:2], y[..., rot:]
    return y[..., :rot // 2], y[..., rot // 2:rot], y[..., rot:]


def _join(c, a, b, rest):
    if c["interleaved"]:
        return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)
    return torch.cat([a, b, rest], -1)


def _norm_rotate(s, x, w, real):
    c = s["case"]
    x = x.unflatten(1, (-1, c["head_dim"])).to(real)
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(real)
    a, b, rest = _split(c, y)
    cos, sin = _cos_sin(s, real)
    return _join(c, a * cos - b * sin, b * cos + a * sin, rest).flatten(1)


def _norm_rotate_grad(s, dy, x, w, real):
    c = s["case"]
    x, dy = x.unflatten(1, (-1, c["head_dim"])).to(real), dy.unflatten(1, (-1, c["head_dim"])).to(real)
    a, b, rest = _split(c, dy)
    cos, sin = _cos_sin(s, real)
    dy = _join(c, a * cos + b * sin, b * cos - a * sin, rest)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dn = dy * w.to(real)
    return (r * (dn - n * (dn * n).mean(-1, keepdim=True))).flatten(1), (dy * n).sum((0, 1))


def _plain_qk(s):
    t = s["q"].dtype
    return dict(q=_norm_rotate(s, s["q"], s["wq"], torch.float32).to(t), k=_norm_rotate(s, s["k"], s["wk"], torch.float32).to(t))


def _plain_qk_grad(s):
    t = s["q"].dtype
    dq, dwq = _norm_rotate_grad(s, s["dq_out"], s["q"], s["wq"], torch.float32)
    dk, dwk = _norm_rotate_grad(s, s["dk_out"], s["k"], s["wk"], torch.float32)
    return dict(dq=dq.to(t), dk=dk.to(t), dwq=dwq, dwk=dwk)


_plain = {"logprob": _plain_logprob, "logprob_grad": _plain_logprob_grad, "ffn": _plain_ffn, "ffn_grad": _plain_ffn_grad,
          "qk": _plain_qk, "qk_grad": _plain_qk_grad}


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


def _act_key(aq, name):
    return {"silu": aq.AQ_ACT_SILU, "gelu": aq.AQ_ACT_GELU, "gelu_tanh": aq.AQ_ACT_GELU_TANH}[name]


def _library_logprob(s):
    c = s["case"]
    aq, st = _stage(c["dtype"])
    aq.aq_token_logprobs(st, s["logits"], c["rows"], c["vocab"], s["ld"], s["targets"], c["scale"], s["k"],
                         s["logprob"], s["entropy"], s["lse"], s["top_ids"], s["top_logprobs"])
    out = dict(lse=s["lse"], entropy=s["entropy"], logprob=s["logprob"])
    if s["k"]:
        out["top_ids"], out["top_logprobs"] = s["top_ids"], s["top_logprobs"]
    return out


def _library_logprob_grad(s):
    c = s["case"]
    aq, st = _stage(c["dtype"])
    aq.aq_token_logprobs_grad(st, s["logits"], c["rows"], c["vocab"], s["ld"], s["targets"], c["scale"], s["lse"], s["entropy"],
                              s["d_logprob"], s["d_entropy"], s["d_logits"], s["ld"])
    return s["d_logits"][:, :c["vocab"]]


def _library_ffn(s):
    c = s["case"]
    aq, st = _stage(c["dtype"])
    d, f = c["hidden"], c["inner"]
    aq.aq_gated_ffn(st, s["x"], d, s["wg"], s["wu"], d, c["rows"], d, f, _act_key(aq, c["act"]), s["h"], f, s["g"], s["u"], f)
    return dict(h=s["h"], g=s["g"], u=s["u"]) if c["save"] else s["h"]


def _library_ffn_grad(s):
    c = s["case"]
    aq, st = _stage(c["dtype"])
    d, f = c["hidden"], c["inner"]
    aq.aq_gated_ffn_grad(st, s["dh"], f, s["x"], d, s["wg"], s["wu"], d, s["g"], s["u"], f, c["rows"], d, f, _act_key(aq, c["act"]),
                         s["dx"], d, s["dwg"], s["dwu"], d)
    return dict(dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"])


def _qk_shape(aq, s):
    if "shape" not in s:
        c = s["case"]
        s["shape"] = aq.QkShape(heads_q=c["heads_q"], heads_k=c["heads_k"], head_dim=c["head_dim"], rot_dim=c["rot"],
                                interleaved=int(c["interleaved"]), eps=EPS, n_positions=s["cos_sin"].shape[0])
    return s["shape"]


def _library_qk(s):
    c = s["case"]
    aq, st = _stage(c["dtype"])
    wide = s["q"].stride(0)
    aq.aq_qk_norm_rope(st, _qk_shape(aq, s), c["rows"], s["q"], wide, s["k"], wide, s["wq"], s["wk"], s["cos_sin"], s["positions"],
                       s["q_out"], c["heads_q"] * c["head_dim"], s["k_out"], c["heads_k"] * c["head_dim"])
    return dict(q=s["q_out"], k=s["k_out"])


def _library_qk_grad(s):
    c = s["case"]
    aq, st = _stage(c["dtype"])
    wide, nq, nk = s["q"].stride(0), c["heads_q"] * c["head_dim"], c["heads_k"] * c["head_dim"]
    dq, dk = s["dqkv"][:, :nq], s["dqkv"][:, nq:nq + nk]
    aq.aq_qk_norm_rope_grad(st, _qk_shape(aq, s), c["rows"], s["dq_out"], nq, s["dk_out"], nk, s["q"], wide, s["k"], wide,
                            s["wq"], s["wk"], s["cos_sin"], s["positions"], dq, wide, dk, wide, s["dwq"], s["dwk"])
    return dict(dq=dq, dk=dk, dwq=s["dwq"], dwk=s["dwk"])


_library = {"logprob": _library_logprob, "logprob_grad": _library_logprob_grad, "ffn": _library_ffn, "ffn_grad": _library_ffn_grad,
            "qk": _library_qk, "qk_grad": _library_qk_grad}


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    c = case
    size = SIZE[c["dtype"]]
    if c["op"] in ("logprob", "logprob_grad"):
        n = c["rows"] * c["vocab"]
        if c["op"] == "logprob":
            return {"bytes": n * size + c["rows"] * (4 + 12 + 8 * min(c["top_k"], c["vocab"])), "flops": 5 * n}
        return {"bytes": 2 * n * size + c["rows"] * 20, "flops": 6 * n}
    if c["op"] in ("ffn", "ffn_grad"):
        m, d, f = c["rows"], c["hidden"], c["inner"]
        if c["op"] == "ffn":
            return {"bytes": size * (m * d + 2 * f * d + m * f * (3 if c["save"] else 1)), "flops": 4 * m * d * f + 8 * m * f}
        return {"bytes": size * (2 * m * d + 4 * f * d + 3 * m * f), "flops": 8 * m * d * f + 16 * m * f}
    n = c["rows"] * (c["heads_q"] + c["heads_k"]) * c["head_dim"]
    table = min(c["rows"], 2048) * c["rot"] * 4 + c["rows"] * 4
    if c["op"] == "qk":
        return {"bytes": 2 * n * size + table + 2 * c["head_dim"] * size, "flops": 8 * n}
    return {"bytes": 3 * n * size + table + 2 * c["head_dim"] * (size + 4), "flops": 16 * n}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    """What run() returns, from the definitions in binary64: rows and heads by matrix forms of their own."""
    s = prepare(case, seed)
    c, f64 = case, torch.float64
    if c["op"] in ("logprob", "logprob_grad"):
        z = s["logits"].to(f64) * c["scale"]
        lp = torch.log_softmax(z, 1)                  # NaN where a row has nothing: put right below
        none = (s["logits"] == -math.inf).all(1)
        lse = torch.logsumexp(z, 1)
        del z
        targets = s["targets"].long()
        if c["op"] == "logprob":
            p = lp.exp()
            entropy = torch.where(none, 0.0, -torch.special.xlogy(p, p).sum(1))
            del p
            at = lp.gather(1, targets.clamp(min=0)[:, None])[:, 0].masked_fill(none, -math.inf).masked_fill(targets < 0, 0.0)
            out = dict(lse=lse, entropy=entropy, logprob=at)
            if s["k"]:
                out["top_ids"] = None
                out["top_logprobs"] = lp.masked_fill(none[:, None], -math.inf).topk(s["k"], 1).values
            return out
        # through the Jacobian of the row's own statistics, as the forward call computes them
        lp[none] = -math.inf
        p = lp.exp()
        gl = s["d_logprob"].to(f64) * (targets >= 0)
        entropy = -torch.special.xlogy(p, p).sum(1, keepdim=True)
        lp = lp.masked_fill(p == 0, 0.0)
        d = -gl[:, None] * p
        d -= s["d_entropy"].to(f64)[:, None] * p * (lp + entropy)
        d.scatter_add_(1, targets.clamp(min=0)[:, None], torch.where(none, 0.0, gl)[:, None])
        return d * c["scale"]
    if c["op"] in ("ffn", "ffn_grad"):
        x, wg, wu = s["x"].to(f64), s["wg"].to(f64), s["wu"].to(f64)
        if c["op"] == "ffn":
            g, u = torch.einsum("md,fd->mf", x, wg), torch.einsum("md,fd->mf", x, wu)
        else:
            g, u = s["g"].to(f64).requires_grad_(True), s["u"].to(f64)
        if c["act"] == "silu":
            a = g / (1 + torch.exp(-g))
        elif c["act"] == "gelu":
            a = 0.5 * g * torch.erfc(-g / math.sqrt(2))
        else:
            a = 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
        if c["op"] == "ffn":
            return dict(h=a * u, g=g, u=u) if c["save"] else a * u
        dh = s["dh"].to(f64)
        dg, = torch.autograd.grad((a * (dh * u)).sum(), g)
        du = dh * a.detach()
        return dict(dx=torch.einsum("mf,fd->md", dg, wg) + torch.einsum("mf,fd->md", du, wu),
                    dwg=torch.einsum("mf,md->fd", dg, x), dwu=torch.einsum("mf,md->fd", du, x))
    # norm and rotation by complex numbers and torch's differentiation
    half = c["rot"] // 2
    cs = s["cos_sin"].to(f64)[s["positions"].long()]
    turn = torch.complex(cs[:, :half], cs[:, half:])[:, None, :]

    def forward(x, w):
        x = x.unflatten(1, (-1, c["head_dim"]))
        y = w * x / torch.sqrt(x.square().sum(-1, keepdim=True) / c["head_dim"] + EPS)
        r = y[..., :c["rot"]]
        pairs = r.unflatten(-1, (half, 2)) if c["interleaved"] else r.unflatten(-1, (2, half)).transpose(-1, -2)
        z = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn)
        r = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([r, y[..., c["rot"]:]], -1).flatten(1)

    q, k, wq, wk = (s[n].to(f64) for n in ("q", "k", "wq", "wk"))
    if c["op"] == "qk":
        return dict(q=forward(q, wq), k=forward(k, wk))
    out = {}
    for n, x, w, dy in (("q", q, wq, s["dq_out"]), ("k", k, wk, s["dk_out"])):
        x, w = x.requires_grad_(True), w.requires_grad_(True)
        out["d" + n], out["dw" + n] = torch.autograd.grad(forward(x, w), (x, w), dy.to(f64))
    return out
