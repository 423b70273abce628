"""A small language model fine-tuned in two pipeline stages on one GPU.

Each stage is a transformer layer: attention whose queries and keys go through `aq_qk_norm_rope`, and a gated feed-forward
block through `aq_gated_ffn`.  The activation crosses from the first stage to the second as 4-bit differences
(`aq_encode`, `aq_wire_copy`, `aq_decode`); the second stage ends in `aq_token_logprobs`, whose mean over the batch is the
loss; the gradient of the activation travels back in 8 bits (`aq_quant_grad`, `aq_wire_copy_grad`, `aq_dequant_grad`).
torch does the plain products, the softmax of the attention and the chain rule between the calls.  With `--norm layer` the
blocks begin with `aq_layer_norm` (which adds the residual in the same pass) instead of torch's RMS norm, and with
`--optimizer adamw` or `adamw8` a step is `aq_grad_norm` and `aq_adamw`, clipped, with moments in 32 bits or in 8.

    python examples/finetune_two_stages.py [--epochs N] [--norm rms|layer] [--optimizer torch|adamw|adamw8]

The data are sequences of a made-up language in which every token has four possible successors: the loss of a guess is
ln 96 = 4.56, that of a model that knows the language ln 4 = 1.39, and less as it comes to know the sequences themselves.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2206_01299_b200 as aq  # noqa: E402

VOCAB, SEQ, HIDDEN, HEADS, KEY_HEADS, HEAD, INNER = 96, 64, 128, 4, 2, 32, 256
SAMPLES, BATCH, EPS = 64, 16, 1e-6
T = torch.bfloat16


class GatedFfn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, stage, x, wg, wu):
        rows, d, f = x.shape[0], x.shape[1], wg.shape[0]
        h, g, u = (torch.empty((rows, f), dtype=T, device="cuda") for _ in range(3))
        aq.aq_gated_ffn(stage, x, d, wg, wu, d, rows, d, f, aq.AQ_ACT_SILU, h, f, g, u, f)
        ctx.stage = stage
        ctx.save_for_backward(x, wg, wu, g, u)
        return h

    @staticmethod
    def backward(ctx, dh):
        x, wg, wu, g, u = ctx.saved_tensors
        rows, d, f = x.shape[0], x.shape[1], wg.shape[0]
        dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
        aq.aq_gated_ffn_grad(ctx.stage, dh.contiguous(), f, x, d, wg, wu, d, g, u, f, rows, d, f, aq.AQ_ACT_SILU, dx, d, dwg, dwu, d)
        return None, dx, dwg, dwu


class QkNormRope(torch.autograd.Function):
    """Queries and keys of [rows, (heads + 2 key heads) * head] projections, normalised and rotated."""

    @staticmethod
    def forward(ctx, stage, shape, qkv, wq, wk, cos_sin, positions):
        rows, wide, nq, nk = qkv.shape[0], qkv.shape[1], HEADS * HEAD, KEY_HEADS * HEAD
        q, k = torch.empty((rows, nq), dtype=T, device="cuda"), torch.empty((rows, nk), dtype=T, device="cuda")
        aq.aq_qk_norm_rope(stage, shape, rows, qkv, wide, qkv[:, nq:], wide, wq, wk, cos_sin, positions, q, nq, k, nk)
        ctx.stage, ctx.shape = stage, shape
        ctx.save_for_backward(qkv, wq, wk, cos_sin, positions)
        return q, k

    @staticmethod
    def backward(ctx, dq, dk):
        qkv, wq, wk, cos_sin, positions = ctx.saved_tensors
        rows, wide, nq, nk = qkv.shape[0], qkv.shape[1], HEADS * HEAD, KEY_HEADS * HEAD
        dqkv = torch.zeros_like(qkv)
        dwq, dwk = (torch.empty(HEAD, dtype=torch.float32, device="cuda") for _ in range(2))
        aq.aq_qk_norm_rope_grad(ctx.stage, ctx.shape, rows, dq.contiguous(), nq, dk.contiguous(), nk, qkv, wide, qkv[:, nq:], wide, wq, wk,
                                cos_sin, positions, dqkv, wide, dqkv[:, nq:], wide, dwq, dwk)
        return None, None, dqkv, dwq.to(T), dwk.to(T), None, None


class LayerNorm(torch.autograd.Function):
    """(s, y): the sum of x and residual (x itself without one), and its norm."""

    @staticmethod
    def forward(ctx, stage, x, residual, w, b):
        rows, d = x.shape
        y, s = torch.empty_like(x), torch.empty_like(x) if residual is not None else None
        mean, rstd = (torch.empty(rows, dtype=torch.float32, device="cuda") for _ in range(2))
        aq.aq_layer_norm(stage, x, d, residual, d, w, b, EPS, rows, d, s, d, y, d, mean, rstd)
        ctx.stage, ctx.alone = stage, residual is None
        ctx.save_for_backward(x if s is None else s, w, mean, rstd)
        return (x.view_as(x) if s is None else s), y

    @staticmethod
    def backward(ctx, ds, dy):
        s, w, mean, rstd = ctx.saved_tensors
        rows, d = s.shape
        dx = torch.empty_like(s)
        dw, db = (torch.empty(d, dtype=torch.float32, device="cuda") for _ in range(2))
        aq.aq_layer_norm_grad(ctx.stage, dy.contiguous(), d, ds.contiguous(), d, s, d, w, mean, rstd, rows, d, dx, d, dw, db)
        return None, dx, None if ctx.alone else dx, dw.to(T), db.to(T)


class TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, stage, logits, targets):
        rows, vocab = logits.shape
        logprob, entropy, lse = (torch.empty(rows, dtype=torch.float32, device="cuda") for _ in range(3))
        aq.aq_token_logprobs(stage, logits, rows, vocab, vocab, targets, 1.0, 0, logprob, entropy, lse, None, None)
        ctx.stage = stage
        ctx.save_for_backward(logits, targets, lse, entropy)
        return logprob, entropy

    @staticmethod
    def backward(ctx, d_logprob, d_entropy):
        logits, targets, lse, entropy = ctx.saved_tensors
        rows, vocab = logits.shape
        d = torch.empty_like(logits)
        aq.aq_token_logprobs_grad(ctx.stage, logits, rows, vocab, vocab, targets, 1.0, lse, entropy, d_logprob.contiguous(),
                                  None if d_entropy is None else d_entropy.contiguous(), d, vocab)
        return None, d, None


class Layer:
    """One stage's transformer layer; binary32 weights, used in bf16."""

    def __init__(self, g, norm="rms"):
        wide = (HEADS + 2 * KEY_HEADS) * HEAD
        shapes = dict(qkv=(wide, HIDDEN), out=(HIDDEN, HEADS * HEAD), wg=(INNER, HIDDEN), wu=(INNER, HIDDEN), down=(HIDDEN, INNER))
        self.p = {n: (torch.randn(s, generator=g) / math.sqrt(s[1])).cuda().requires_grad_(True) for n, s in shapes.items()}
        for n in ("wq", "wk"):
            self.p[n] = torch.ones(HEAD, device="cuda").requires_grad_(True)
        self.norm = norm
        if norm == "layer":
            for n in ("n1", "n2"):
                self.p[n + "w"] = torch.ones(HIDDEN, device="cuda").requires_grad_(True)
                self.p[n + "b"] = torch.zeros(HIDDEN, device="cuda").requires_grad_(True)
        angle = torch.arange(SEQ, dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(HEAD // 2, dtype=torch.float64) * 2 / HEAD)
        self.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        self.shape = aq.QkShape(heads_q=HEADS, heads_k=KEY_HEADS, head_dim=HEAD, rot_dim=HEAD, interleaved=0, eps=EPS, n_positions=SEQ)

    def forward(self, stage, x):
        """x [batch, seq, hidden] -> the same."""
        b, p = x.shape[0], {n: w.to(T) for n, w in self.p.items()}
        rms = lambda v: (v.float() * torch.rsqrt(v.float().square().mean(-1, keepdim=True) + EPS)).to(T)  # noqa: E731
        if self.norm == "layer":
            stream, rows = LayerNorm.apply(stage, x.reshape(b * SEQ, HIDDEN), None, p["n1w"], p["n1b"])
        else:
            rows = rms(x).reshape(b * SEQ, HIDDEN)
        qkv = rows @ p["qkv"].T
        positions = torch.arange(SEQ, dtype=torch.int32, device="cuda").repeat(b)
        q, k = QkNormRope.apply(stage, self.shape, qkv, p["wq"], p["wk"], self.cos_sin, positions)
        v = qkv[:, (HEADS + KEY_HEADS) * HEAD:]
        q = q.view(b, SEQ, HEADS, HEAD).transpose(1, 2)
        k, v = (t.reshape(b, SEQ, KEY_HEADS, HEAD).transpose(1, 2).repeat_interleave(HEADS // KEY_HEADS, 1) for t in (k, v))
        score = (q @ k.transpose(-1, -2)).float() / math.sqrt(HEAD)
        score = score.masked_fill(torch.ones(SEQ, SEQ, device="cuda").triu(1).bool(), -math.inf)
        mixed = (score.softmax(-1).to(T) @ v).transpose(1, 2).reshape(b, SEQ, HEADS * HEAD)
        if self.norm == "layer":
            stream, rows = LayerNorm.apply(stage, (mixed @ p["out"].T).reshape(b * SEQ, HIDDEN), stream, p["n2w"], p["n2b"])
            h = GatedFfn.apply(stage, rows, p["wg"], p["wu"])
            return (stream + h @ p["down"].T).view(b, SEQ, HIDDEN)
        x = x + mixed @ p["out"].T
        h = GatedFfn.apply(stage, rms(x).reshape(b * SEQ, HIDDEN), p["wg"], p["wu"])
        return x + (h @ p["down"].T).view(b, SEQ, HIDDEN)


class AdamW:
    """The optimizer's step over all binary32 weights: their gradients' norm, its clipping factor and the update in two launches."""

    def __init__(self, params, lr, state_bits):
        self.stage = aq.aq_stage_create()
        aq.aq_stage_configure(self.stage, aq.AQ_DTYPE, aq.AQ_FP32)
        self.params = params
        for p in params:
            p.grad = torch.zeros_like(p)                         # stays where it is: backward passes add to it
        zeros = lambda t, n=None: [torch.zeros(n(p) if n else p.numel(), dtype=t, device="cuda") for p in params]  # noqa: E731
        if state_bits == 8:
            blocks = lambda p: -(-p.numel() // 256)  # noqa: E731
            self.state = dict(m=zeros(torch.float8_e4m3fn), v=zeros(torch.float8_e5m2), m_scale=zeros(torch.float32, blocks), v_scale=zeros(torch.float32, blocks))
        else:
            self.state = dict(m=zeros(torch.float32), v=zeros(torch.float32))
        self.table = aq.aq_adam_table(self.stage, params=[p.detach() for p in params], grads=[p.grad for p in params],
                                      weight_decay=[0.01 if p.dim() > 1 else 0.0 for p in params], **self.state)
        self.config = aq.AdamwConfig(lr=lr, beta1=0.9, beta2=0.999, eps=1e-8, state_bits=state_bits)
        self.norm, self.factor = (torch.empty(1, device="cuda") for _ in range(2))
        self.count = torch.zeros(1, dtype=torch.int64, device="cuda")

    def zero_grad(self):
        for p in self.params:
            p.grad.zero_()

    def step(self):
        aq.aq_grad_norm(self.stage, self.table, len(self.params), 1.0, 1.0, self.norm, self.factor, self.count)
        aq.aq_adamw(self.stage, self.config, self.table, len(self.params), self.factor, None, self.count)

    def close(self):
        assert aq.aq_stage_status(self.stage) == 0
        aq.aq_stage_destroy(self.stage)


class Boundary:
    """Sender and receiver of the activation between the two stages."""

    def __init__(self):
        self.snd, self.rcv = (aq.aq_create(SAMPLES, SEQ, HIDDEN, 4, 32) for _ in range(2))
        for h in (self.snd, self.rcv):
            aq.aq_configure(h, aq.AQ_DTYPE, aq.AQ_BF16)
            aq.aq_configure(h, aq.AQ_BATCH, BATCH)
        make = lambda n: [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(2)]  # noqa: E731
        steps = lambda n: [torch.empty(n, dtype=torch.float32, device="cuda") for _ in range(2)]  # noqa: E731
        self.codes, self.scales = make(BATCH * aq.aq_packed_bytes_per_sample(self.snd)), steps(BATCH * aq.aq_scales_per_sample(self.snd))
        self.n = BATCH * SEQ * HIDDEN
        self.g_codes, self.g_scales = make(self.n), steps(self.n // 32)

    def forward(self, act, ids, first):
        """What the second stage receives; `first`: the samples' first visit, whose message is the activation itself."""
        out, raw = torch.empty_like(act), torch.empty_like(act) if first else None
        aq.aq_encode(self.snd, act, ids, self.codes[0], self.scales[0])
        aq.aq_wire_copy(self.snd, 0, self.codes[1], self.scales[1], raw, self.codes[0], self.scales[0], act if first else None)
        aq.aq_configure(self.rcv, aq.AQ_RAW, raw)
        aq.aq_decode(self.rcv, self.codes[1], self.scales[1], ids, out)
        return out

    def backward(self, grad):
        out = torch.empty_like(grad)
        aq.aq_quant_grad(self.rcv, grad, self.n, 8, self.g_codes[0], self.g_scales[0])
        aq.aq_wire_copy_grad(self.rcv, 0, self.g_codes[1], self.g_scales[1], self.g_codes[0], self.g_scales[0], self.n, 8)
        aq.aq_dequant_grad(self.snd, self.g_codes[1], self.g_scales[1], self.n, 8, out)
        return out

    def close(self):
        assert aq.aq_status(self.snd) == 0 and aq.aq_status(self.rcv) == 0
        assert aq.aq_state_checksum(self.snd) == aq.aq_state_checksum(self.rcv)
        aq.aq_destroy(self.snd)
        aq.aq_destroy(self.rcv)


def language(seed=0):
    """[SAMPLES, SEQ + 1] tokens: each followed by one of four successors of its own."""
    g = torch.Generator().manual_seed(seed)
    successors = torch.randint(0, VOCAB, (VOCAB, 4), generator=g)
    tokens = torch.randint(0, VOCAB, (SAMPLES, SEQ + 1), generator=g)
    for t in range(SEQ):
        tokens[:, t + 1] = successors[tokens[:, t], torch.randint(0, 4, (SAMPLES,), generator=g)]
    return tokens.cuda()


def train(epochs=20, lr=0.005, say=print, norm="rms", optimizer="torch"):
    """Losses of every step."""
    g = torch.Generator().manual_seed(1)
    tokens, layers, boundary = language(), [Layer(g, norm), Layer(g, norm)], Boundary()
    embed, head = (0.3 * torch.randn(VOCAB, HIDDEN, generator=g)).cuda().requires_grad_(True), (torch.randn(VOCAB, HIDDEN, generator=g) / 12).cuda().requires_grad_(True)
    params = [embed, head] + [w for layer in layers for w in layer.p.values()]
    adam = torch.optim.Adam(params, lr=lr) if optimizer == "torch" else AdamW(params, lr, 8 if optimizer == "adamw8" else 32)
    stage = aq.aq_stage_create()
    aq.aq_stage_configure(stage, aq.AQ_DTYPE, aq.AQ_BF16)
    losses = []
    for epoch in range(epochs):
        for ids in torch.randperm(SAMPLES, generator=g).split(BATCH):
            batch = tokens[ids.cuda()]
            act = layers[0].forward(stage, embed.to(T)[batch[:, :-1]])                       # first stage
            received = boundary.forward(act.detach(), ids.int().cuda(), epoch == 0).requires_grad_(True)
            x = layers[1].forward(stage, received)                                           # second stage
            logits = x.reshape(-1, HIDDEN) @ head.to(T).T
            logprob, entropy = TokenLogprobs.apply(stage, logits, batch[:, 1:].reshape(-1).int().contiguous())
            loss = -logprob.mean()
            adam.zero_grad()
            loss.backward()                                                                  # second stage's share
            act.backward(boundary.backward(received.grad))                                   # first stage's
            adam.step()
            losses.append(loss.item())
        say(f"epoch {epoch}: loss {losses[-1]:.3f}, entropy {entropy.mean().item():.3f}")
    assert aq.aq_stage_status(stage) == 0
    aq.aq_stage_destroy(stage)
    if optimizer != "torch":
        adam.close()
    boundary.close()
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--epochs", type=int, default=20)
    ap.add_argument("--norm", choices=["rms", "layer"], default="rms")
    ap.add_argument("--optimizer", choices=["torch", "adamw", "adamw8"], default="torch")
    args = ap.parse_args()
    train(args.epochs, norm=args.norm, optimizer=args.optimizer)
