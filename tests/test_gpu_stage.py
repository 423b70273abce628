"""Stage operators on the GPU against plain 64-bit forms (stage_forms.py).

Tolerances.  u is one rounding to the output type, e = 2^-24 one binary32 rounding.
* A 16-bit output computed in binary32: u |y| plus what the binary32 sum carries.
* A sum of K products: each partial sum is rounded (or cut, on the tensor cores) to binary32, so at most K steps of 2e of
  the sum of magnitudes; the steps fall in both directions, and sqrt(K) of them, times four, is used.
* ln S, entropy: a thread adds up to V/256 + 12 terms, each off by up to 4e (2^x) plus e times the exponent's size:
  (V/256 + 12 + 4 + |exponent|) e relative to S; 2e-5 covers V = 50257.  scale (x - x_max) adds 2e of its size.
"""
import math

import pytest
import torch

from tests import stage_forms as forms

pytestmark = pytest.mark.gpu
F64 = torch.float64
E = 2.0 ** -24


@pytest.fixture(scope="module")
def aq():
    import paper_2206_01299_b200 as aq
    aq.lib()
    return aq


@pytest.fixture
def stage(aq):
    st = aq.aq_stage_create()
    yield st
    aq.aq_stage_destroy(st)


def set_type(aq, st, dtype):
    aq.aq_stage_configure(st, aq.AQ_DTYPE, {"fp16": aq.AQ_FP16, "bf16": aq.AQ_BF16, "fp32": aq.AQ_FP32}[dtype])


class Guarded:
    """A [rows, cols] buffer with a row stride, inside a larger one whose other elements must not change."""

    def __init__(self, rows, cols, dtype, pad=0, offset=0, fill=-7.0):
        self.ld = cols + pad
        self.offset = 64 + offset
        self.flat = torch.full((self.offset + rows * self.ld + 64,), fill, dtype=dtype, device="cuda")
        self.view = self.flat[self.offset:self.offset + rows * self.ld].view(rows, self.ld)[:, :cols] if rows * cols else self.flat[:0].view(rows, cols)
        self.fill = fill

    def put(self, x):
        self.view.copy_(x)
        return self

    def check(self):
        outside = self.flat.clone()
        rows, cols = self.view.shape
        if rows * cols:
            outside[self.offset:self.offset + rows * self.ld].view(rows, self.ld)[:, :cols] = self.fill
        assert bool((outside == self.fill).all()), "a write outside the buffer"


def floats(n, k=None):
    return torch.full((n,) if k is None else (n, k), 77.0, device="cuda")


# ---- token log probabilities ---------------------------------------------------------------------------------

def run_logprobs(aq, st, buf, targets, scale, k):
    rows, vocab = buf.view.shape
    lp, h, lse = floats(rows), floats(rows), floats(rows)
    ids, top = torch.full((rows, k), -9, dtype=torch.int32, device="cuda"), floats(rows, k)
    aq.aq_token_logprobs(st, buf.view, rows, vocab, buf.ld, targets.cuda(), scale, k, lp, h, lse, ids, top)
    torch.cuda.synchronize()
    return lp.cpu().double(), h.cpu().double(), lse.cpu().double(), ids.cpu().long(), top.cpu().double()


def check_logprobs(x, targets, scale, k, got):
    """x: the stored logits as binary64, on the CPU."""
    s32 = torch.tensor(scale, dtype=torch.float32).double().item()
    for r in range(x.shape[0]):
        lp, h, lse, ids, top = forms.logprobs(x[r], int(targets[r]), s32, k)
        tol = 2e-5
        spread = lambda v: 4 * E * abs(v) if math.isfinite(v) else 0.0  # noqa: E731
        for want, have in ((lp, got[0][r].item()), (lse, got[2][r].item())):
            assert want == have or abs(want - have) <= tol + spread(want), (r, want, have)
        assert abs(h - got[1][r].item()) <= 2 * tol + spread(h), (r, h, got[1][r].item())
        assert got[3][r].tolist() == ids.tolist(), r
        for want, have in zip(top.tolist(), got[4][r].tolist()):
            assert want == have or abs(want - have) <= tol + spread(want), (r, want, have)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab,pad,offset", [
    (1, 1, 0, 0), (3, 2, 1, 1), (2, 7, 0, 3), (5, 8, 0, 0), (4, 50, 3, 0), (3, 257, 0, 1), (90, 1000, 5, 2), (2, 4096, 0, 0),
    (1, 4097, 0, 5), (3, 8191, 2, 7), (75, 4099, 0, 0), (1, 50257, 0, 0), (7, 50257, 0, 1), (80, 20000, 1, 3)])
def test_logprobs(aq, stage, dtype, rows, vocab, pad, offset):
    set_type(aq, stage, dtype)
    g = torch.Generator().manual_seed(rows * 100003 + vocab)
    x = 3 * torch.randn((rows, vocab), generator=g)
    x[torch.rand((rows, vocab), generator=g) < 0.1] = -math.inf
    x[:, vocab // 2] = 1.5
    x = x.to(forms.TYPES[dtype])
    targets = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    targets[rows // 2] = vocab // 2
    if rows > 2:
        targets[0] = -5
    k = min(vocab, 1 + (rows * 7 + vocab) % 32)
    buf = Guarded(rows, vocab, forms.TYPES[dtype], pad, offset).put(x)
    got = run_logprobs(aq, stage, buf, targets, 0.8, k)
    buf.check()
    check_logprobs(x.double(), targets, 0.8, k, got)
    assert aq.aq_stage_status(stage) == 0


@pytest.mark.parametrize("rows", [2, 100])
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_logprobs_ties_go_to_the_lowest_id(aq, stage, dtype, rows):
    """Few distinct values, so that every place of the alternatives is tied; whole rows of one value; zeros of both signs."""
    set_type(aq, stage, dtype)
    vocab = 9001
    g = torch.Generator().manual_seed(5)
    x = torch.randint(-3, 4, (rows, vocab), generator=g).float()
    x[0] = 2.0
    x[1] = torch.where(torch.arange(vocab) % 3 == 0, -0.0, 0.0)
    x = x.to(forms.TYPES[dtype])
    targets = torch.zeros(rows, dtype=torch.int32)
    buf = Guarded(rows, vocab, forms.TYPES[dtype], 0, 1).put(x)
    check_logprobs(x.double(), targets, 1.0, 32, run_logprobs(aq, stage, buf, targets, 1.0, 32))


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab,k,pad", [(3, 512, 32, 0), (9, 513, 9, 1), (9, 1024, 8, 3), (2, 1024, 32, 0), (5, 1025, 32, 0), (90, 2049, 20, 1), (17, 40, 32, 5)])
def test_logprobs_where_the_way_of_working_changes(aq, stage, dtype, rows, vocab, k, pad):
    """Row lengths and numbers of alternatives on both sides of every choice; half of the logits masked."""
    set_type(aq, stage, dtype)
    g = torch.Generator().manual_seed(vocab + k)
    x = 3 * torch.randn((rows, vocab), generator=g)
    x[torch.rand((rows, vocab), generator=g) < 0.5] = -math.inf
    x = x.to(forms.TYPES[dtype])
    targets = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    buf = Guarded(rows, vocab, forms.TYPES[dtype], pad, 1).put(x)
    check_logprobs(x.double(), targets, 1.0, k, run_logprobs(aq, stage, buf, targets, 1.0, k))
    buf.check()


@pytest.mark.parametrize("rows,vocab", [(2, 700), (2, 6001), (120, 6001)])
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_logprobs_fewer_tokens_left_than_alternatives(aq, stage, dtype, rows, vocab):
    """Three tokens of a row are allowed, twenty alternatives asked for: then come the lowest ids that are masked."""
    set_type(aq, stage, dtype)
    x = torch.full((rows, vocab), -math.inf)
    allowed = torch.tensor([5, vocab // 2, vocab - 1])
    x[:, allowed] = torch.tensor([0.5, -1.0, 2.0])
    x[1, allowed] = torch.tensor([1.0, 1.0, 1.0])
    x = x.to(forms.TYPES[dtype])
    targets = torch.full((rows,), vocab - 1, dtype=torch.int32)
    buf = Guarded(rows, vocab, forms.TYPES[dtype], 1, 0).put(x)
    check_logprobs(x.double(), targets, 1.0, 20, run_logprobs(aq, stage, buf, targets, 1.0, 20))


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_logprobs_of_barely_scaled_logits(aq, stage, dtype):
    """A scale at which the type's lowest value and -infinity are not the same thing any more."""
    set_type(aq, stage, dtype)
    vocab, scale = 5000, 1e-4
    x = 100 * torch.randn((90, vocab), generator=torch.Generator().manual_seed(9))
    x[:, ::3] = -math.inf
    x[:, 1::3] = torch.finfo(forms.TYPES[dtype]).min if dtype == "fp16" else -60000.0
    x = x.to(forms.TYPES[dtype])
    targets = torch.full((90,), 4, dtype=torch.int32)
    buf = Guarded(90, vocab, forms.TYPES[dtype]).put(x)
    got = run_logprobs(aq, stage, buf, targets, scale, 3)
    check_logprobs(x.double(), targets, scale, 3, got)
    out = Guarded(90, vocab, forms.TYPES[dtype])
    gl = torch.full((90,), 512.0)
    run_logprobs_grad(aq, stage, buf, out, targets.cuda(), scale, got[2].float().cuda(), None, gl.cuda(), None)
    s32 = torch.tensor(scale, dtype=torch.float32).double().item()
    for r in (0, 89):
        want = forms.logprobs_grad(x[r].double(), 4, s32, 512.0, 0.0)
        within(out.view[r], want, forms.UNIT[dtype] * want.abs() * 1.1 + forms.TINY[dtype] + 1e-4 * want.abs())


@pytest.mark.parametrize("rows", [3, 200])
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
def test_logprobs_masked_rows(aq, stage, dtype, rows):
    """Nothing left; one token left; nothing but the type's lowest value; the lowest value beside real logits; very large logits."""
    set_type(aq, stage, dtype)
    vocab = 6001
    low = torch.finfo(forms.TYPES[dtype]).min
    big = 60000.0 if dtype == "fp16" else 1e30
    g = torch.Generator().manual_seed(6)
    x = torch.randn((rows, vocab), generator=g)
    targets = torch.full((rows,), 4321, dtype=torch.int32)
    for r in range(0, rows - 2, 50):
        x[r] = -math.inf
        x[r + 1] = -math.inf
        x[r + 1, 4321] = -2.0
        x[r + 2] = low
    if rows > 10:
        x[5] = torch.where(torch.rand(vocab, generator=g) < 0.5, low, x[5])
        x[6] = x[6] * 0.5 + big
        x[7] = -big
        x[8, 17] = big
    x = x.to(forms.TYPES[dtype])
    buf = Guarded(rows, vocab, forms.TYPES[dtype]).put(x)
    check_logprobs(x.double(), targets, 1.0, 5, run_logprobs(aq, stage, buf, targets, 1.0, 5))


@pytest.mark.parametrize("rows", [2, 100])
def test_logprobs_nan_and_infinity(aq, stage, rows):
    set_type(aq, stage, "fp32")
    vocab = 5000
    x = torch.randn((rows, vocab), generator=torch.Generator().manual_seed(7))
    x[0, 4000] = math.nan
    x[1] = math.nan
    x[1, 3] = 1.0
    targets = torch.full((rows,), 10, dtype=torch.int32)
    lp, h, lse, ids, top = run_logprobs(aq, stage, Guarded(rows, vocab, torch.float32).put(x), targets, 1.0, 4)
    for v in (lp, h, lse):
        assert torch.isnan(v[:2]).all() and torch.isfinite(v[2:]).all()
    assert 4000 not in ids[0].tolist() and ids[0].tolist() == torch.topk(torch.nan_to_num(x[0], nan=-1e9), 4).indices.tolist()
    assert ids[1].tolist() == [3, -1, -1, -1] and torch.isnan(top[1, 1:]).all()
    x[0, 4000] = math.inf
    lp, h, lse, ids, top = run_logprobs(aq, stage, Guarded(rows, vocab, torch.float32).put(x), targets, 1.0, 4)
    assert torch.isnan(lse[0]) and torch.isnan(h[0]) and torch.isnan(lp[0]) and ids[0, 0].item() == 4000


def test_logprobs_bad_target_sets_the_status(aq, stage):
    set_type(aq, stage, "fp16")
    x = torch.randn((3, 100)).half()
    targets = torch.tensor([5, 100, -1], dtype=torch.int32)
    got = run_logprobs(aq, stage, Guarded(3, 100, torch.float16).put(x), targets, 1.0, 0)
    check_logprobs(x.double(), targets, 1.0, 0, got)
    assert aq.aq_stage_status(stage) == aq.AQ_ST_BAD_ID and aq.aq_stage_status(stage) == 0


def test_logprobs_null_outputs_and_no_rows(aq, stage):
    set_type(aq, stage, "bf16")
    x = torch.randn((2, 300)).bfloat16().cuda()
    aq.aq_token_logprobs(stage, x, 2, 300, 300, None, 1.0, 3, None, None, None, None, None)
    lse = floats(2)
    aq.aq_token_logprobs(stage, x, 2, 300, 300, None, 1.0, 0, None, None, lse, None, None)
    aq.aq_token_logprobs(stage, None, 0, 300, 300, None, 1.0, 0, None, None, None, None, None)
    assert (lse.cpu().double() - torch.logsumexp(x.cpu().double(), 1)).abs().max() < 2e-5


def run_logprobs_grad(aq, st, buf, out, targets, scale, lse, h, gl, gh):
    rows, vocab = buf.view.shape
    aq.aq_token_logprobs_grad(st, buf.view, rows, vocab, buf.ld, targets, scale, lse, h, gl, gh, out.view, out.ld)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab,pad,offset,pad_d,offset_d", [
    (1, 1, 0, 0, 0, 0), (3, 2, 1, 1, 1, 1), (2, 7, 0, 3, 2, 1), (4, 50, 3, 0, 3, 8), (3, 257, 0, 1, 0, 1), (20, 1000, 0, 2, 4, 0),
    (2, 8192, 0, 0, 0, 0), (2, 8193, 7, 0, 7, 0), (3, 50257, 0, 1, 0, 1), (2, 20000, 1, 0, 0, 0), (9, 1024, 0, 0, 0, 0), (5, 1025, 0, 1, 0, 1),
    (9, 2048, 3, 5, 3, 13), (5, 2049, 0, 0, 0, 0)])
def test_logprobs_gradient(aq, stage, dtype, rows, vocab, pad, offset, pad_d, offset_d):
    """d within one rounding of the type of the formula's, plus binary32's: ln p is known to (|z| + |lse|) 2e, and so
    is p to that times its size; the terms' sum adds 4e of their magnitudes."""
    set_type(aq, stage, dtype)
    t = forms.TYPES[dtype]
    g = torch.Generator().manual_seed(vocab)
    x = 3 * torch.randn((rows, vocab), generator=g)
    x[torch.rand((rows, vocab), generator=g) < 0.1] = -math.inf
    x[:, vocab // 2] = 1.5
    if rows > 3:
        x[3] = -math.inf
    if rows > 2:
        x[2] = torch.finfo(t).min
    x = x.to(t)
    targets = torch.full((rows,), vocab // 2, dtype=torch.int32)
    if rows > 1:
        targets[1] = -1
    gl, gh = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    buf = Guarded(rows, vocab, t, pad, offset).put(x)
    lse, h = floats(rows), floats(rows)
    aq.aq_token_logprobs(stage, buf.view, rows, vocab, buf.ld, None, 0.8, 0, None, h, lse, None, None)
    s32 = torch.tensor(0.8, dtype=torch.float32).double().item()
    for use_l, use_h in ((True, True), (True, False), (False, True)):
        out = Guarded(rows, vocab, t, pad_d, offset_d)
        run_logprobs_grad(aq, stage, buf, out, targets.cuda(), 0.8, lse, h if use_h else None, gl.cuda() if use_l else None, gh.cuda() if use_h else None)
        out.check()
        buf.check()
        for r in range(rows):
            l, e = (gl[r].item() if use_l else 0.0), (gh[r].item() if use_h else 0.0)
            want = forms.logprobs_grad(x[r].double(), int(targets[r]), s32, l, e)
            z = x[r].double() * s32
            if z.max() == -math.inf:
                assert bool((out.view[r] == 0).all())
                continue
            lp = torch.log_softmax(z, 0)
            p = lp.exp()
            lp = torch.where(p > 0, lp, torch.zeros_like(lp))
            hh = -(p * lp).sum()
            size = s32 * p * (abs(l) + abs(e) * (lp.abs() + hh.abs()))
            size[int(targets[r])] += s32 * abs(l)
            near = torch.where(p > 0, z.abs().clamp(max=200.0), torch.zeros_like(z))
            tol = forms.UNIT[dtype] * want.abs() + forms.TINY[dtype] + size * E * (8 + 2 * near + 2 * abs(lse[r].item() if abs(lse[r].item()) < 1e30 else 0)) \
                + 2e-5 * s32 * abs(e) * p + 2e-5 * size
            off = (out.view[r].cpu().double() - want).abs()
            assert bool((off <= tol).all()), (r, (off / tol).max())


def test_logprobs_gradient_in_place(aq, stage):
    set_type(aq, stage, "bf16")
    x = torch.randn((5, 3001)).bfloat16().cuda()
    x[2] = torch.finfo(torch.bfloat16).min
    lse, h, gl = floats(5), floats(5), torch.randn(5, device="cuda")
    targets = torch.tensor([1, 2, 3, 4, 5], dtype=torch.int32, device="cuda")
    aq.aq_token_logprobs(stage, x, 5, 3001, 3001, None, 1.0, 0, None, h, lse, None, None)
    out = torch.empty_like(x)
    aq.aq_token_logprobs_grad(stage, x, 5, 3001, 3001, targets, 1.0, lse, h, gl, gl, out, 3001)
    aq.aq_token_logprobs_grad(stage, x, 5, 3001, 3001, targets, 1.0, lse, h, gl, gl, x, 3001)
    torch.cuda.synchronize()
    assert torch.equal(x, out)


def test_logprobs_gradient_against_differences(aq, stage):
    """Central differences of the library's own forward call along random directions.  The forward's error is up to 2e-5 per
    value, over 2h = 0.02 that is 2e-3; the third derivative's term is h^2 of the direction's size: 1e-4."""
    set_type(aq, stage, "fp32")
    rows, vocab, hstep = 4, 700, 1e-2
    g = torch.Generator().manual_seed(3)
    x = 2 * torch.randn((rows, vocab), generator=g)
    v = torch.randn((rows, vocab), generator=g)
    targets = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    gl, gh = torch.randn(rows, generator=g), torch.randn(rows, generator=g)
    value = []
    for sign in (1, -1):
        lp, h, *_ = run_logprobs(aq, stage, Guarded(rows, vocab, torch.float32).put(x + sign * hstep * v), targets, 1.0, 0)
        value.append(gl.double() * lp + gh.double() * h)
    lse, h = floats(rows), floats(rows)
    buf = Guarded(rows, vocab, torch.float32).put(x)
    aq.aq_token_logprobs(stage, buf.view, rows, vocab, buf.ld, None, 1.0, 0, None, h, lse, None, None)
    out = Guarded(rows, vocab, torch.float32)
    run_logprobs_grad(aq, stage, buf, out, targets.cuda(), 1.0, lse, h, gl.cuda(), gh.cuda())
    along = (out.view.cpu().double() * v.double()).sum(1)
    assert ((value[0] - value[1]) / (2 * hstep) - along).abs().max() < 1e-2


# ---- gated feed-forward ----------------------------------------------------------------------------------------

ACTS = ["silu", "gelu", "gelu_tanh"]


def act_key(aq, name):
    return {"silu": aq.AQ_ACT_SILU, "gelu": aq.AQ_ACT_GELU, "gelu_tanh": aq.AQ_ACT_GELU_TANH}[name]


def within(got, want, tol):
    off = (got.cpu().double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


FFN_SHAPES = [(1, 8, 8, 0), (1, 1600, 640, 0), (2, 72, 40, 8), (5, 64, 136, 8), (16, 200, 264, 0), (17, 768, 72, 8), (33, 136, 1000, 0), (127, 64, 128, 0),
              (128, 128, 256, 8), (129, 72, 264, 0), (255, 520, 392, 8), (257, 320, 128, 0), (300, 8, 520, 0), (640, 256, 1288, 16)]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rows,hidden,inner,pad", FFN_SHAPES)
def test_gated_ffn(aq, stage, dtype, rows, hidden, inner, pad):
    set_type(aq, stage, dtype)
    t, u = forms.TYPES[dtype], forms.UNIT[dtype]
    name = ACTS[(rows + hidden // 8) % 3]
    g = torch.Generator().manual_seed(rows + hidden + inner)
    x = Guarded(rows, hidden, t, pad).put(torch.randn((rows, hidden), generator=g))
    wg, wu = (Guarded(inner, hidden, t, pad).put(torch.randn((inner, hidden), generator=g) / math.sqrt(hidden)) for _ in range(2))
    x64, g64, u64 = x.view.cpu().double(), wg.view.cpu().double(), wu.view.cpu().double()
    h_want, g_want, u_want = forms.ffn(x64, g64, u64, name)
    e = 4 * math.sqrt(hidden) * 2 * E                                  # of the sums' magnitudes
    mg, mu = x64.abs() @ g64.abs().T, x64.abs() @ u64.abs().T
    for save in (True, False):
        h, gg, uu = Guarded(rows, inner, t, pad), Guarded(rows, inner, t, pad + 8), Guarded(rows, inner, t, pad + 8)
        aq.aq_gated_ffn(stage, x.view, x.ld, wg.view, wu.view, wg.ld, rows, hidden, inner, act_key(aq, name), h.view, h.ld,
                        gg.view if save else None, uu.view if save else None, gg.ld)
        torch.cuda.synchronize()
        for b in (h, gg, uu, x, wg, wu):
            b.check()
        # |act'| <= 1.13; the activation itself is good to 16 roundings of the larger of |g| and |act|
        h_tol = u * h_want.abs() + forms.TINY[dtype] + 1.13 * e * (mg * u_want.abs() + mu * g_want.abs()) + 16 * E * (g_want * u_want).abs()
        within(h.view, h_want, h_tol)
        if save:
            within(gg.view, g_want, u * g_want.abs() + e * mg + forms.TINY[dtype])
            within(uu.view, u_want, u * u_want.abs() + e * mu + forms.TINY[dtype])
        else:
            assert bool((gg.view == -7).all() and (uu.view == -7).all())


@pytest.mark.parametrize("name", ACTS)
def test_gated_ffn_activation_over_its_range(aq, stage, name):
    """Weights that pass x through: g and u are single values, from far below to far above zero."""
    set_type(aq, stage, "bf16")
    n = 512
    v = torch.cat([torch.linspace(-30, 30, n - 8), torch.tensor([0.0, -0.0, 300.0, -300.0, 1e4, -1e4, 1e-3, -1e-3])]).bfloat16()
    x = torch.zeros((n, 16), dtype=torch.bfloat16)
    x[:, 0], x[:, 8] = v, 1.0
    wg, wu = torch.zeros((8, 16), dtype=torch.bfloat16), torch.zeros((8, 16), dtype=torch.bfloat16)
    wg[:, 0], wu[:, 8] = 1.0, 1.0
    h = torch.empty((n, 8), dtype=torch.bfloat16, device="cuda")
    aq.aq_gated_ffn(stage, x.cuda(), 16, wg.cuda(), wu.cuda(), 16, n, 16, 8, act_key(aq, name), h, 8, None, None, 8)
    want = forms.act(name, v.double())[:, None].expand(n, 8)
    within(h, want, forms.UNIT["bf16"] * want.abs() + 16 * E * v.double().abs()[:, None] + 1e-30)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rows,hidden,inner,pad", FFN_SHAPES)
def test_gated_ffn_gradient(aq, stage, dtype, rows, hidden, inner, pad):
    """dg and du carry one rounding of the type each into the products, the products one more."""
    set_type(aq, stage, dtype)
    t, u = forms.TYPES[dtype], forms.UNIT[dtype]
    name = ACTS[(rows + hidden // 8 + 1) % 3]
    gen = torch.Generator().manual_seed(rows + hidden + inner)
    put = lambda r, c, p, s=1.0: Guarded(r, c, t, p).put(s * torch.randn((r, c), generator=gen))  # noqa: E731
    x, dh = put(rows, hidden, pad), put(rows, inner, pad + 8)
    wg, wu = put(inner, hidden, pad, hidden ** -0.5), put(inner, hidden, pad, hidden ** -0.5)
    gg, uu = put(rows, inner, pad), put(rows, inner, pad)
    dbl = lambda b: b.view.cpu().double()  # noqa: E731
    dg, du, dx, dwg, dwu = forms.ffn_grad(dbl(dh), dbl(x), dbl(wg), dbl(wu), dbl(gg), dbl(uu), name)
    tiny = forms.TINY[dtype]
    # dg, du in binary32: 16 roundings of the factors' sizes (|act'| <= 1.13, but made of parts up to 1 + |g|), then one of the type
    eg = u * dg.abs() + tiny + 16 * E * (dbl(dh) * dbl(uu)).abs() * (1 + dbl(gg).abs())
    eu = u * du.abs() + tiny + 16 * E * (dbl(dh) * dbl(gg)).abs()
    em, er = 4 * math.sqrt(2 * inner) * 2 * E, 4 * math.sqrt(rows) * 2 * E
    dx_tol = u * dx.abs() + tiny + eg @ dbl(wg).abs() + eu @ dbl(wu).abs() + em * (dg.abs() @ dbl(wg).abs() + du.abs() @ dbl(wu).abs())
    for want_dx, want_dw in ((True, True), (True, False), (False, True)):
        o_dx, o_dwg, o_dwu = Guarded(rows, hidden, t, pad + 8), Guarded(inner, hidden, t, pad + 8), Guarded(inner, hidden, t, pad + 8)
        aq.aq_gated_ffn_grad(stage, dh.view, dh.ld, x.view, x.ld, wg.view, wu.view, wg.ld, gg.view, uu.view, gg.ld, rows, hidden, inner,
                             act_key(aq, name), o_dx.view if want_dx else None, o_dx.ld, o_dwg.view if want_dw else None,
                             o_dwu.view if want_dw else None, o_dwg.ld)
        torch.cuda.synchronize()
        for b in (x, dh, wg, wu, gg, uu, o_dx, o_dwg, o_dwu):
            b.check()
        if want_dx:
            within(o_dx.view, dx, dx_tol)
        else:
            assert bool((o_dx.view == -7).all())
        if want_dw:
            within(o_dwg.view, dwg, u * dwg.abs() + tiny + eg.T @ dbl(x).abs() + er * (dg.abs().T @ dbl(x).abs()))
            within(o_dwu.view, dwu, u * dwu.abs() + tiny + eu.T @ dbl(x).abs() + er * (du.abs().T @ dbl(x).abs()))
        else:
            assert bool((o_dwg.view == -7).all() and (o_dwu.view == -7).all())


def test_gated_ffn_gradient_against_differences(aq, stage):
    """Directional differences of the 64-bit forward form against the library's gradients.  Each of the n products of a
    directional sum is off by up to 2u of its size (its own rounding and dg's): 2u sqrt(n) rms, times four."""
    set_type(aq, stage, "fp16")
    rows, hidden, inner, name = 60, 72, 80, "silu"
    gen = torch.Generator().manual_seed(11)
    r = lambda *s: torch.randn(s, generator=gen).half()  # noqa: E731
    x, wg, wu, dh = r(rows, hidden), (r(inner, hidden) / 8).half(), (r(inner, hidden) / 8).half(), r(rows, inner)
    h, g, u = (torch.empty((rows, inner), dtype=torch.float16, device="cuda") for _ in range(3))
    c = [v.cuda() for v in (x, wg, wu, dh)]
    aq.aq_gated_ffn(stage, c[0], hidden, c[1], c[2], hidden, rows, hidden, inner, aq.AQ_ACT_SILU, h, inner, g, u, inner)
    grads = [torch.empty_like(c[0]), torch.empty_like(c[1]), torch.empty_like(c[2])]
    aq.aq_gated_ffn_grad(stage, c[3], inner, c[0], hidden, c[1], c[2], hidden, g, u, inner, rows, hidden, inner, aq.AQ_ACT_SILU,
                         grads[0], hidden, grads[1], grads[2], hidden)
    args = [x.double(), wg.double(), wu.double()]
    for at in range(3):
        v = torch.randn(args[at].shape, generator=gen, dtype=F64)
        f = lambda y: (forms.ffn(*[y if i == at else a for i, a in enumerate(args)], name)[0] * dh.double()).sum()  # noqa: E731
        want = ((f(args[at] + 1e-4 * v) - f(args[at] - 1e-4 * v)) / 2e-4).item()
        terms = grads[at].cpu().double() * v
        assert abs(terms.sum().item() - want) < 4 * 2 * forms.UNIT["fp16"] * terms.square().sum().sqrt().item() * 4


def test_gated_ffn_no_rows(aq, stage):
    set_type(aq, stage, "fp16")
    w = torch.ones((16, 8), dtype=torch.float16, device="cuda")
    d = Guarded(16, 8, torch.float16, 8)
    e = Guarded(16, 8, torch.float16, 8)
    aq.aq_gated_ffn(stage, None, 8, w, w, 8, 0, 8, 16, 0, None, 16, None, None, 16)
    aq.aq_gated_ffn_grad(stage, None, 16, None, 8, w, w, 8, None, None, 16, 0, 8, 16, 0, None, 8, d.view, e.view, d.ld)
    torch.cuda.synchronize()
    assert bool((d.view == 0).all() and (e.view == 0).all())
    d.check()


# ---- norm and rotation of query and key heads ------------------------------------------------------------------

def table(n, rot):
    a = torch.arange(n, dtype=F64)[:, None] * 100.0 ** (-torch.arange(rot // 2, dtype=F64) * 2 / max(rot, 1))[None]
    return torch.cat([a.cos(), a.sin()], 1).float()


QK_SHAPES = [  # rows, heads_q, heads_k, head_dim, rot, interleaved
    (1, 1, 1, 8, 8, False), (1, 25, 25, 64, 64, False), (3, 25, 25, 64, 64, True), (7, 12, 4, 64, 32, False), (5, 3, 1, 8, 2, True),
    (4, 5, 2, 16, 4, False), (9, 7, 0, 24, 24, False), (6, 0, 3, 40, 40, True), (11, 6, 2, 40, 20, False), (5, 4, 4, 80, 80, False),
    (13, 3, 3, 96, 96, False), (2, 8, 2, 128, 128, False), (300, 9, 3, 128, 64, True), (33, 2, 1, 136, 136, False), (3, 2, 2, 192, 50, False),
    (5, 3, 1, 256, 256, False), (4, 2, 2, 256, 0, False), (2000, 4, 2, 32, 16, False)]


def qk_buffers(dtype, rows, nq, nk, dh, gen, pad=8):
    t = forms.TYPES[dtype]
    wide = Guarded(rows, (nq + nk) * dh + 16, t, pad).put(torch.randn((rows, (nq + nk) * dh + 16), generator=gen))
    return wide, wide.view[:, :nq * dh], wide.view[:, nq * dh:(nq + nk) * dh]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rows,nq,nk,dh,rot,interleaved", QK_SHAPES)
def test_qk_norm_rope(aq, stage, dtype, rows, nq, nk, dh, rot, interleaved):
    """Every value is a handful of binary32 operations on the head's elements: 16 roundings of the pair's size, then one of the type."""
    set_type(aq, stage, dtype)
    t, u = forms.TYPES[dtype], forms.UNIT[dtype]
    gen = torch.Generator().manual_seed(rows + 17 * dh + rot)
    wide, q, k = qk_buffers(dtype, rows, nq, nk, dh, gen)
    if rows > 2:
        wide.view[2] = 0.0                                       # a token of zeros: eps alone
    weights = rot != 2
    wq, wk = ((1 + 0.3 * torch.randn(dh, generator=gen)).to(t) for _ in range(2))
    n_pos = 40
    cs, positions = table(n_pos, rot), torch.randint(0, n_pos, (rows,), generator=gen, dtype=torch.int32)
    positions[-1] = n_pos - 1
    shape = aq.QkShape(heads_q=nq, heads_k=nk, head_dim=dh, rot_dim=rot, interleaved=int(interleaved), eps=1e-5, n_positions=n_pos)
    eps = torch.tensor(1e-5, dtype=torch.float32).double().item()
    want = []
    for x, w, heads in ((q, wq, nq), (k, wk, nk)):
        x64 = x.cpu().double().reshape(rows, heads, dh)
        w64 = w.double() if weights else torch.ones(dh, dtype=F64)
        y = forms.qk(x64, w64, eps, cs.double(), positions.long(), rot, interleaved).reshape(rows, -1)
        size = forms.qk(x64, w64, eps, torch.cat([torch.ones(n_pos, rot // 2), torch.zeros(n_pos, rot // 2)], 1).double(), positions.long(), rot, interleaved)
        want.append((y, u * y.abs() + forms.TINY[dtype] + 32 * E * size.abs().amax(-1, keepdim=True).expand(rows, heads, dh).reshape(rows, -1)))
    tables = (cs.cuda(), positions.cuda()) if rot else (None, None)
    w_dev = (wq.cuda(), wk.cuda()) if weights else (None, None)
    oq, ok = Guarded(rows, nq * dh, t, 8), Guarded(rows, nk * dh, t, 16)
    aq.aq_qk_norm_rope(stage, shape, rows, q, wide.ld, k, wide.ld, *w_dev, *tables, oq.view if nq else None, oq.ld, ok.view if nk else None, ok.ld)
    torch.cuda.synchronize()
    for b in (oq, ok, wide):
        b.check()
    for out, (y, tol) in ((oq, want[0]), (ok, want[1])):
        if y.numel():
            within(out.view, y, tol)
    # in place
    aq.aq_qk_norm_rope(stage, shape, rows, q, wide.ld, k, wide.ld, *w_dev, *tables, q, wide.ld, k, wide.ld)
    torch.cuda.synchronize()
    assert torch.equal(q, oq.view) and torch.equal(k, ok.view)
    wide.check()
    assert aq.aq_stage_status(stage) == 0


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rows,nq,nk,dh,rot,interleaved", QK_SHAPES)
def test_qk_norm_rope_gradient(aq, stage, dtype, rows, nq, nk, dh, rot, interleaved):
    """Against torch's differentiation of the 64-bit form.  dx: 64 binary32 roundings of the largest term of its head.  dw: a
    sum of rows * heads products, 4 sqrt(n) 2e of their magnitudes and 32e each."""
    set_type(aq, stage, dtype)
    t, u = forms.TYPES[dtype], forms.UNIT[dtype]
    gen = torch.Generator().manual_seed(rows + 17 * dh + rot + 1)
    wide, q, k = qk_buffers(dtype, rows, nq, nk, dh, gen)
    gwide, gq, gk = qk_buffers(dtype, rows, nq, nk, dh, gen)
    wq, wk = ((1 + 0.3 * torch.randn(dh, generator=gen)).to(t) for _ in range(2))
    n_pos = 40
    cs, positions = table(n_pos, rot), torch.randint(0, n_pos, (rows,), generator=gen, dtype=torch.int32)
    shape = aq.QkShape(heads_q=nq, heads_k=nk, head_dim=dh, rot_dim=rot, interleaved=int(interleaved), eps=1e-5, n_positions=n_pos)
    eps = torch.tensor(1e-5, dtype=torch.float32).double().item()
    tables = (cs.cuda(), positions.cuda()) if rot else (None, None)
    oq, ok = Guarded(rows, nq * dh, t, 8), Guarded(rows, nk * dh, t, 16)
    dwq, dwk = floats(dh), floats(dh)
    args = (rows, gq, gwide.ld, gk, gwide.ld, q, wide.ld, k, wide.ld, wq.cuda(), wk.cuda(), *tables)
    aq.aq_qk_norm_rope_grad(stage, shape, *args, oq.view if nq else None, oq.ld, ok.view if nk else None, ok.ld, dwq, dwk)
    torch.cuda.synchronize()
    for b in (oq, ok, wide, gwide):
        b.check()
    for x, dy, w, heads, out, dw in ((q, gq, wq, nq, oq, dwq), (k, gk, wk, nk, ok, dwk)):
        if not heads:
            assert bool((dw == 0).all())
            continue
        x64 = x.cpu().double().reshape(rows, heads, dh).requires_grad_(True)
        w64 = w.double().requires_grad_(True)
        dy64 = dy.cpu().double().reshape(rows, heads, dh)
        y = forms.qk(x64, w64, eps, cs.double(), positions.long(), rot, interleaved)
        dx, dw_want = torch.autograd.grad(y, (x64, w64), dy64)
        r = 1 / torch.sqrt(x64.detach().square().mean(-1, keepdim=True) + eps)
        largest = (r * dy64.abs().amax(-1, keepdim=True) * w.double().abs().max() * (1 + (x64.detach() * r).abs().amax(-1, keepdim=True)) ** 2).expand_as(dx)
        within(out.view, dx.reshape(rows, -1), (u * dx.abs() + forms.TINY[dtype] + 64 * E * largest).reshape(rows, -1))
        n = rows * heads
        mags = ((x64.detach() * r).abs() * 1.5 * dy64.abs().amax(-1, keepdim=True)).sum((0, 1))
        within(dw, dw_want, mags * E * (8 * math.sqrt(n) + 32))
    # the same bits again, in place, and without the weights' sums
    dwq2, dwk2 = floats(dh), floats(dh)
    aq.aq_qk_norm_rope_grad(stage, shape, *args, oq.view if nq else None, oq.ld, ok.view if nk else None, ok.ld, dwq2, dwk2)
    aq.aq_qk_norm_rope_grad(stage, shape, *args, gq, gwide.ld, gk, gwide.ld, None, None)
    torch.cuda.synchronize()
    assert torch.equal(dwq, dwq2) and torch.equal(dwk, dwk2)
    assert torch.equal(gq, oq.view) and torch.equal(gk, ok.view)


def test_qk_bad_position_zero_fills_the_token(aq, stage):
    set_type(aq, stage, "fp16")
    rows, nq, nk, dh = 5, 3, 2, 16
    x = torch.randn((rows, (nq + nk) * dh)).half().cuda()
    cs = table(10, 16).cuda()
    good, bad = torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32, device="cuda"), torch.tensor([0, 10, 2, -1, 4], dtype=torch.int32, device="cuda")
    shape = aq.QkShape(heads_q=nq, heads_k=nk, head_dim=dh, rot_dim=16, interleaved=0, eps=1e-6, n_positions=10)
    ld = (nq + nk) * dh

    def both(positions, grad):
        out = torch.full_like(x, 5.0)
        dw = floats(dh), floats(dh)
        if grad:
            aq.aq_qk_norm_rope_grad(stage, shape, rows, x, ld, x[:, nq * dh:], ld, x, ld, x[:, nq * dh:], ld, None, None, cs, positions,
                                    out, ld, out[:, nq * dh:], ld, *dw)
        else:
            aq.aq_qk_norm_rope(stage, shape, rows, x, ld, x[:, nq * dh:], ld, None, None, cs, positions, out, ld, out[:, nq * dh:], ld)
        torch.cuda.synchronize()
        return out, dw
    for grad in (False, True):
        a, _ = both(good, grad)
        assert aq.aq_stage_status(stage) == 0
        b, dw = both(bad, grad)
        assert aq.aq_stage_status(stage) == aq.AQ_ST_BAD_ID
        assert bool((b[[1, 3]] == 0).all()) and torch.equal(a[[0, 2, 4]], b[[0, 2, 4]])
        if grad:
            keep = x[[0, 2, 4]].contiguous()
            out = torch.empty_like(keep)
            dw3 = floats(dh), floats(dh)
            aq.aq_qk_norm_rope_grad(stage, shape, 3, keep, ld, keep[:, nq * dh:], ld, keep, ld, keep[:, nq * dh:], ld, None, None, cs,
                                    good[[0, 2, 4]].contiguous(), out, ld, out[:, nq * dh:], ld, *dw3)
            assert torch.allclose(dw[0], dw3[0], rtol=1e-5, atol=1e-5) and torch.allclose(dw[1], dw3[1], rtol=1e-5, atol=1e-5)


# ---- streams, handles, refusals --------------------------------------------------------------------------------

def test_another_stream_and_a_captured_graph(aq, stage):
    set_type(aq, stage, "bf16")
    side = torch.cuda.Stream()
    rows, vocab, hidden, inner = 6, 5000, 64, 128
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    logits, x, wg, wu, dh = rnd(rows, vocab), rnd(rows, hidden), rnd(inner, hidden), rnd(inner, hidden), rnd(rows, inner)
    targets = torch.arange(rows, dtype=torch.int32, device="cuda")
    lp, ent, lse = floats(rows), floats(rows), floats(rows)
    d, h, g, u, dx, dwg, dwu = (torch.zeros_like(v) for v in (logits, dh, dh, dh, x, wg, wu))

    def calls():
        aq.aq_token_logprobs(stage, logits, rows, vocab, vocab, targets, 1.0, 0, lp, ent, lse, None, None)
        aq.aq_token_logprobs_grad(stage, logits, rows, vocab, vocab, targets, 1.0, lse, None, lp, None, d, vocab)
        aq.aq_gated_ffn(stage, x, hidden, wg, wu, hidden, rows, hidden, inner, 0, h, inner, g, u, inner)
        aq.aq_gated_ffn_grad(stage, dh, inner, x, hidden, wg, wu, hidden, g, u, inner, rows, hidden, inner, 0, dx, hidden, dwg, dwu, hidden)
    calls()
    torch.cuda.synchronize()
    outs = [lp, ent, lse, d, h, g, u, dx, dwg, dwu]
    want = [v.clone() for v in outs]
    for v in outs:
        v.zero_()
    torch.cuda.synchronize()
    aq.aq_stage_configure(stage, aq.AQ_STREAM, side.cuda_stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert torch.equal(a, b)
    # a capture that would need a larger workspace is refused, not broken
    big = 4096
    x2, dh2, g2 = (torch.zeros((big, n), dtype=torch.bfloat16, device="cuda") for n in (hidden, inner, inner))
    refused = []
    graph2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph2, stream=side):
        try:
            aq.aq_gated_ffn_grad(stage, dh2, inner, x2, hidden, wg, wu, hidden, g2, g2, inner, big, hidden, inner, 0, x2, hidden, dwg, dwu, hidden)
        except aq.AqError as e:
            refused.append(e.code)
        h.zero_()
    assert refused == [aq.AQ_EUNSUPPORTED]
    aq.aq_stage_configure(stage, aq.AQ_STREAM, 0)


def test_two_handles_on_two_streams(aq):
    """The same calls on two handles side by side, many times: each has its own counters and workspace."""
    rows, hidden, inner = 700, 200, 1000
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    x, wg, wu, dh = rnd(rows, hidden), rnd(inner, hidden) / 14, rnd(inner, hidden) / 14, rnd(rows, inner)
    qk, dqk, cs, pos = rnd(rows, 6 * 64), rnd(rows, 6 * 64), table(40, 64).cuda(), torch.arange(rows, dtype=torch.int32, device="cuda") % 40
    shape = aq.QkShape(heads_q=4, heads_k=2, head_dim=64, rot_dim=64, interleaved=0, eps=1e-6, n_positions=40)
    sides = []
    for i in range(2):
        st, stream = aq.aq_stage_create(), torch.cuda.Stream()
        set_type(aq, st, "bf16")
        aq.aq_stage_configure(st, aq.AQ_STREAM, stream.cuda_stream)
        outs = [torch.zeros_like(v) for v in (dh, dh, dh, x, wg, wu, dqk)] + [floats(64), floats(64)]
        sides.append((st, stream, outs))
    torch.cuda.synchronize()

    def calls(st, o):
        aq.aq_gated_ffn(st, x, hidden, wg, wu, hidden, rows, hidden, inner, 0, o[0], inner, o[1], o[2], inner)
        aq.aq_gated_ffn_grad(st, dh, inner, x, hidden, wg, wu, hidden, o[1], o[2], inner, rows, hidden, inner, 0, o[3], hidden, o[4], o[5], hidden)
        aq.aq_qk_norm_rope_grad(st, shape, rows, dqk, 384, dqk[:, 256:], 384, qk, 384, qk[:, 256:], 384, None, None, cs, pos, o[6], 384,
                                o[6][:, 256:], 384, o[7], o[8])
    calls(sides[0][0], sides[0][2])
    torch.cuda.synchronize()
    want = [v.clone() for v in sides[0][2]]
    for _ in range(20):
        for st, _, outs in sides:
            calls(st, outs)
    torch.cuda.synchronize()
    for st, _, outs in sides:
        assert aq.aq_stage_status(st) == 0
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
        aq.aq_stage_destroy(st)


def test_offsets_beyond_32_bits(aq, stage):
    """Buffers of more than 2^31 elements: the last rows against the same rows alone."""
    set_type(aq, stage, "bf16")
    rows, ld = 40000, 60000                                         # 2.4e9 elements
    big = torch.zeros((rows, ld), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((64, 5003), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    big[-64:, :5003] = tail
    targets = torch.full((rows,), 7, dtype=torch.int32, device="cuda")
    lp, ent, lse = floats(rows), floats(rows), floats(rows)
    aq.aq_token_logprobs(stage, big, rows, 5003, ld, targets, 1.0, 0, lp, ent, lse, None, None)
    one, e1, l1 = floats(64), floats(64), floats(64)
    aq.aq_token_logprobs(stage, tail, 64, 5003, 5003, targets, 1.0, 0, one, e1, l1, None, None)
    torch.cuda.synchronize()
    assert torch.allclose(lp[-64:], one, atol=2e-5) and torch.allclose(ent[-64:], e1, atol=4e-5)
    d, d1 = torch.empty_like(tail), torch.empty_like(tail)
    aq.aq_token_logprobs_grad(stage, big, rows, 5003, ld, targets, 1.0, lse, None, torch.ones_like(lp), None, big, ld)       # in place
    aq.aq_token_logprobs_grad(stage, tail, 64, 5003, 5003, targets, 1.0, lse[-64:].clone(), None, torch.ones_like(one), None, d1, 5003)
    torch.cuda.synchronize()
    assert torch.equal(big[-64:, :5003], d1)
    del d
    # heads and the feed-forward product on the same buffer: 64 columns of rows that far apart
    big[-64:, :256] = torch.randn((64, 256), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
    part = big[-64:, :256].clone()
    cs, pos = table(40, 64).cuda(), torch.arange(rows, dtype=torch.int32, device="cuda") % 40
    shape = aq.QkShape(heads_q=2, heads_k=1, head_dim=64, rot_dim=64, interleaved=0, eps=1e-6, n_positions=40)
    w = torch.randn((72, 64), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").bfloat16()
    h, h1 = (torch.empty((n, 72), dtype=torch.bfloat16, device="cuda") for n in (rows, 64))
    aq.aq_gated_ffn(stage, big, ld, w, w, 64, rows, 64, 72, 0, h, 72, None, None, 72)
    aq.aq_gated_ffn(stage, part, 256, w, w, 64, 64, 64, 72, 0, h1, 72, None, None, 72)
    aq.aq_qk_norm_rope(stage, shape, rows, big, ld, big[:, 128:], ld, None, None, cs, pos, big, ld, big[:, 128:], ld)
    aq.aq_qk_norm_rope(stage, shape, 64, part, 256, part[:, 128:], 256, None, None, cs, pos[-64:].clone(), part, 256, part[:, 128:], 256)
    torch.cuda.synchronize()
    assert torch.equal(h[-64:], h1) and torch.equal(big[-64:, :256], part)
    assert aq.aq_stage_status(stage) == 0


def test_refusals(aq, stage):
    L, F = aq.lib(), torch.float16
    x = torch.zeros((64, 64), dtype=F, device="cuda")
    f, i32 = floats(64), torch.zeros(64, dtype=torch.int32, device="cuda")
    p = x.data_ptr()

    def refused(code, name, *args):
        assert getattr(L, name)(stage, *args) == code, (name, args)
        assert aq.aq_stage_last_error(stage) and aq.aq_stage_last_error_code(stage) == code
    I, U = aq.AQ_EINVAL, aq.AQ_EUNSUPPORTED
    refused(I, "aq_stage_configure", aq.AQ_DTYPE, 3)
    refused(I, "aq_stage_configure", aq.AQ_BATCH, 1)
    lp = lambda logits=p, rows=4, vocab=64, ld=64, t=i32.data_ptr(), scale=1.0, k=0: (logits, rows, vocab, ld, t, scale, k, f.data_ptr(), None, None, None, None)  # noqa: E731
    for bad in (lp(logits=None), lp(logits=p + 1), lp(rows=-1), lp(vocab=0), lp(ld=63), lp(scale=0.0), lp(scale=-1.0), lp(scale=math.inf), lp(scale=math.nan),
                lp(k=-1), lp(k=33), lp(vocab=5, k=6), lp(t=None), lp(t=i32.data_ptr() + 2)):
        refused(I, "aq_token_logprobs", *bad)
    gr = lambda lse=f.data_ptr(), ent=None, dl=f.data_ptr(), de=None, out=p, ldd=64, t=i32.data_ptr(): (p, 4, 64, 64, t, 1.0, lse, ent, dl, de, out, ldd)  # noqa: E731
    for bad in (gr(lse=None), gr(de=f.data_ptr()), gr(out=None), gr(ldd=63), gr(ldd=65), gr(t=None), gr(out=p + 1)):
        refused(I, "aq_token_logprobs_grad", *bad)
    ff = lambda x=p, ldx=64, wg=p, wu=p, ldw=64, rows=4, hidden=64, inner=64, act=0, h=p, ldh=64, g=None, u=None, ldgu=64: (x, ldx, wg, wu, ldw, rows, hidden, inner, act, h, ldh, g, u, ldgu)  # noqa: E731
    for bad in (ff(x=None), ff(x=p + 2), ff(ldx=56), ff(ldx=68), ff(wg=None), ff(wu=p + 8), ff(ldw=60), ff(rows=-1), ff(hidden=0), ff(act=3), ff(h=None), ff(g=p), ff(u=p),
                ff(ldh=63), ff(g=p, u=p, ldgu=8)):
        refused(I, "aq_gated_ffn", *bad)
    refused(U, "aq_gated_ffn", *ff(hidden=60))
    refused(U, "aq_gated_ffn", *ff(inner=12))
    fg = lambda dh=p, x=p, g=p, u=p, dx=p, dwg=p, dwu=p, lddw=64, act=0, inner=64: (dh, 64, x, 64, p, p, 64, g, u, 64, 4, 64, inner, act, dx, 64, dwg, dwu, lddw)  # noqa: E731
    for bad in (fg(dh=None), fg(x=None), fg(g=None), fg(u=None), fg(dx=p + 4), fg(dwg=None), fg(dwu=None), fg(lddw=8), fg(act=-1)):
        refused(I, "aq_gated_ffn_grad", *bad)
    refused(U, "aq_gated_ffn_grad", *fg(inner=20))
    import ctypes
    sh = lambda **k: ctypes.byref(aq.QkShape(**{**dict(heads_q=2, heads_k=2, head_dim=16, rot_dim=16, interleaved=0, eps=1e-6, n_positions=8), **k}))  # noqa: E731
    qk = lambda shape=sh(), rows=2, q=p, qs=64, k=p, ks=64, wq=None, cs=f.data_ptr(), pos=i32.data_ptr(), oq=p, oqs=64, ok=p, oks=64: (shape, rows, q, qs, k, ks, wq, None, cs, pos, oq, oqs, ok, oks)  # noqa: E731
    for bad in (qk(shape=None), qk(shape=sh(heads_q=-1)), qk(shape=sh(heads_q=0, heads_k=0)), qk(shape=sh(head_dim=12)), qk(shape=sh(head_dim=264)),
                qk(shape=sh(rot_dim=3)), qk(shape=sh(rot_dim=18)), qk(shape=sh(eps=-1.0)), qk(shape=sh(eps=math.nan)), qk(shape=sh(n_positions=0)), qk(rows=-1),
                qk(q=None), qk(q=p + 8), qk(qs=31), qk(qs=24), qk(k=None), qk(wq=p + 2), qk(cs=None), qk(pos=None), qk(oq=None), qk(oqs=72), qk(oks=16)):
        refused(I, "aq_qk_norm_rope", *bad)
    qg = lambda shape=sh(), gq=p, q=p, dq=p, dqs=64, dwq=None: (shape, 2, gq, 64, p, 64, q, 64, p, 64, None, None, f.data_ptr(), i32.data_ptr(), dq, dqs, p, 64, dwq, None)  # noqa: E731
    for bad in (qg(shape=None), qg(gq=None), qg(q=None), qg(dq=None), qg(dqs=72), qg(dwq=f.data_ptr() + 2)):
        refused(I, "aq_qk_norm_rope_grad", *bad)
    set_type(aq, stage, "fp32")
    refused(U, "aq_gated_ffn", *ff())
    refused(U, "aq_gated_ffn_grad", *fg())
    refused(U, "aq_qk_norm_rope", *qk())
    refused(U, "aq_qk_norm_rope_grad", *qg())
    # nothing was launched by any of them
    assert aq.aq_stage_status(stage) == 0 and bool((x == 0).all()) and bool((f == 77).all())
