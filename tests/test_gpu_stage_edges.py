"""Stage operators where data, sizes or histories are out of the ordinary, against the plain 64-bit forms (stage_forms.py).

Tolerances as in test_gpu_stage.py: u is one rounding to the output type, E = 2^-24 one binary32 rounding.
"""
import math

import pytest
import torch

from tests import stage_forms as forms
from tests.test_gpu_stage import E, F64, Guarded, act_key, aq, check_logprobs, floats, run_logprobs, run_logprobs_grad, set_type, stage, table, within  # noqa: F401

pytestmark = pytest.mark.gpu


# ---- the workspace of the feed-forward gradient -----------------------------------------------------------------------

def test_a_captured_gradient_survives_a_larger_workspace(aq, stage):
    """Graphs of the gradient call at two sizes, larger calls between, then replays on new inputs: what the eager calls give.  The larger
    calls' outputs are in other memory, and so must be the workspaces that the graphs hold."""
    set_type(aq, stage, "bf16")
    hidden, inner = 64, 136
    gen = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    wg, wu = rnd(inner, hidden) / 8, rnd(inner, hidden) / 8

    def operands(rows):
        ins = [rnd(rows, inner), rnd(rows, hidden), rnd(rows, inner), rnd(rows, inner)]
        return ins, [torch.zeros((n, hidden), dtype=torch.bfloat16, device="cuda") for n in (rows, inner, inner)]

    def call(ins, outs):
        (dh, x, g, u), (dx, dwg, dwu) = ins, outs
        aq.aq_gated_ffn_grad(stage, dh, inner, x, hidden, wg, wu, hidden, g, u, inner, x.shape[0], hidden, inner, aq.AQ_ACT_SILU, dx, hidden, dwg, dwu, hidden)

    side = torch.cuda.Stream()
    aq.aq_stage_configure(stage, aq.AQ_STREAM, side.cuda_stream)
    graphs = []
    for rows in (40, 300):                                         # the second outgrows the first one's workspace
        ins, outs = operands(rows)
        torch.cuda.synchronize()
        call(ins, outs)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(ins, outs)
        graphs.append((graph, ins, outs))
    large = operands(5000)                                         # outgrows both
    torch.cuda.synchronize()
    call(*large)
    torch.cuda.synchronize()
    between = [v.clone() for v in large[1]]
    filler = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(64)]      # whatever was freed has new owners
    for graph, ins, outs in graphs:
        for v in ins:
            v.copy_(rnd(*v.shape))
        torch.cuda.synchronize()
        call(ins, outs)
        torch.cuda.synchronize()
        want = [v.clone() for v in outs]
        for v in outs:
            v.zero_()
        torch.cuda.synchronize()
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
    assert all(bool(torch.isnan(v).all()) for v in filler)
    call(*large)
    torch.cuda.synchronize()
    for a, b in zip(large[1], between):
        assert torch.equal(a, b)
    assert aq.aq_stage_status(stage) == 0
    aq.aq_stage_configure(stage, aq.AQ_STREAM, 0)


def test_an_outgrown_workspace_that_no_graph_holds_is_freed(aq, stage):
    """Sixteen growing calls, 1 to 16 times 32 MB of workspace: 4.4 GB were all kept, 0.5 GB when only the last is."""
    set_type(aq, stage, "fp16")
    hidden, inner = 8, 8192
    w = torch.zeros((inner, hidden), dtype=torch.float16, device="cuda")
    d = [torch.zeros((inner, hidden), dtype=torch.float16, device="cuda") for _ in range(2)]
    rows = 16 * 1024
    x, g = torch.zeros((rows, hidden), dtype=torch.float16, device="cuda"), torch.zeros((rows, inner), dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for i in range(1, 17):
        aq.aq_gated_ffn_grad(stage, g, inner, x, hidden, w, w, hidden, g, g, inner, i * 1024, hidden, inner, 0, None, 8, d[0], d[1], hidden)
    torch.cuda.synchronize()
    assert free - torch.cuda.mem_get_info()[0] < 1.5e9


# ---- norm and rotation: what must not reach the weights' gradients --------------------------------------------------

QK_WAYS = [  # rows, heads_q, heads_k, head_dim, rot, interleaved: each way to a pair's other member, heads that do and do not fill a warp
    (40, 3, 2, 64, 64, False), (40, 5, 1, 64, 32, True), (40, 3, 3, 40, 40, False), (2500, 3, 1, 128, 64, False), (40, 7, 3, 24, 12, False)]


def qk_grad_call(aq, st, shape, x, dy, nq, cs, positions, w):
    """Outputs of the gradient call on [rows, (heads_q + heads_k) * head_dim] tensors, with the weights' sums."""
    rows, ld = x.shape
    out, dwq, dwk = torch.full_like(x, 5.0), floats(shape.head_dim), floats(shape.head_dim)
    aq.aq_qk_norm_rope_grad(st, shape, rows, dy, ld, dy[:, nq:], ld, x, ld, x[:, nq:], ld, w, w, cs, positions, out, ld, out[:, nq:], ld, dwq, dwk)
    torch.cuda.synchronize()
    return out, dwq, dwk


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rows,heads_q,heads_k,dh,rot,interleaved", QK_WAYS)
def test_qk_gradient_tokens_outside_the_table_may_hold_anything(aq, stage, dtype, rows, heads_q, heads_k, dh, rot, interleaved):
    """Padding is often uninitialised memory: its NaNs and infinities change no bit of anything."""
    set_type(aq, stage, dtype)
    t, nq, wide = forms.TYPES[dtype], heads_q * dh, (heads_q + heads_k) * dh
    gen = torch.Generator().manual_seed(dh + rot)
    x, dy = (torch.randn((rows, wide), generator=gen).to(t).cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(dh, generator=gen)).to(t).cuda()
    positions = torch.randint(0, 40, (rows,), generator=gen, dtype=torch.int32)
    off = torch.rand(rows, generator=gen) < 0.3
    off[0], off[-1] = True, True
    positions[off] = torch.where(torch.rand(int(off.sum()), generator=gen) < 0.5, -1, 40).int()
    shape = aq.QkShape(heads_q=heads_q, heads_k=heads_k, head_dim=dh, rot_dim=rot, interleaved=int(interleaved), eps=1e-6, n_positions=40)
    cs, positions, off = table(40, rot).cuda(), positions.cuda(), off.cuda()
    want = qk_grad_call(aq, stage, shape, x, dy, nq, cs, positions, w)
    assert aq.aq_stage_status(stage) == aq.AQ_ST_BAD_ID
    assert all(bool(torch.isfinite(v).all()) for v in want)
    n = int(off.sum())
    junk = torch.tensor([math.nan, math.inf, -math.inf, 1.0])
    for where in (x, dy):
        kept = where.clone()
        where[off] = junk[torch.randint(0, 4, (n, wide), generator=gen)].to(t).cuda()
        got = qk_grad_call(aq, stage, shape, x, dy, nq, cs, positions, w)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        if where is x:
            where.copy_(kept)                                     # then in dy alone
    assert aq.aq_stage_status(stage) == aq.AQ_ST_BAD_ID


@pytest.mark.parametrize("rows,heads_q,heads_k,dh,rot,interleaved", QK_WAYS)
@pytest.mark.parametrize("where", ["x", "dy"])
def test_qk_gradient_an_infinity_stays_in_its_columns(aq, stage, rows, heads_q, heads_k, dh, rot, interleaved, where):
    """One infinite element in the last head.  dw sums dy n over rows and heads, column by column: an infinite x_e makes n_e NaN and the
    head's other n 0; an infinite dy_e reaches, turned back, its own column and that of the other member of its pair (neighbours,
    where pairs are neighbours).  No other column, and no weight of the other tensor, may notice."""
    set_type(aq, stage, "bf16")
    nq, wide = heads_q * dh, (heads_q + heads_k) * dh
    gen = torch.Generator().manual_seed(dh + rot)
    x, dy = (torch.randn((rows, wide), generator=gen).bfloat16().cuda() for _ in range(2))
    w = (1 + 0.3 * torch.randn(dh, generator=gen)).bfloat16().cuda()
    positions = torch.randint(1, 40, (rows,), generator=gen, dtype=torch.int32).cuda()
    shape = aq.QkShape(heads_q=heads_q, heads_k=heads_k, head_dim=dh, rot_dim=rot, interleaved=int(interleaved), eps=1e-6, n_positions=40)
    for first, heads, which in ((0, heads_q, 1), (nq, heads_k, 2)):
        for e in (dh - 1, dh - 8):
            a, b = x.clone(), dy.clone()
            (a if where == "x" else b)[rows // 2, first + (heads - 1) * dh + e] = math.inf
            got = qk_grad_call(aq, stage, shape, a, b, nq, table(40, rot).cuda(), positions, w)
            partner = e ^ 1 if interleaved else e if e >= rot else (e + rot // 2) % rot
            touched = {e} if where == "x" else {e, partner}
            assert bool(torch.isfinite(got[3 - which]).all())
            assert set(torch.nonzero(~torch.isfinite(got[which])).flatten().tolist()) == touched


# ---- feed-forward: many tiles a pair ------------------------------------------------------------------------------

def ffn_case(rows, hidden, inner, t, seed, pad=0):
    """Operands of a call, its weights scaled to outputs near one; the 64-bit forms are evaluated on the GPU."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    put = lambda r, c, s=1.0: Guarded(r, c, t, pad).put(s * torch.randn((r, c), generator=gen, device="cuda"))  # noqa: E731
    return put(rows, hidden), put(inner, hidden, hidden ** -0.5), put(inner, hidden, hidden ** -0.5)


def call_ffn(aq, st, x, wg, wu, name, out):
    rows, hidden = x.view.shape
    aq.aq_gated_ffn(st, x.view, x.ld, wg.view, wu.view, wg.ld, rows, hidden, wg.view.shape[0], act_key(aq, name), *out)


def forward_tiles(rows, inner):
    return -(-rows // 256) * -(-inner // 128)                      # at least: a tile has 256 rows and up to 128 outputs


def backward_tiles(rows, hidden, inner):
    return (-(-rows // 256) + 2 * -(-inner // 256)) * -(-hidden // 256)     # at least: 256 x up to 256, dx whole


def pairs_at_most():
    return torch.cuda.get_device_properties(0).multi_processor_count // 2


def test_gated_ffn_after_a_call_that_gave_up(aq, stage):
    """A kernel whose wait ran out may leave its tile counter anywhere.  The counter is put there by hand (nothing else that is safe
    makes a wait run out): the call that meets it is lost, the ones after it are whole again."""
    import ctypes

    class Head(ctypes.Structure):                                  # what the handle begins with
        _fields_ = [("device", ctypes.c_int), ("sms", ctypes.c_int), ("pairs", ctypes.c_int), ("dtype", ctypes.c_int), ("stream", ctypes.c_void_p),
                    ("status", ctypes.c_void_p), ("ticket", ctypes.c_void_p), ("next", ctypes.c_void_p)]
    head = Head.from_address(stage)
    assert head.sms == torch.cuda.get_device_properties(0).multi_processor_count and 0 < head.pairs <= head.sms // 2
    assert head.ticket == head.status + 64 and head.next == head.status + 128
    counter = torch.as_tensor(type("Word", (), {"__cuda_array_interface__": dict(shape=(1,), typestr="<i4", data=(head.next, False), version=3)})(), device="cuda")
    rows, hidden, inner = 2100, 64, 2056                           # 9 x 17 tiles
    assert forward_tiles(rows, inner) > head.pairs
    x, wg, wu = ffn_case(rows, hidden, inner, torch.float16, 1)
    h = torch.zeros((rows, inner), dtype=torch.float16, device="cuda")
    out = (h, inner, None, None, inner)
    call_ffn(aq, stage, x, wg, wu, "silu", out)
    torch.cuda.synchronize()
    want = h.clone()
    assert counter.item() == 0
    tiles = forward_tiles(rows, inner)
    for left in (1, tiles - head.pairs, tiles - head.pairs + 3, tiles - 1, tiles, tiles + 1000):
        counter.fill_(left)
        torch.cuda.synchronize()
        call_ffn(aq, stage, x, wg, wu, "silu", out)
        torch.cuda.synchronize()
        assert counter.item() == 0, left
        h.zero_()
        call_ffn(aq, stage, x, wg, wu, "silu", out)
        torch.cuda.synchronize()
        assert torch.equal(h, want) and counter.item() == 0, left


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rows,hidden,inner,pad", [(2100, 840, 2600, 8), (4000, 64, 1000, 0), (33, 72, 24008, 0), (1025, 200, 5000, 8)])
def test_gated_ffn_of_many_tiles(aq, stage, dtype, rows, hidden, inner, pad):
    """More tiles than the GPU holds pairs: every pair takes several, from the counter, with both halves of its tensor memory."""
    assert forward_tiles(rows, inner) > pairs_at_most()
    set_type(aq, stage, dtype)
    t, u = forms.TYPES[dtype], forms.UNIT[dtype]
    for name in ("silu", "gelu", "gelu_tanh"):
        x, wg, wu = ffn_case(rows, hidden, inner, t, rows + hidden, pad)
        h, g, up = Guarded(rows, inner, t, pad), Guarded(rows, inner, t, pad + 8), Guarded(rows, inner, t, pad + 8)
        call_ffn(aq, stage, x, wg, wu, name, (h.view, h.ld, g.view, up.view, g.ld))
        torch.cuda.synchronize()
        for b in (h, g, up, x, wg, wu):
            b.check()
        x64, g64, u64 = x.view.double(), wg.view.double(), wu.view.double()
        h_want, g_want, u_want = forms.ffn(x64, g64, u64, name)
        e = 4 * math.sqrt(hidden) * 2 * E                          # as in test_gated_ffn
        mg, mu = x64.abs() @ g64.abs().T, x64.abs() @ u64.abs().T
        near(g.view, g_want, u * g_want.abs() + e * mg + forms.TINY[dtype])
        near(up.view, u_want, u * u_want.abs() + e * mu + forms.TINY[dtype])
        near(h.view, h_want, u * h_want.abs() + forms.TINY[dtype] + 1.13 * e * (mg * u_want.abs() + mu * g_want.abs()) + 16 * E * (g_want * u_want).abs())
    assert aq.aq_stage_status(stage) == 0


def near(got, want, tol):
    """within(), on the GPU."""
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


MANY_TILES = [  # several rounds of tiles: with a narrow last column of tiles (1400, 840), a widened one (264, 392), dx in parts (the last three)
    (2100, 1400, 5000, 0), (2100, 840, 2600, 8), (300, 2048, 8192, 0), (1000, 264, 9000, 8), (1500, 392, 4104, 0)]


def ffn_grad_case(rows, hidden, inner, t, seed, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    put = lambda r, c, s=1.0: Guarded(r, c, t, pad).put(s * torch.randn((r, c), generator=gen, device="cuda"))  # noqa: E731
    return [put(rows, inner), put(rows, hidden), put(inner, hidden, hidden ** -0.5), put(inner, hidden, hidden ** -0.5), put(rows, inner), put(rows, inner)]


def call_ffn_grad(aq, st, ops, name, dx, dwg, dwu):
    dh, x, wg, wu, g, u = ops
    rows, hidden = x.view.shape
    aq.aq_gated_ffn_grad(st, dh.view, dh.ld, x.view, x.ld, wg.view, wu.view, wg.ld, g.view, u.view, g.ld, rows, hidden, wg.view.shape[0],
                         act_key(aq, name), dx.view if dx else None, dx.ld if dx else 8, dwg.view if dwg else None, dwu.view if dwu else None, dwg.ld if dwg else 8)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("rows,hidden,inner,pad", MANY_TILES)
def test_gated_ffn_gradient_of_many_tiles(aq, stage, dtype, rows, hidden, inner, pad):
    """Every element of dx and of the weights' gradients, all three outputs at once and apart."""
    assert backward_tiles(rows, hidden, inner) > pairs_at_most()
    set_type(aq, stage, dtype)
    t, u, tiny = forms.TYPES[dtype], forms.UNIT[dtype], forms.TINY[dtype]
    name = ("silu", "gelu", "gelu_tanh")[(rows + hidden) % 3]
    ops = ffn_grad_case(rows, hidden, inner, t, rows + inner, pad)
    dh, x, wg, wu, g, up = (b.view.double() for b in ops)
    dg, du, dx, dwg, dwu = forms.ffn_grad(dh, x, wg, wu, g, up, name)
    eg = u * dg.abs() + tiny + 16 * E * (dh * up).abs() * (1 + g.abs())               # as in test_gated_ffn_gradient
    eu = u * du.abs() + tiny + 16 * E * (dh * g).abs()
    em, er = 4 * math.sqrt(2 * inner) * 2 * E, 4 * math.sqrt(rows) * 2 * E
    dx_tol = u * dx.abs() + tiny + eg @ wg.abs() + eu @ wu.abs() + em * (dg.abs() @ wg.abs() + du.abs() @ wu.abs())
    wg_tol = u * dwg.abs() + tiny + eg.T @ x.abs() + er * (dg.abs().T @ x.abs())
    wu_tol = u * dwu.abs() + tiny + eu.T @ x.abs() + er * (du.abs().T @ x.abs())
    for want_dx, want_dw in ((True, True), (True, False), (False, True)):
        o = [Guarded(r, hidden, t, pad + 8) for r in (rows, inner, inner)]
        call_ffn_grad(aq, stage, ops, name, o[0] if want_dx else None, o[1] if want_dw else None, o[2] if want_dw else None)
        torch.cuda.synchronize()
        for b in ops + o:
            b.check()
        if want_dx:
            near(o[0].view, dx, dx_tol)
        if want_dw:
            near(o[1].view, dwg, wg_tol)
            near(o[2].view, dwu, wu_tol)
    assert aq.aq_stage_status(stage) == 0


def test_two_handles_with_many_tiles_each(aq):
    """Calls of several rounds of tiles on two handles and streams side by side: each takes its tiles from its own counter."""
    rows, hidden, inner = 1500, 392, 4104
    ops = ffn_grad_case(rows, hidden, inner, torch.bfloat16, 3)
    assert backward_tiles(rows, hidden, inner) > pairs_at_most() and forward_tiles(rows, inner) > pairs_at_most()
    sides = []
    for _ in range(2):
        st, stream = aq.aq_stage_create(), torch.cuda.Stream()
        set_type(aq, st, "bf16")
        aq.aq_stage_configure(st, aq.AQ_STREAM, stream.cuda_stream)
        sides.append((st, [Guarded(rows, inner, torch.bfloat16)] + [Guarded(r, hidden, torch.bfloat16) for r in (rows, inner, inner)]))
    torch.cuda.synchronize()

    def calls(st, o):
        call_ffn(aq, st, ops[1], ops[2], ops[3], "gelu", (o[0].view, o[0].ld, None, None, o[0].ld))
        call_ffn_grad(aq, st, ops, "gelu", *o[1:])
    calls(*sides[0])
    torch.cuda.synchronize()
    want = [b.flat.clone() for b in sides[0][1]]
    for _ in range(10):
        for side in sides:
            calls(*side)
    torch.cuda.synchronize()
    for st, o in sides:
        assert aq.aq_stage_status(st) == 0
        for b, w in zip(o, want):
            assert torch.equal(b.flat, w)
        aq.aq_stage_destroy(st)


# ---- the activations over their whole range ----------------------------------------------------------------------------

ACT_RANGE = torch.cat([torch.linspace(-14, 14, 1601), torch.linspace(-100, 100, 401), torch.tensor([-0.0, 1e-4, -1e-4, 1e4, -1e4])])


def exponent_of(name, g):
    """The largest exponent that the form of an activation at g raises e to."""
    return {"silu": g.abs(), "gelu": 0.5 * g * g, "gelu_tanh": 1.6 * g.abs() * (1 + 0.0448 * g * g)}[name]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
def test_activations_relative_to_their_own_size(aq, stage, dtype, name):
    """g and u = 1 through weights that pass them on, so that h = act(g), du = act(g) and dg = act'(g).

    Relative to the value: one rounding of the type; the exponent y of e^y is formed in up to four roundings (a product or two, and
    times log2 e), which cost 4 E |y|, and the rest (polynomial, reciprocal, products) 16 E.  For the derivative, whose two
    terms cancel near its zero, relative to the sum of their magnitudes.  Below: e^-y beyond 2^126 counts as infinite, so
    sigmoids under 2^-125 may be 0, which g (in the derivative, g y') magnifies."""
    set_type(aq, stage, dtype)
    t, u = forms.TYPES[dtype], forms.UNIT[dtype]
    v = ACT_RANGE.to(t)
    n = v.numel()
    g = v.double()
    y = math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)
    x = torch.zeros((n, 16), dtype=t)
    x[:, 0], x[:, 8] = v, 1.0
    wg, wu = torch.zeros((8, 16), dtype=t), torch.zeros((8, 16), dtype=t)
    wg[:, 0], wu[:, 8] = 1.0, 1.0
    few = torch.empty((16, 8), dtype=t, device="cuda")             # the kernel for few rows, too
    h, gg, uu = (torch.empty((n, 8), dtype=t, device="cuda") for _ in range(3))
    args = (16, wg.cuda(), wu.cuda(), 16)
    aq.aq_gated_ffn(stage, x.cuda(), *args, n, 16, 8, act_key(aq, name), h, 8, gg, uu, 8)
    aq.aq_gated_ffn(stage, x[:1600:100].contiguous().cuda(), *args, 16, 16, 8, act_key(aq, name), few, 8, None, None, 8)
    # sigma or Phi, never as one minus something, and what multiplies g in the derivative
    over, bend = {"silu": lambda: (torch.sigmoid(g), torch.sigmoid(g) * torch.sigmoid(-g)),
                  "gelu": lambda: (0.5 * torch.erfc(-g / math.sqrt(2.0)), torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)),
                  "gelu_tanh": lambda: (torch.sigmoid(y), torch.sigmoid(y) * torch.sigmoid(-y) * math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * g * g))}[name]()
    value, slope = g * over, over + g * bend
    rough = 16 * E + 4 * E * exponent_of(name, g)
    floor = forms.TINY[dtype] + 2.0 ** -125 * (1 + g.abs())
    tol = (u * value.abs() + rough.clamp(max=1.0) * value.abs() + floor)[:, None].expand(n, 8)
    within(h, value[:, None].expand(n, 8), tol)
    within(few, value[:1600:100, None].expand(16, 8), tol[:1600:100])
    # dx = dg wg + du wu with wg, wu the two halves of an identity, dh = u = 1
    one = torch.ones((n, 8), dtype=t, device="cuda")
    wg, wu, zero = torch.zeros((8, 16), dtype=t), torch.zeros((8, 16), dtype=t), torch.zeros((8, 16), dtype=t, device="cuda")
    wg[:, :8], wu[:, 8:] = torch.eye(8), torch.eye(8)
    dx = torch.empty((n, 16), dtype=t, device="cuda")
    aq.aq_gated_ffn_grad(stage, one, 8, x.cuda(), 16, wg.cuda(), wu.cuda(), 16, gg, one, 8, n, 16, 8, act_key(aq, name), dx, 16, None, None, 16)
    size, steep = over + (g * bend).abs(), 1.6 * (1 + 0.135 * g * g) if name == "gelu_tanh" else torch.ones_like(g)
    slope_tol = u * slope.abs() + rough.clamp(max=1.0) * size + forms.TINY[dtype] + 2.0 ** -125 * (1 + (g * steep).abs())
    within(dx[:, :8], slope[:, None].expand(n, 8), slope_tol[:, None].expand(n, 8))
    within(dx[:, 8:], value[:, None].expand(n, 8), tol)


# ---- log probabilities far from zero, and with extreme scales -----------------------------------------------------------

@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(3, 700), (2, 9001), (90, 9001)])
@pytest.mark.parametrize("scale", [1e34, 3e38])
def test_logprobs_with_a_very_large_scale(aq, stage, dtype, rows, vocab, scale):
    """1 / temperature near the end of binary32: nothing but the largest logits is left, whatever is masked."""
    set_type(aq, stage, dtype)
    x = torch.zeros((rows, vocab))
    x[:, ::3] = -math.inf
    x[:, 1::3] = -2.0
    x[1] = torch.where(torch.arange(vocab) < 5, 0.0, -math.inf)
    x = x.to(forms.TYPES[dtype])
    targets = torch.full((rows,), 2, dtype=torch.int32)
    buf, out = Guarded(rows, vocab, forms.TYPES[dtype]).put(x), Guarded(rows, vocab, forms.TYPES[dtype])
    got = run_logprobs(aq, stage, buf, targets, scale, 4)
    check_logprobs(x.double(), targets, scale, 4, got)
    gl = torch.full((rows,), 1 / scale)
    run_logprobs_grad(aq, stage, buf, out, targets.cuda(), scale, got[2].float().cuda(), got[1].float().cuda(), gl.cuda(), gl.cuda())
    s32, l32 = (torch.tensor(v, dtype=torch.float32).double().item() for v in (scale, 1 / scale))
    for r in (0, 1, rows - 1):
        want = forms.logprobs_grad(x[r].double(), 2, s32, l32, l32)
        within(out.view[r], want, forms.UNIT[dtype] * want.abs() + forms.TINY[dtype] + 1e-4 * want.abs() + 1e-5)


@pytest.mark.parametrize("dtype,offset,scale", [("fp16", 7000.0, 1.0), ("fp16", -30000.0, 0.25), ("bf16", 20000.0, 0.25), ("fp32", 5000.0, 1.0), ("fp32", -1e6, 1.0),
                                                ("fp32", 1e30, 2.0 ** -75)])
@pytest.mark.parametrize("rows,vocab", [(3, 700), (2, 30011)])
def test_logprobs_gradient_of_far_rows(aq, stage, dtype, offset, scale, rows, vocab):
    """Rows whose logits lie far from zero, where lse has no digits left for ln p, with a distribution under the offset: steps of
    the type there (0.5 at least), some masked; beside a row that is near zero.

    The gradient forms the row's sum again relative to its largest logit, so p is good to the sum's 2e-5 and 4 E of the distance;
    only the entropy, an input, and the output's rounding come on top."""
    set_type(aq, stage, dtype)
    t = forms.TYPES[dtype]
    gen = torch.Generator().manual_seed(vocab)
    step = 2.0 ** (math.floor(math.log2(abs(offset))) - {"fp16": 10, "bf16": 7, "fp32": 23}[dtype])
    unit = max(step, 0.5)
    x = offset - unit * torch.randint(0, 7, (rows, vocab), generator=gen, dtype=F64)
    x[torch.rand((rows, vocab), generator=gen) < 0.1] = -math.inf
    x[-1] = 3 * torch.randn(vocab, generator=gen, dtype=F64)
    x[:, vocab // 3] = torch.where(torch.isfinite(x[:, vocab // 3]), x[:, vocab // 3], offset)
    x = x.to(t)
    targets = torch.full((rows,), vocab // 3, dtype=torch.int32)
    s32 = torch.tensor(scale, dtype=torch.float32).double().item()
    assert abs(x[0].double().max().item() * s32) > 4096
    buf, out = Guarded(rows, vocab, t, 3, 1).put(x), Guarded(rows, vocab, t, 3, 1)
    lp, h, lse, _, _ = run_logprobs(aq, stage, buf, targets, scale, 0)
    gl, gh = torch.randn(rows, generator=gen), torch.randn(rows, generator=gen)
    run_logprobs_grad(aq, stage, buf, out, targets.cuda(), scale, lse.float().cuda(), h.float().cuda(), gl.cuda(), gh.cuda())
    out.check()
    for r in range(rows):
        z = x[r].double() * s32
        want = forms.logprobs_grad(x[r].double(), int(targets[r]), s32, gl[r].item(), gh[r].item())
        p = torch.softmax(z, 0)
        below = torch.where(p > 0, torch.log_softmax(z, 0), torch.zeros_like(z))
        hh = -(p * below).sum()
        size = s32 * p * (abs(gl[r].item()) + abs(gh[r].item()) * (below.abs() + hh))
        near_zero = 2 * E * (z[p > 0].abs().max() + abs(lse[r].item())) if abs(lse[r].item()) < 4096 else 0.0      # lse's own digits
        size[int(targets[r])] += s32 * abs(gl[r].item())
        tol = forms.UNIT[dtype] * want.abs() + forms.TINY[dtype] + size * (6e-5 + E * (8 + 4 * below.abs()) + near_zero) + s32 * 4e-5 * abs(gh[r].item()) * p
        within(out.view[r], want, tol)


# ---- several host threads ---------------------------------------------------------------------------------------------------

def test_host_threads_with_a_handle_each():
    """Four threads make their handles and call side by side, in a process of its own so that their first calls are the library's first."""
    import os
    import subprocess
    import sys
    code = """
import threading, torch
import paper_2206_01299_b200 as aq
rows, hidden, inner = 300, 136, 520
g = torch.Generator(device="cuda").manual_seed(1)
x, wg, wu, dh = (torch.randn(s, generator=g, device="cuda").half() for s in ((rows, hidden), (inner, hidden), (inner, hidden), (rows, inner)))
torch.cuda.synchronize()
outs, errors, ready = [None] * 4, [], threading.Barrier(4)
def work(i):
    try:
        st, stream = aq.aq_stage_create(), torch.cuda.Stream()
        aq.aq_stage_configure(st, aq.AQ_STREAM, stream.cuda_stream)
        with torch.cuda.stream(stream):
            h, g, u = (torch.empty_like(dh) for _ in range(3))
            d = [torch.empty_like(v) for v in (x, wg, wu)]
        stream.synchronize()
        ready.wait()
        for _ in range(10):
            aq.aq_gated_ffn(st, x, hidden, wg, wu, hidden, rows, hidden, inner, aq.AQ_ACT_GELU, h, inner, g, u, inner)
            aq.aq_gated_ffn_grad(st, dh, inner, x, hidden, wg, wu, hidden, g, u, inner, rows, hidden, inner, aq.AQ_ACT_GELU, d[0], hidden, d[1], d[2], hidden)
        assert aq.aq_stage_status(st) == 0
        aq.aq_stage_destroy(st)
        outs[i] = [h, g, u] + d
    except Exception as e:
        errors.append(e)
threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
[t.start() for t in threads]
[t.join() for t in threads]
assert not errors, errors
assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(o, outs[0])) and torch.isfinite(outs[0][0]).all()
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
