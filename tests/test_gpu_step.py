"""Layer norm, the gradients' norm and the optimizer's step on the GPU against plain 64-bit forms (step_forms.py).

Tolerances.  u is one rounding to the output type, e = 2^-24 one binary32 rounding.
* A sum in binary32 of a row: a thread adds at most 64 terms one by one, then trees of at most 13 steps: 80 e of the sum of
  magnitudes.  The mean is off by dm = 80 e mean|s|.
* rstd: the differences are off by dm and a rounding, the squares by two more and the sum by 80 e; dm enters the variance as its
  square alone, since the differences add up to nothing.  With the root half of it: (45 e + (dm rstd)^2) rstd; 60 for the roundings of
  the root and quotient.
* y: |w| rstd (dm + e |s - mean|) + |w n| (the error of rstd + 3 e) + e |y|, and u |y|.
* dx, from the given mean and rstd: 3 e |n| an element; sums of 80 e.
* dw, db: a thread adds at most rows one by one, with the grids used here at most 300, then trees and up to 150 CTAs' sums: 470 e of
  the sum of magnitudes (or rows + 170).
* Moments are the same operations in binary32 and have to be the same bits; stored in 8 bits too.
* A step: m / (sqrt(v / c2) + eps) with the approximate root and quotient, 2^-22 each, and at most eight roundings: 24 e.
"""
import math

import pytest
import torch

from tests import step_forms as forms
from tests.stage_forms import TINY, TYPES, UNIT
from tests.test_gpu_stage import E, Guarded, set_type

pytestmark = pytest.mark.gpu
F64, F32 = torch.float64, torch.float32


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


def same(a, b):
    """The same bits, NaN among them."""
    return torch.equal(a.cpu().contiguous().view(torch.uint8), b.cpu().contiguous().view(torch.uint8))


def rounding(dtype, y):
    return UNIT[dtype] * y.abs() + TINY[dtype]


def close(have, want, tol, what):
    have, want = have.double().cpu(), want.double().cpu()
    bad = ~((have - want).abs() <= tol) & ~(have == want) & ~(have.isnan() & want.isnan())
    assert not bool(bad.any()), (what, int(bad.sum()), (have - want).abs()[bad][:4].tolist(), want[bad][:4].tolist())


# ---- layer norm ----------------------------------------------------------------------------------------------

WIDTHS = [1, 2, 3, 7, 8, 16, 40, 64, 65, 255, 256, 257, 264, 512, 520, 768, 1000, 1021, 1024, 1025, 1600, 2048, 2056, 4096, 4097, 8192, 8193, 8200,
          12000, 16384, 33000, 40001]


def norm_inputs(rows, d, dtype, seed=0, offset=0.0):
    g = torch.Generator().manual_seed(rows * 100003 + d + seed)
    t = TYPES[dtype]
    x = (torch.randn((rows, d), generator=g) + offset).to(t)
    r = (2 * torch.randn((rows, d), generator=g)).to(t)
    w, b = (1 + 0.3 * torch.randn(d, generator=g)).to(t), (0.2 * torch.randn(d, generator=g)).to(t)
    dy, dsum = torch.randn((rows, d), generator=g).to(t), torch.randn((rows, d), generator=g).to(t)
    return x, r, w, b, dy, dsum


def check_norm(dtype, s, w, b, eps, y, mean, rstd):
    """s, w, b: the stored values; the rest as the kernel left it."""
    s, w, b = (v.double().cpu() for v in (s, w, b))
    y64, mean64, rstd64 = forms.layer_norm(s, w, b, eps)
    dm = 80 * E * s.abs().mean(1) + 1e-45
    dr = (60 * E + (dm * rstd64) ** 2) * rstd64
    close(mean, mean64, dm, "mean")
    close(rstd, rstd64, dr, "rstd")
    n, dm, dr, r = (s - mean64[:, None]), dm[:, None], dr[:, None], rstd64[:, None]
    tol = w.abs() * (r * (dm + E * n.abs()) + n.abs() * dr + 3 * E * (n * r).abs()) + E * (y64.abs() + b.abs()) + rounding(dtype, y64)
    close(y, y64, tol, "y")


def run_norm(aq, st, dtype, x, r, w, b, eps, pad=0, offset=0, keep=True, offset_y=None):
    """With guarded buffers; (s, y, mean, rstd)."""
    rows, d = x.shape
    t = TYPES[dtype]
    bx, by = Guarded(rows, d, t, pad, offset).put(x), Guarded(rows, d, t, pad, offset if offset_y is None else offset_y)
    br = None if r is None else Guarded(rows, d, t, pad, offset).put(r)
    bs = Guarded(rows, d, t, pad, offset) if r is not None and keep else None
    mean, rstd = torch.zeros(rows + 8, device="cuda"), torch.zeros(rows + 8, device="cuda")
    aq.aq_layer_norm(st, bx.view, bx.ld, br and br.view, br.ld if br else 0, w if w is None else w.cuda(), b if b is None else b.cuda(), eps, rows, d,
                     bs and bs.view, bs.ld if bs else 0, by.view, by.ld, mean, rstd)
    torch.cuda.synchronize()
    for buf in (bx, by, br, bs):
        if buf is not None:
            buf.check()
    assert not mean[rows:].any() and not rstd[rows:].any()
    assert same(bx.view, x)
    s = x if r is None else (x.float() + r.float()).to(t)
    if bs:
        assert same(bs.view, s)
    return s, by.view.clone(), mean[:rows], rstd[:rows]


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm(aq, stage, dtype, d):
    set_type(aq, stage, dtype)
    for rows, pad, offset, residual, keep in ((1, 0, 0, False, True), (5, 0, 0, True, True), (3, 8, 8, True, False), (6, 1, 3, True, True)):
        x, r, w, b, _, _ = norm_inputs(rows, d, dtype)
        s, y, mean, rstd = run_norm(aq, stage, dtype, x, r if residual else None, w, b, 1e-5, pad, offset, keep)
        check_norm(dtype, s, w, b, 1e-5, y, mean, rstd)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm_rows_off_the_boundaries(aq, stage, dtype, d):
    """Rows that begin anywhere in 16 bytes, in all operands alike or not, weights too."""
    set_type(aq, stage, dtype)
    for rows, pad, offset, offset_y in ((9, 0, 0, 0), (9, 3, 0, 0), (9, 2, 1, 1), (9, 4, 5, 5), (5, 1, 0, 1), (5, 8, 2, 0)):
        x, r, w, b, _, _ = norm_inputs(rows, d, dtype, seed=pad)
        wide = torch.zeros(d + 3, dtype=TYPES[dtype], device="cuda")
        wide[3:] = w.cuda()
        s, y, mean, rstd = run_norm(aq, stage, dtype, x, r, wide[3:], b, 1e-5, pad, offset, True, offset_y)
        check_norm(dtype, s, w, b, 1e-5, y, mean, rstd)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,d", [(1000, 768), (700, 1021), (4096, 24), (300, 5000), (150, 12000)])
def test_layer_norm_many_rows_without_weights(aq, stage, dtype, rows, d):
    set_type(aq, stage, dtype)
    x, r, _, _, _, _ = norm_inputs(rows, d, dtype)
    one, zero = torch.ones(d), torch.zeros(d)
    s, y, mean, rstd = run_norm(aq, stage, dtype, x, r, None, None, 1e-6)
    check_norm(dtype, s, one, zero, 1e-6, y, mean, rstd)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("d", [96, 1600, 1021, 9000, 40001])
def test_layer_norm_rows_far_from_zero(aq, stage, dtype, d):
    """Mean 500 deviations out: a variance from the mean of squares would have lost 18 of 24 bits."""
    set_type(aq, stage, dtype)
    x, _, w, b, _, _ = norm_inputs(4, d, dtype, offset=500.0)
    s, y, mean, rstd = run_norm(aq, stage, dtype, x, None, w, b, 1e-5)
    check_norm(dtype, s, w, b, 1e-5, y, mean, rstd)


@pytest.mark.parametrize("d", [64, 1600, 1021, 5000, 40001])
def test_layer_norm_equal_values_and_rows_that_are_not_finite(aq, stage, d):
    set_type(aq, stage, "bf16")
    x, r, w, b, _, _ = norm_inputs(6, d, "bf16")
    x[1] = 3.0
    x[2, d // 2] = math.nan
    x[4, d - 1] = math.inf
    _, y, mean, rstd = run_norm(aq, stage, "bf16", x, None, w, b, 1e-5)
    assert torch.equal(y[1].cpu(), b) and mean[1] == 3 and abs(rstd[1].item() / 1e-5 ** -0.5 - 1) < 1e-6
    assert bool(y[2].isnan().all()) and bool(y[4].isnan().all())
    keep = torch.tensor([0, 3, 5])
    check_norm("bf16", x[keep], w, b, 1e-5, y[keep.cuda()], mean[keep.cuda()], rstd[keep.cuda()])


def run_norm_grad(aq, st, dtype, dy, dsum, s, w, mean, rstd, pad=0, offset=0, sums=True, dx=True):
    rows, d = s.shape
    t = TYPES[dtype]
    bufs = [None if v is None else Guarded(rows, d, t, pad, offset).put(v) for v in (dy, dsum, s)]
    out = Guarded(rows, d, t, pad, offset) if dx else None
    dw, db = (torch.full((d + 4,), 9.0, device="cuda") for _ in range(2)) if sums else (None, None)
    aq.aq_layer_norm_grad(st, bufs[0].view, bufs[0].ld, bufs[1] and bufs[1].view, bufs[1].ld if bufs[1] else 0, bufs[2].view, bufs[2].ld,
                          None if w is None else w.cuda(), mean.cuda(), rstd.cuda(), rows, d, out and out.view, out.ld if out else 0, dw, db)
    torch.cuda.synchronize()
    for buf in bufs + [out]:
        if buf is not None:
            buf.check()
    if sums:
        assert bool((dw[d:] == 9).all()) and bool((db[d:] == 9).all())
        dw, db = dw[:d], db[:d]
    return out and out.view.clone(), dw, db


def check_norm_grad(dtype, dy, dsum, s, w, mean, rstd, got):
    dy, s, w, mean, rstd = (v.double().cpu() for v in (dy, s, w, mean, rstd))
    dsum = None if dsum is None else dsum.double().cpu()
    want = forms.layer_norm_grad(dy, dsum, s, w, mean, rstd)
    n, g, r = (s - mean[:, None]) * rstd[:, None], dy * w, rstd[:, None]
    if got[0] is not None:
        c1, c2 = g.mean(1, keepdim=True).abs(), (g * n).mean(1, keepdim=True).abs()
        tol = r * (84 * E * g.abs().mean(1, keepdim=True) + n.abs() * 90 * E * (g * n).abs().mean(1, keepdim=True) + 6 * E * (g.abs() + c1 + n.abs() * c2))
        if dsum is not None:
            tol = tol + E * (dsum.abs() + (want[0] - dsum).abs())
        close(got[0], want[0], tol + rounding(dtype, want[0]), "dx")
    k = (min(s.shape[0], 300) + 170) * E
    if got[1] is not None:
        close(got[1], want[1], k * (dy * n).abs().sum(0) + 1e-40, "dw")
        close(got[2], want[2], k * dy.abs().sum(0) + 1e-40, "db")


def statistics(s, eps=1e-5):
    _, mean, rstd = forms.layer_norm(s.double(), 1.0, 0.0, eps)
    return mean.float(), rstd.float()


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm_grad(aq, stage, dtype, d):
    set_type(aq, stage, dtype)
    for rows, pad, offset, skip in ((1, 0, 0, False), (5, 0, 0, True), (37, 8, 8, True), (6, 1, 3, True), (41, 3, 0, True), (23, 1, 0, False), (19, 2, 0, True)):
        s, _, w, _, dy, dsum = norm_inputs(rows, d, dtype, seed=1)
        mean, rstd = statistics(s)
        got = run_norm_grad(aq, stage, dtype, dy, dsum if skip else None, s, w, mean, rstd, pad, offset)
        check_norm_grad(dtype, dy, dsum if skip else None, s, w, mean, rstd, got)


@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,d,pad", [(5000, 768, 0), (3001, 1600, 0), (3001, 1600, 4), (2000, 1021, 0), (2000, 1021, 3), (20011, 24, 0), (20011, 24, 1), (700, 5000, 0),
                                        (700, 5001, 1), (301, 12000, 0), (9000, 3, 0), (1500, 250, 1), (1500, 2045, 0), (900, 8190, 0), (1200, 8201, 7), (300, 12001, 0), (5000, 8200, 0)])
def test_layer_norm_grad_many_rows(aq, stage, dtype, rows, d, pad):
    set_type(aq, stage, dtype)
    s, _, w, _, dy, dsum = norm_inputs(rows, d, dtype, seed=2)
    mean, rstd = statistics(s)
    got = run_norm_grad(aq, stage, dtype, dy, dsum, s, w, mean, rstd, pad)
    check_norm_grad(dtype, dy, dsum, s, w, mean, rstd, got)
    again = run_norm_grad(aq, stage, dtype, dy, dsum, s, w, mean, rstd, pad)
    assert all(torch.equal(a, b) for a, b in zip(got, again))               # the same bits


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d,pad", [(30, 1), (64, 3), (1021, 0), (1021, 3), (1600, 5), (4099, 0), (9001, 2)])
def test_layer_norm_grad_next_to_rows_and_padding_that_are_not_finite(aq, stage, dtype, d, pad):
    """A row of NaN makes its own dx NaN and dw, db; without it in them the others are as if it were not there; padding counts for nothing."""
    set_type(aq, stage, dtype)
    rows, t = 21, TYPES[dtype]
    s, _, w, _, dy, dsum = norm_inputs(rows, d, dtype, seed=6)
    mean, rstd = statistics(s)
    bufs = []
    for v in (dy, dsum, s):
        buf = torch.full((rows, d + pad), math.nan, dtype=t, device="cuda")
        buf[:, :d] = v.cuda()
        bufs.append(buf)
    out, ld = torch.zeros((rows, d + pad), dtype=t, device="cuda"), d + pad
    dw, db = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    call = lambda: aq.aq_layer_norm_grad(stage, bufs[0], ld, bufs[1], ld, bufs[2], ld, w.cuda(), mean.cuda(), rstd.cuda(), rows, d, out, ld, dw, db)  # noqa: E731
    call()
    check_norm_grad(dtype, dy, dsum, s, w, mean, rstd, (out[:, :d], dw, db))
    assert not out[:, d:].any()
    bufs[0][7, :d] = math.nan
    call()
    keep = [r for r in range(rows) if r != 7]
    assert bool(out[7, :d].isnan().all()) and bool(dw.isnan().all()) and bool(db.isnan().all())
    check_norm_grad(dtype, dy[keep], dsum[keep], s[keep], w, mean[keep], rstd[keep], (out[keep, :d], None, None))


@pytest.mark.parametrize("d", [64, 1600, 1021])
def test_layer_norm_grad_parts_of_the_outputs(aq, stage, d):
    set_type(aq, stage, "fp16")
    s, _, w, _, dy, dsum = norm_inputs(333, d, "fp16", seed=3)
    mean, rstd = statistics(s)
    whole = run_norm_grad(aq, stage, "fp16", dy, dsum, s, w, mean, rstd)
    dx, _, _ = run_norm_grad(aq, stage, "fp16", dy, dsum, s, w, mean, rstd, sums=False)
    _, dw, db = run_norm_grad(aq, stage, "fp16", dy, dsum, s, w, mean, rstd, dx=False)
    assert torch.equal(dx, whole[0]) and torch.equal(dw, whole[1]) and torch.equal(db, whole[2])
    only = torch.zeros(d, device="cuda")
    for at in (1, 2):
        args = [None, None]
        args[at - 1] = only
        aq.aq_layer_norm_grad(stage, dy.cuda(), d, None, 0, s.cuda(), d, w.cuda(), mean.cuda(), rstd.cuda(), 333, d, None, 0, *args)
        assert torch.equal(only, whole[at])
    got = run_norm_grad(aq, stage, "fp16", dy, None, s, None, mean, rstd)
    check_norm_grad("fp16", dy, None, s, torch.ones(d), mean, rstd, got)


@pytest.mark.parametrize("d", [64, 1600, 1021, 9000])
def test_layer_norm_without_rows(aq, stage, d):
    set_type(aq, stage, "bf16")
    dw, db = torch.full((d,), 5.0, device="cuda"), torch.full((d,), 5.0, device="cuda")
    aq.aq_layer_norm(stage, None, d, None, d, None, None, 1e-5, 0, d, None, d, None, d, None, None)
    aq.aq_layer_norm_grad(stage, None, d, None, d, None, d, None, None, None, 0, d, None, d, dw, db)
    torch.cuda.synchronize()
    assert not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,d", [(40, 64), (600, 1600), (77, 1021), (13, 9000), (5, 40001)])
def test_layer_norm_in_place(aq, stage, dtype, rows, d):
    set_type(aq, stage, dtype)
    x, r, w, b, dy, dsum = (v.cuda() for v in norm_inputs(rows, d, dtype, seed=4))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")

    def norm(x, r, s, y):
        aq.aq_layer_norm(stage, x, d, r, d, w, b, 1e-5, rows, d, s, d, y, d, mean, rstd)
        return s, y
    s, y = norm(x, r, torch.empty_like(x), torch.empty_like(x))
    x1, r1 = x.clone(), r.clone()
    assert all(torch.equal(p, q) for p, q in zip(norm(x1, r1, r1, x1), (s, y)))          # the stream takes the sum, the branch the norm
    x1, r1 = x.clone(), r.clone()
    assert all(torch.equal(p, q) for p, q in zip(norm(x1, r1, x1, r1), (s, y)))
    x1 = x.clone()
    want = norm(x, None, None, torch.empty_like(x))[1]
    assert torch.equal(norm(x1, None, None, x1)[1], want)

    norm(x, r, s, y)
    dw, db, dw1, db1 = (torch.empty(d, device="cuda") for _ in range(4))
    dx = torch.empty_like(x)
    aq.aq_layer_norm_grad(stage, dy, d, dsum, d, s, d, w, mean, rstd, rows, d, dx, d, dw, db)
    for name in ("dy", "dsum", "s"):
        a = {"dy": dy.clone(), "dsum": dsum.clone(), "s": s.clone()}
        aq.aq_layer_norm_grad(stage, a["dy"], d, a["dsum"], d, a["s"], d, w, mean, rstd, rows, d, a[name], d, dw1, db1)
        assert torch.equal(a[name], dx) and torch.equal(dw, dw1) and torch.equal(db, db1), name


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_layer_norm_of_the_widest_rows(aq, stage, dtype):
    set_type(aq, stage, dtype)
    x, r, w, b, dy, dsum = norm_inputs(2, 2 ** 20, dtype, seed=7)
    s, y, mean, rstd = run_norm(aq, stage, dtype, x, r, w, b, 1e-5)
    check_norm(dtype, s, w, b, 1e-5, y, mean, rstd)
    mean, rstd = statistics(s)
    check_norm_grad(dtype, dy, dsum, s, w, mean, rstd, run_norm_grad(aq, stage, dtype, dy, dsum, s, w, mean, rstd))


def test_layer_norm_grad_of_many_rows_that_begin_anywhere(aq, stage):
    set_type(aq, stage, "fp32")
    s, _, w, _, dy, dsum = norm_inputs(300000, 5, "fp32", seed=8)
    mean, rstd = statistics(s)
    check_norm_grad("fp32", dy, dsum, s, w, mean, rstd, run_norm_grad(aq, stage, "fp32", dy, dsum, s, w, mean, rstd, 0, 3))


def test_layer_norm_grad_against_differences(aq, stage):
    """The kernels' own forward pass moved along a direction, in binary32: the slope of sum(dy y) + sum(dsum s).  With h = 2^-7 the difference
    is off by h^2 / 6 of the third derivative (a few times the sum: 1e-4) and the roundings of y, 1e-7 |y| / h."""
    set_type(aq, stage, "fp32")
    for rows, d in ((9, 32), (7, 1021), (5, 1600)):
        s, _, w, b, dy, dsum = norm_inputs(rows, d, "fp32", seed=5)
        mean, rstd = statistics(s)
        got = run_norm_grad(aq, stage, "fp32", dy, dsum, s, w, mean, rstd)
        g = torch.Generator().manual_seed(d)
        h = 2.0 ** -7

        def f(s, w, b):
            y = run_norm(aq, stage, "fp32", s, None, w, b, 1e-5)[1]
            return ((y.cpu().double() * dy.double()).sum() + (s.double() * dsum.double()).sum()).item()
        args = [s, w, b]
        for i, grad in enumerate(got):
            v = torch.randn(args[i].shape, generator=g)
            at = lambda t: f(*[a + t * v if j == i else a for j, a in enumerate(args)])  # noqa: E731
            slope, want = (at(h) - at(-h)) / (2 * h), (grad.cpu().double() * v.double()).sum().item()
            size = (grad.cpu().double() * v.double()).norm().item() + dy.double().norm().item()
            assert abs(slope - want) < 2e-3 * size, (rows, d, i, slope, want)


def test_layer_norm_beyond_32_bit_offsets(aq, stage):
    """2.2e9 elements; the last rows, and a few in between."""
    set_type(aq, stage, "bf16")
    rows, d = 1375000, 1600
    x = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, 125000):
        x[r:r + 125000] = torch.randn((125000, d), device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    w, b = torch.full((d,), 1.5, device="cuda").bfloat16(), torch.full((d,), 0.25, device="cuda").bfloat16()
    aq.aq_layer_norm(stage, x, d, None, 0, w, b, 1e-5, rows, d, None, 0, y, d, mean, rstd)
    at = torch.tensor([0, 1342177, 1342178, rows - 2, rows - 1], device="cuda")
    check_norm("bf16", x[at], w, b, 1e-5, y[at], mean[at], rstd[at])
    dw, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dx = torch.empty_like(x)
    aq.aq_layer_norm_grad(stage, y, d, None, 0, x, d, w, mean, rstd, rows, d, dx, d, dw, db)
    check_norm_grad("bf16", y[at], None, x[at], w, mean[at], rstd[at], (dx[at], None, None))
    want = sum(y[r:r + 125000].sum(0, dtype=torch.float64) for r in range(0, rows, 125000))
    size = sum(y[r:r + 125000].abs().sum(0, dtype=torch.float64) for r in range(0, rows, 125000))
    close(db, want, (8000 * E * size).cpu(), "db")                            # 1375000 / 296 CTAs rows one by one, and what follows


# ---- the gradients' norm -------------------------------------------------------------------------------------

SIZES = [1, 5, 0, 255, 256, 257, 2047, 2048, 2049, 100003, 8, 64]


def laid_out(sizes, dtype, shift=0, fill=None):
    """Tensors behind one another in a guarded buffer (with `shift` elements between them, which no call may change)."""
    n = sum(sizes) + (len(sizes) + 1) * shift
    buf = torch.empty(n, dtype=dtype, device="cuda")
    if dtype.itemsize == 1:
        buf.view(torch.uint8).fill_(0x33)
    else:
        buf.fill_(-7.0)
    parts, at = [], shift
    for i, k in enumerate(sizes):
        parts.append(buf[at:at + k])
        if fill is not None:
            parts[-1].copy_(fill[i])
        at += k + shift
    return buf, parts


def aligned(sizes, dtype, fill=None):
    parts = [torch.zeros(k, dtype=dtype, device="cuda") for k in sizes]
    for p, f in zip(parts, fill or []):
        p.copy_(f)
    return parts


def gradients(sizes, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [scale * torch.randn(k, generator=g) * torch.exp(torch.randn(k, generator=g)) for k in sizes]


@pytest.mark.parametrize("dtype,grads", [("fp16", "fp16"), ("fp16", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("copies", [1, 40])
def test_grad_norm(aq, stage, dtype, grads, packed, copies):
    set_type(aq, stage, dtype)
    sizes = SIZES * copies if copies == 1 else [k % 5000 for k in SIZES] * copies       # 480 tensors: more than one launch takes
    values = [v.to(TYPES[grads]) for v in gradients(sizes, 7)]
    parts = laid_out(sizes, TYPES[grads], 1, values)[1] if packed else aligned(sizes, TYPES[grads], values)
    table = aq.aq_adam_table(stage, grads=parts)
    norm, factor, step = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.tensor([41], device="cuda")
    for inv_scale, limit in ((1.0, 1.0), (1 / 1024, 0.5), (0.25, 0.0), (1.0, math.inf), (1.0, 1e9)):
        aq.aq_grad_norm(stage, table, len(sizes), inv_scale, limit, norm, factor, step)
        want = forms.clip(values, inv_scale, 0.0 if limit == math.inf else limit)
        # eight squares in binary32: 9 e of the sum, halved by the root, and the roundings of the outputs
        assert abs(norm.item() / want[0] - 1) < 6 * E and abs(factor.item() / want[1] - 1) < 7 * E
    assert step.item() == 46
    again = torch.zeros(1, device="cuda")
    aq.aq_grad_norm(stage, table, len(sizes), 1.0, 1e9, again, None, None)
    assert torch.equal(again, norm)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("at", [0, 4, 9, 11])
def test_grad_norm_that_is_not_finite(aq, stage, bad, at):
    set_type(aq, stage, "bf16")
    sizes = [k or 3 for k in SIZES]
    values = [v.bfloat16() for v in gradients(sizes, 8)]
    values[at][-1] = bad
    parts = aligned(sizes, torch.bfloat16, values)
    norm, factor, step = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.tensor([3], device="cuda")
    aq.aq_grad_norm(stage, aq.aq_adam_table(stage, grads=parts), len(sizes), 1.0, 1.0, norm, factor, step)
    assert not math.isfinite(norm.item()) and math.isnan(factor.item()) and step.item() == 3
    values[at][-1] = 1.0
    parts[at][-1] = 1.0
    aq.aq_grad_norm(stage, aq.aq_adam_table(stage, grads=parts), len(sizes), 1.0, 1.0, norm, factor, step)
    assert abs(norm.item() / forms.clip(values, 1.0, 1.0)[0] - 1) < 6 * E and step.item() == 4


@pytest.mark.parametrize("n", [0, 1, 3])
def test_grad_norm_of_nothing(aq, stage, n):
    set_type(aq, stage, "fp32")
    table = aq.aq_adam_table(stage, grads=[torch.empty(0, device="cuda") for _ in range(n)])
    norm, factor, step = torch.ones(1, device="cuda"), torch.zeros(1, device="cuda"), torch.tensor([0], device="cuda")
    aq.aq_grad_norm(stage, table, n, 0.5, 1.0, norm, factor, step)
    assert norm.item() == 0 and factor.item() == 0.5 and step.item() == 1


# ---- the optimizer's step ------------------------------------------------------------------------------------

class Set:
    """Tensors of a step with their state, on the GPU, and the same on the CPU for the plain form."""

    def __init__(self, sizes, dtype, grads, bits, master, packed, seed=11, decay=0.01):
        self.sizes, self.dtype, self.bits, self.grads_type = sizes, dtype, bits, grads
        t = TYPES[dtype]
        g = torch.Generator().manual_seed(seed)
        r = lambda scale: [scale * torch.randn(k, generator=g) for k in sizes]  # noqa: E731
        wide = r(0.5)
        self.decay = [decay * (i % 3) for i in range(len(sizes))]
        place = (lambda name, d, fill: self._keep(name, *laid_out(sizes, d, 1, fill))) if packed else (lambda name, d, fill: aligned(sizes, d, fill))
        self.buffers = {}
        self.master = place("master", F32, wide) if master else None
        self.param = place("param", t, [w.to(t) for w in wide])
        self.grad = place("grad", TYPES[grads], [v.to(TYPES[grads]) for v in gradients(sizes, seed + 1, 0.01)])
        m, v = r(0.003), [x.square() + 1e-9 for x in r(0.01)]
        self.m_scale = self.v_scale = None
        if bits == 32:
            self.m, self.v = place("m", F32, m), place("v", F32, v)
        else:
            self.m = place("m", torch.float8_e4m3fn, [torch.zeros(k).to(torch.float8_e4m3fn) for k in sizes])
            self.v = place("v", torch.float8_e5m2, [torch.zeros(k).to(torch.float8_e5m2) for k in sizes])
            blocks = [-(-k // 256) for k in sizes]
            self.m_scale, self.v_scale = ([torch.zeros(b, device="cuda") for b in blocks] for _ in range(2))
            for i, k in enumerate(sizes):
                for name, x, kind in (("m", m[i], "e4m3"), ("v", v[i], "e5m2")):
                    if k:
                        z, scale = forms.store8(x, torch.zeros(k, dtype=F64), kind)
                        getattr(self, name)[i].copy_(z.float().to(getattr(self, name)[i].dtype))
                        getattr(self, name + "_scale")[i].copy_(scale)

    def _keep(self, name, buf, parts):
        self.buffers[name] = (buf, parts)
        return parts

    def check_between(self):
        for name, (buf, parts) in self.buffers.items():
            for p in parts:
                (p.view(torch.uint8) if p.dtype.itemsize == 1 else p).fill_(0x33 if p.dtype.itemsize == 1 else -7.0)
            assert bool((buf.view(torch.uint8) == 0x33).all() if buf.dtype.itemsize == 1 else (buf == -7).all()), name

    def table(self, aq, st):
        return aq.aq_adam_table(st, params=self.param, masters=self.master, grads=self.grad, m=self.m, v=self.v, m_scale=self.m_scale,
                                v_scale=self.v_scale, weight_decay=self.decay)

    def moments(self, i):
        """(m, v) of a tensor as binary32, on the CPU."""
        out = []
        for name in ("m", "v"):
            x = getattr(self, name)[i].cpu().float()
            if self.bits == 8:
                x = x * getattr(self, name + "_scale")[i].cpu().repeat_interleave(256)[:x.numel()]
            out.append(x)
        return out

    def snapshot(self):
        out = {"p": [(self.param if self.master is None else self.master)[i].cpu().double() for i in range(len(self.sizes))],
               "g": [x.cpu().float() for x in self.grad], "mv": [self.moments(i) for i in range(len(self.sizes))]}
        return out

    def check(self, before, lr, step, factor=1.0):
        for i, k in enumerate(self.sizes):
            if not k:
                continue
            m, v = forms.moments32(before["g"][i], *before["mv"][i], factor)
            if self.bits == 32:
                assert torch.equal(self.m[i].cpu(), m) and torch.equal(self.v[i].cpu(), v), i
            else:
                um, uv = forms.random(k, step)
                for name, x, u, kind in (("m", m, um, "e4m3"), ("v", v, uv, "e5m2")):
                    z, scale = forms.store8(x, u, kind)
                    assert torch.equal(getattr(self, name + "_scale")[i].cpu().double(), scale), (i, name)
                    assert torch.equal(getattr(self, name)[i].cpu().double(), z), (i, name)
            c1, c2 = 1 - 0.9 ** step, 1 - 0.999 ** step
            p, m, v = before["p"][i], m.double(), v.double()
            update = lr / c1 * m / (torch.sqrt(v / c2) + 1e-8)
            want = p - lr * self.decay[i] * p - update
            tol = 24 * E * update.abs() + 4 * E * lr * self.decay[i] * p.abs() + 2 * E * want.abs()
            if self.master is not None:
                close(self.master[i], want, tol, ("master", i))
                assert torch.equal(self.param[i], self.master[i].to(self.param[i].dtype))
            else:
                close(self.param[i], want, tol + rounding(self.dtype, want), ("param", i))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grads,master", [("fp32", "fp32", False), ("fp16", "fp16", False), ("fp16", "fp16", True), ("fp16", "fp32", True),
                                                ("bf16", "bf16", False), ("bf16", "fp32", False), ("bf16", "bf16", True)])
@pytest.mark.parametrize("packed", [False, True])
def test_adamw(aq, stage, bits, dtype, grads, master, packed):
    set_type(aq, stage, dtype)
    s = Set(SIZES, dtype, grads, bits, master, packed)
    table = s.table(aq, stage)
    for step, lr, factor in ((1, 1e-3, None), (2, 1e-3, 0.37), (1000, 3e-4, 1.0), (100000, 1e-5, 0.5)):
        before = s.snapshot()
        f = None if factor is None else torch.tensor([factor], device="cuda")
        aq.aq_adamw(stage, aq.AdamwConfig(lr=lr, beta1=0.9, beta2=0.999, eps=1e-8, step=step, state_bits=bits), table, len(SIZES), f, None, None)
        torch.cuda.synchronize()
        s.check(before, lr, step, 1.0 if factor is None else torch.tensor(factor, dtype=F32).item())
    s.check_between()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grads,master", [("fp32", "fp32", False), ("bf16", "bf16", False), ("fp16", "fp32", True), ("bf16", "bf16", True)])
@pytest.mark.parametrize("shift", list(range(8)))
def test_adamw_of_tensors_off_the_grid_of_eight(aq, stage, bits, dtype, grads, master, shift):
    """Tensors that all begin `shift` elements behind a multiple of eight, of lengths about those of blocks, units and pieces; and
    operands that do not begin alike."""
    set_type(aq, stage, dtype)
    sizes = [600, 256, 264 + shift, 263 - shift, 1000, 1024, 2304, 2048 + 255, 70001, 300]
    for alike in (True, False):
        s = Set(sizes, dtype, grads, bits, master, False)
        for name in ["param", "grad", "m", "v"] + (["master"] if master else []):
            for i, x in enumerate(getattr(s, name)):
                n = shift if alike or name != "grad" else (shift + 3) % 8
                buf = torch.zeros(x.numel() + 32, dtype=x.dtype, device="cuda")
                buf.view(torch.uint8).fill_(0x33)
                buf[8 + n:8 + n + x.numel()].copy_(x)
                getattr(s, name)[i] = buf[8 + n:8 + n + x.numel()]
                s.buffers[name, i] = (buf, [getattr(s, name)[i]])
        table = s.table(aq, stage)
        for step in (1, 500):
            before = s.snapshot()
            aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=step, state_bits=bits), table, len(sizes), None, None, None)
            s.check(before, 1e-3, step)
        for buf, (x,) in s.buffers.values():
            x.view(torch.uint8).fill_(0x33)
            assert bool((buf.view(torch.uint8) == 0x33).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_more_tensors_than_a_launch_takes(aq, stage, bits):
    set_type(aq, stage, "bf16")
    sizes = [(i * 37) % 700 for i in range(1005)]
    s = Set(sizes, "bf16", "bf16", bits, False, False)
    before = s.snapshot()
    aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=7, state_bits=bits), s.table(aq, stage), len(sizes), None, None, None)
    s.check(before, 1e-3, 7)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("factor", [math.nan, math.inf, -math.inf])
def test_adamw_that_is_left_out(aq, stage, bits, factor):
    set_type(aq, stage, "fp16")
    s = Set(SIZES, "fp16", "fp16", bits, True, False)
    keep = [[x.clone() for x in part] for part in (s.param, s.master, s.m, s.v)]
    aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=7, state_bits=bits), s.table(aq, stage), len(SIZES),
                torch.tensor([factor], device="cuda"), None, None)
    for part, old in zip((s.param, s.master, s.m, s.v), keep):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(part, old))


def test_adamw_from_zeros_and_with_zeros(aq, stage):
    """The first step moves every weight with a gradient by lr; weights without one only decay; states of zeros stay zeros."""
    set_type(aq, stage, "fp32")
    for bits in (32, 8):
        n = 1000
        p, g = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
        g[::2] = torch.randn(n // 2, device="cuda").abs() + 0.1
        state = dict(m=[torch.zeros(n, device="cuda")], v=[torch.zeros(n, device="cuda")])
        if bits == 8:
            state = dict(m=[torch.zeros(n, dtype=torch.uint8, device="cuda")], v=[torch.zeros(n, dtype=torch.uint8, device="cuda")],
                         m_scale=[torch.zeros(4, device="cuda")], v_scale=[torch.zeros(4, device="cuda")])
        table = aq.aq_adam_table(stage, params=[p], grads=[g], weight_decay=0.5, **state)
        aq.aq_adamw(stage, aq.AdamwConfig(lr=0.01, beta1=0.9, beta2=0.999, eps=1e-8, step=1, state_bits=bits), table, 1, None, None, None)
        # g / sqrt(g^2) is 1 but for the roundings of 24 e, of c1 and c2 (1e-3 in binary32: 6e-8) and eps / |g| of 1e-7
        assert bool(((p[::2] - (1 - 0.005 - 0.01)).abs() < 0.01 * 3e-6 + 2 * E).all()) and bool(((p[1::2] - 0.995).abs() < 2 * E).all())
        assert not state["m"][0][1::2].any() and not state["v"][0][1::2].any() and bool((state["v"][0][::2] != 0).all())


def test_second_moments_in_8_bits_never_vanish(aq, stage):
    """An element whose v is far below its block's largest keeps one, so that a gradient's end does not divide by eps alone."""
    set_type(aq, stage, "fp32")
    n = 512
    p, g = torch.zeros(n, device="cuda"), torch.full((n,), 1e-9, device="cuda")
    g[100] = 1e3
    g[300] = 0.0
    m, v = torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(n, dtype=torch.float8_e5m2, device="cuda")
    ms, vs = torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    table = aq.aq_adam_table(stage, params=[p], grads=[g], m=[m], v=[v], m_scale=[ms], v_scale=[vs])
    aq.aq_adamw(stage, aq.AdamwConfig(lr=0.0, beta1=0.9, beta2=0.999, eps=1e-8, step=1, state_bits=8), table, 1, None, None, None)
    stored = v.float()
    assert bool((stored[:256] > 0).all()) and stored[300] == 0 and bool((stored[301:] > 0).all()) and bool((stored[:100] == 2.0 ** -16).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_with_gradients_that_are_not_finite_and_no_factor(aq, stage, bits):
    """32 bits: its element alone.  8 bits: the block's scale is NaN, other blocks are as they would have been."""
    set_type(aq, stage, "bf16")
    s = Set([2000], "bf16", "bf16", bits, False, False)
    s.grad[0][700] = math.nan
    before = s.snapshot()
    aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=3, state_bits=bits), s.table(aq, stage), 1, None, None, None)
    p = s.param[0].cpu()
    assert bool(p[700].isnan()) and int(p.isnan().sum()) == 1
    if bits == 32:
        assert bool(s.m[0][700].isnan()) and int(s.m[0].isnan().sum()) == 1 and int(s.v[0].isnan().sum()) == 1
    else:
        assert s.m_scale[0].isnan().nonzero().flatten().tolist() == [2] and s.v_scale[0].isnan().nonzero().flatten().tolist() == [2]
        m, v = forms.moments32(before["g"][0], *before["mv"][0])
        z, _ = forms.store8(m[1024:1280], forms.random(256, 3, 1024)[0], "e4m3")
        assert torch.equal(s.m[0][1024:1280].cpu().double(), z)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_moments_at_the_ends_of_the_range(aq, stage, bits):
    """Gradients from 1e-18 to 1e18 in the same and in different blocks: blocks of one value, one large among small, powers of two."""
    set_type(aq, stage, "fp32")
    sizes = [256, 256, 256, 256, 256, 256]
    s = Set(sizes, "fp32", "fp32", bits, False, False)
    for i, g in enumerate([torch.full((256,), 1e-18), torch.full((256,), 1e18), torch.logspace(-18, 18, 256), torch.logspace(-6, 0, 256),
                           2.0 ** torch.arange(-40, 24).repeat(4).float(), torch.full((256,), 1.75).cumsum(0)]):
        s.grad[i].copy_(g * torch.where(torch.arange(256) % 3 == 0, -1.0, 1.0))
        s.m[i].view(torch.uint8).zero_()
        s.v[i].view(torch.uint8).zero_()
    for step in (1, 2, 3):
        before = s.snapshot()
        aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=step, state_bits=bits), s.table(aq, stage), 6, None, None, None)
        s.check(before, 1e-3, step)


def test_adamw_follows_the_mean_of_a_falling_second_moment(aq, stage):
    """As the plain form's test has it: 1500 steps of v falling by a thousandth, 4 standard errors of the mean of 16384 elements, 0.019."""
    set_type(aq, stage, "fp32")
    n = 16384
    s = Set([n], "fp32", "fp32", 8, False, False)
    s.grad[0].zero_()
    start = s.moments(0)[1].double()
    table = s.table(aq, stage)
    c = aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=0, state_bits=8)
    for step in range(1, 1501):
        c.step = step
        aq.aq_adamw(stage, c, table, 1, None, None, None)
    assert abs(s.moments(0)[1].double().mean() / (start.mean() * 0.999 ** 1500) - 1) < 4 * math.sqrt(0.375 / n) * 3
    # (the mean goes by the squares: elements are not alike, which raises the standard error by sqrt(mean v^2) / mean v = sqrt(3), below 3)


def test_step_in_a_captured_graph(aq, stage):
    """Norm, factor, step's number and learning rate on the device: replays do what eager calls with host settings do."""
    set_type(aq, stage, "bf16")
    for bits in (32, 8):
        one, two = (Set(SIZES, "bf16", "bf16", bits, True, False) for _ in range(2))
        norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        lr, step = torch.tensor([1e-3], device="cuda"), torch.tensor([0], device="cuda")
        config = aq.AdamwConfig(lr=math.nan, beta1=0.9, beta2=0.999, eps=1e-8, step=0, state_bits=bits)
        table = one.table(aq, stage)
        stream = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            aq.aq_stage_configure(stage, aq.AQ_STREAM, torch.cuda.current_stream().cuda_stream)
            aq.aq_grad_norm(stage, table, len(SIZES), 1.0, 0.5, norm, factor, step)
            aq.aq_adamw(stage, config, table, len(SIZES), factor, lr, step)
        aq.aq_stage_configure(stage, aq.AQ_STREAM, 0)
        for i in range(1, 5):
            lr.fill_(1e-3 / i)
            for a, b in zip(one.grad, two.grad):
                a.mul_(1.25)
                b.mul_(1.25)
            if i == 3:                                                       # a step that overflowed
                one.grad[9][5] = math.inf
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            if i == 3:
                assert math.isnan(factor.item())
                one.grad[9][5] = two.grad[9][5]
                continue
            at = i if i < 3 else i - 1
            assert step.item() == at
            c = aq.AdamwConfig(lr=torch.tensor(1e-3 / i, dtype=F32).item(), beta1=0.9, beta2=0.999, eps=1e-8, step=at, state_bits=bits)
            aq.aq_adamw(stage, c, two.table(aq, stage), len(SIZES), factor, None, None)
            for x, y in zip(one.param + one.m + one.v, two.param + two.m + two.v):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
        del graph


def test_layer_norm_in_a_captured_graph(aq, stage):
    """The norm and its gradient, captured after one call that grew the workspace; a larger call in between takes another, and the
    graph goes on with its own.  Without the call before, a capture is refused."""
    set_type(aq, stage, "bf16")
    rows, d = 300, 768
    x, r, w, b, dy, dsum = norm_inputs(rows, d, "bf16", seed=9)
    c = {n: v.cuda() for n, v in dict(x=x, r=r, w=w, b=b, dy=dy, dsum=dsum).items()}
    s, y, dx = (torch.empty_like(c["x"]) for _ in range(3))
    mean, rstd, dw, db = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")

    def call():
        aq.aq_layer_norm(stage, c["x"], d, c["r"], d, c["w"], c["b"], 1e-5, rows, d, s, d, y, d, mean, rstd)
        aq.aq_layer_norm_grad(stage, c["dy"], d, c["dsum"], d, s, d, c["w"], mean, rstd, rows, d, dx, d, dw, db)

    def capture():
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            aq.aq_stage_configure(stage, aq.AQ_STREAM, torch.cuda.current_stream().cuda_stream)
            try:
                call()
            finally:
                aq.aq_stage_configure(stage, aq.AQ_STREAM, 0)
        return graph
    with pytest.raises(aq.AqError) as e:
        capture()
    assert e.value.code == aq.AQ_EUNSUPPORTED
    call()
    graph = capture()
    wide = torch.zeros((600, 4096), dtype=torch.bfloat16, device="cuda")
    f = torch.zeros(4096, device="cuda")
    aq.aq_layer_norm_grad(stage, wide, 4096, None, 0, wide, 4096, None, torch.zeros(600, device="cuda"), torch.ones(600, device="cuda"), 600, 4096, wide, 4096, f, f.clone())
    c["x"].mul_(0.5)
    c["dy"].mul_(2.0)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    total = (c["x"].cpu().float() + r.float()).bfloat16()
    assert torch.equal(s.cpu(), total)
    check_norm("bf16", total, w, b, 1e-5, y, mean, rstd)
    check_norm_grad("bf16", c["dy"], dsum, total, w, mean, rstd, (dx, dw, db))
    del graph


def test_two_handles_on_two_streams(aq):
    """Calls on two handles at once, each on its own stream, give what each gives alone."""
    handles = [aq.aq_stage_create() for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    sizes = [300000, 77, 4096]
    norms = [torch.zeros(1, device="cuda") for _ in range(2)]
    sets, grads = [], []
    for i, h in enumerate(handles):
        aq.aq_stage_configure(h, aq.AQ_DTYPE, aq.AQ_FP16)
        aq.aq_stage_configure(h, aq.AQ_STREAM, streams[i].cuda_stream)
        sets.append(Set(sizes, "fp16", "fp16", 8, True, False, seed=20 + i))
        s, _, w, _, dy, _ = norm_inputs(2000, 1600, "fp16", seed=i)
        mean, rstd = statistics(s)
        grads.append([v.cuda() for v in (dy, s, w, mean, rstd)] + [torch.empty_like(s, device="cuda")] + [torch.empty(1600, device="cuda") for _ in range(2)])
    before = [s.snapshot() for s in sets]
    torch.cuda.synchronize()
    config = aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=5, state_bits=8)
    tables = [s.table(aq, h) for s, h in zip(sets, handles)]
    for _ in range(20):
        for i, h in enumerate(handles):
            dy, s, w, mean, rstd, dx, dw, db = grads[i]
            aq.aq_layer_norm_grad(h, dy, 1600, None, 0, s, 1600, w, mean, rstd, 2000, 1600, dx, 1600, dw, db)
            aq.aq_grad_norm(h, tables[i], 3, 1.0, 1.0, norms[i], None, None)
    for i, h in enumerate(handles):
        aq.aq_adamw(h, config, tables[i], 3, None, None, None)
    torch.cuda.synchronize()
    for i in range(2):
        dy, s, w, mean, rstd, dx, dw, db = grads[i]
        check_norm_grad("fp16", dy, None, s, w, mean, rstd, (dx, dw, db))
        sets[i].check(before[i], 1e-3, 5)
        assert abs(norms[i].item() / forms.clip(before[i]["g"], 1.0, 1.0)[0] - 1) < 6 * E
    for h in handles:
        aq.aq_stage_destroy(h)


def test_four_threads_with_a_handle_each(aq):
    """Different widths and kinds of moments at once: what the threads share on the host is set once and for all sizes."""
    import threading
    results = {}

    def work(i):
        st = aq.aq_stage_create()
        stream = torch.cuda.Stream()
        aq.aq_stage_configure(st, aq.AQ_DTYPE, aq.AQ_BF16)
        aq.aq_stage_configure(st, aq.AQ_STREAM, stream.cuda_stream)
        try:
            d = (264, 1600, 2056, 5000)[i]
            s, _, w, _, dy, _ = norm_inputs(64, d, "bf16", seed=i)
            mean, rstd = statistics(s)
            with torch.cuda.stream(stream):
                bufs = [v.cuda() for v in (dy, s, w, mean, rstd)] + [torch.empty((64, d), dtype=torch.bfloat16, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")]
                tensors = Set([3000, 77], "bf16", "bf16", 8 if i % 2 else 32, bool(i // 2), False, seed=i)
                stream.synchronize()
                before, table = tensors.snapshot(), tensors.table(aq, st)
                config = aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, state_bits=tensors.bits)
                for _ in range(20):
                    aq.aq_layer_norm_grad(st, bufs[0], d, None, 0, bufs[1], d, bufs[2], bufs[3], bufs[4], 64, d, bufs[5], d, bufs[6], bufs[7])
                aq.aq_adamw(st, config, table, 2, None, None, None)
                stream.synchronize()
                check_norm_grad("bf16", dy, None, s, w, mean, rstd, bufs[5:])
                tensors.check(before, 1e-3, 1)
            results[i] = "done"
        finally:
            aq.aq_stage_destroy(st)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert results == {i: "done" for i in range(4)}


def test_step_of_a_tensor_beyond_32_bit_offsets(aq, stage):
    """2^31 + 4097 elements with moments in 8 bits: the last blocks, and the norm of all."""
    set_type(aq, stage, "bf16")
    n = 2 ** 31 + 4097
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    tail = 5000
    g[-tail:] = torch.randn(tail, device="cuda") * 0.01
    m, v = torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(n, dtype=torch.float8_e5m2, device="cuda")
    ms, vs = torch.zeros(-(-n // 256), device="cuda"), torch.zeros(-(-n // 256), device="cuda")
    table = aq.aq_adam_table(stage, params=[p], grads=[g], m=[m], v=[v], m_scale=[ms], v_scale=[vs])
    norm = torch.zeros(1, device="cuda")
    aq.aq_grad_norm(stage, table, 1, 1.0, 0.0, norm, None, None)
    want = math.sqrt((n - tail) * 2.0 ** -20 + g[-tail:].double().square().sum().item())
    assert abs(norm.item() / want - 1) < 6 * E
    aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=9, state_bits=8), table, 1, None, None, None)
    begin = n - n % 256 - 4096                                               # whole blocks of the tail and the last one
    k = n - begin
    zero = torch.zeros(k)
    m32, v32 = forms.moments32(g[begin:].cpu().float(), zero, zero)
    um, uv = forms.random(k, 9, begin)
    for x, u, kind, codes, scales in ((m32, um, "e4m3", m, ms), (v32, uv, "e5m2", v, vs)):
        z, scale = forms.store8(x, u, kind)
        assert torch.equal(codes[begin:].cpu().double(), z) and torch.equal(scales[begin // 256:].cpu().double(), scale)
    update = 1e-3 / (1 - 0.9 ** 9) * m32.double() / (torch.sqrt(v32.double() / (1 - 0.999 ** 9)) + 1e-8)
    close(p[begin:], -update, 24 * E * update.abs() + rounding("bf16", update), "param")
    assert bool((p[:begin:4099] != 0).all())


def test_a_training_step_of_all(aq, stage):
    """Norm, its gradient, the clipping and the step as a user strings them together, on one stream without a wait, against torch in binary64."""
    set_type(aq, stage, "fp32")
    rows, d, steps = 96, 200, 5
    g = torch.Generator().manual_seed(5)
    x, r, target = (torch.randn((rows, d), generator=g) for _ in range(3))
    w, b = torch.ones(d).cuda(), torch.zeros(d).cuda()
    state = [[torch.zeros(d, device="cuda") for _ in range(2)] for _ in range(3)]            # gradients, m, v
    table = aq.aq_adam_table(stage, params=[w, b], grads=state[0], m=state[1], v=state[2], weight_decay=[0.1, 0.0])
    s, y, dx = (torch.empty((rows, d), device="cuda") for _ in range(3))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    norm, factor, step = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    config = aq.AdamwConfig(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, state_bits=32)
    xc, rc, tc = x.cuda(), r.cuda(), target.cuda()
    for _ in range(steps):
        aq.aq_layer_norm(stage, xc, d, rc, d, w, b, 1e-5, rows, d, s, d, y, d, mean, rstd)
        dy = (y - tc) * (2 / rows)
        aq.aq_layer_norm_grad(stage, dy, d, None, 0, s, d, w, mean, rstd, rows, d, dx, d, *state[0])
        aq.aq_grad_norm(stage, table, 2, 1.0, 1.0, norm, factor, step)
        aq.aq_adamw(stage, config, table, 2, factor, None, step)
    w64, b64 = torch.ones(d, dtype=F64, requires_grad=True), torch.zeros(d, dtype=F64, requires_grad=True)
    x64 = (x + r).double().requires_grad_(True)
    adam = torch.optim.AdamW([{"params": [w64], "weight_decay": 0.1}, {"params": [b64], "weight_decay": 0.0}], lr=1e-2)
    for _ in range(steps):
        adam.zero_grad()
        x64.grad = None
        ((torch.nn.functional.layer_norm(x64, (d,), w64, b64, 1e-5) - target.double()).square().sum() / rows).backward()
        size = torch.nn.utils.clip_grad_norm_([w64, b64], 1.0)
        adam.step()
    # five steps whose every quantity is off by less than 1e-5 of it; updates are 0.01 each
    assert step.item() == steps and abs(norm.item() / size.item() - 1) < 1e-4
    close(w, w64.detach(), 1e-5, "w")
    close(b, b64.detach(), 1e-5, "b")
    close(dx, x64.grad, 1e-5 * x64.grad.abs().max(), "dx")


# ---- refusals ------------------------------------------------------------------------------------------------

def refused(aq, code, call, *args):
    with pytest.raises(aq.AqError) as e:
        call(*args)
    assert e.value.code == code
    return str(e.value)


def test_layer_norm_refusals(aq, stage):
    set_type(aq, stage, "fp16")
    x = torch.zeros((8, 64), dtype=torch.float16, device="cuda")
    y, s, w, f = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(64, dtype=torch.float16, device="cuda"), torch.zeros(64, device="cuda")
    odd = x.data_ptr() + 1
    good = dict(x=x, ldx=64, residual=y, ldr=64, w=w, b=w, eps=1e-5, rows=4, hidden=64, sum=s, lds=64, y=torch.zeros_like(x), ldy=64, mean=f, rstd=f)
    for change in (dict(x=None), dict(x=odd), dict(ldx=63), dict(residual=odd), dict(ldr=10), dict(w=odd), dict(b=odd), dict(eps=-1.0), dict(eps=math.nan),
                   dict(eps=math.inf), dict(rows=-1), dict(rows=2 ** 31), dict(hidden=0), dict(hidden=-5), dict(hidden=2 ** 20 + 1), dict(sum=odd), dict(lds=1),
                   dict(residual=None), dict(y=None), dict(y=odd), dict(ldy=63), dict(mean=odd), dict(rstd=odd), dict(sum=x, lds=128),
                   dict(y=x, ldy=72), dict(sum=y, y=y), dict(sum=y, lds=65)):
        assert "aq_layer_norm" in refused(aq, aq.AQ_EINVAL, aq.aq_layer_norm, stage, *dict(good, **change).values()), change
    good = dict(dy=x, lddy=64, dsum=y, ldds=64, s=s, lds=64, w=w, mean=f, rstd=f, rows=4, hidden=64, dx=torch.zeros_like(x), lddx=64, dw=f, db=f)
    for change in (dict(dy=None), dict(dy=odd), dict(lddy=63), dict(dsum=odd), dict(ldds=3), dict(s=None), dict(s=odd), dict(lds=63), dict(w=odd),
                   dict(mean=None), dict(rstd=None), dict(mean=odd), dict(rows=-1), dict(rows=2 ** 31), dict(hidden=0), dict(hidden=2 ** 20 + 1), dict(dx=odd),
                   dict(lddx=63), dict(dw=odd), dict(db=odd), dict(dx=x, lddx=72), dict(dx=y, lddx=72), dict(dx=s, lddx=72)):
        assert "aq_layer_norm_grad" in refused(aq, aq.AQ_EINVAL, aq.aq_layer_norm_grad, stage, *dict(good, **change).values()), change
    torch.cuda.synchronize()
    assert not x.any() and not s.any() and not f.any() and aq.aq_stage_status(stage) == 0


def test_step_refusals(aq, stage):
    set_type(aq, stage, "fp16")
    h = lambda n: torch.zeros(n, dtype=torch.float16, device="cuda")  # noqa: E731
    p, g, ms, m, v, f = h(300), h(300), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(8, device="cuda")

    def table(**change):
        t = aq.aq_adam_table(stage, params=[p], grads=[g], masters=[ms], m=[m], v=[v])
        for name, x in change.items():
            setattr(t[0], name, x)
        return t
    fine = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, state_bits=32)
    config = lambda **c: aq.AdamwConfig(**dict(fine, **c))  # noqa: E731
    odd = f.data_ptr() + 1
    call = lambda c, t, n=1, *rest: (aq.aq_adamw, stage, c, t, n, *(rest or (None, None, None)))  # noqa: E731
    for c in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=math.nan), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=math.nan), dict(eps=1e31),
              dict(lr=math.nan), dict(lr=math.inf), dict(lr=1e39), dict(step=0), dict(step=-3), dict(state_bits=16), dict(state_bits=0)):
        assert "aq_adamw" in refused(aq, aq.AQ_EINVAL, *call(config(**c), table())), c
    for t in (dict(numel=-1), dict(numel=2 ** 41), dict(param=None), dict(param=odd), dict(master=odd), dict(grad=None), dict(grad=odd), dict(m=None), dict(m=odd),
              dict(v=None), dict(v=odd), dict(weight_decay=-1.0), dict(weight_decay=math.nan), dict(weight_decay=math.inf), dict(grad_dtype=aq.AQ_BF16), dict(grad_dtype=9)):
        assert "tensor 0" in refused(aq, aq.AQ_EINVAL, *call(config(), table(**t))), t
    refused(aq, aq.AQ_EINVAL, *call(config(state_bits=8), table()))          # no scales
    refused(aq, aq.AQ_EINVAL, *call(config(), None))
    refused(aq, aq.AQ_EINVAL, *call(config(), table(), -1))
    for rest in ((odd, None, None), (None, odd, None), (None, None, f.data_ptr() + 4)):
        refused(aq, aq.AQ_EINVAL, *call(config(), table(), 1, *rest))
    t = table(grad_dtype=aq.AQ_FP32)
    set_type(aq, stage, "fp32")
    refused(aq, aq.AQ_EINVAL, *call(config(), t))                            # a master beside binary32 parameters
    set_type(aq, stage, "fp16")
    norm = lambda t, n=1, inv=1.0, limit=1.0, a=f, b=None, c=None: (aq.aq_grad_norm, stage, t, n, inv, limit, a, b, c)  # noqa: E731
    for args in (norm(None), norm(table(), -1), norm(table(), inv=0.0), norm(table(), inv=-1.0), norm(table(), inv=math.nan), norm(table(), inv=math.inf),
                 norm(table(), limit=-1.0), norm(table(), limit=math.nan), norm(table(), a=odd), norm(table(), b=odd), norm(table(), c=f.data_ptr() + 4),
                 norm(table(grad=None)), norm(table(grad=odd)), norm(table(numel=-1)), norm(table(grad_dtype=aq.AQ_BF16))):
        assert "aq_grad_norm" in refused(aq, aq.AQ_EINVAL, *args)
    torch.cuda.synchronize()
    assert not p.any() and not m.any() and not f.any() and aq.aq_stage_status(stage) == 0
    aq.aq_adamw(stage, config(), None, 0, None, None, None)                   # no tensors: nothing to do
