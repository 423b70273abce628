"""The gradients' norm, the step and the layer norm at the ends of their ranges."""
import math

import pytest
import torch

from tests import step_forms as forms
from tests.stage_forms import TYPES
from tests.test_gpu_stage import E, set_type
from tests.test_gpu_step import Set, aq, check_norm, check_norm_grad, norm_inputs, run_norm, run_norm_grad, stage, statistics  # noqa: F401

pytestmark = pytest.mark.gpu


def norm_of(aq, stage, grads, inv_scale=1.0, limit=1.0):
    norm, factor, step = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    aq.aq_grad_norm(stage, aq.aq_adam_table(stage, grads=grads), len(grads), inv_scale, limit, norm, factor, step)
    return norm.item(), factor.item(), step.item()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,at", [(8, range(8)), (8192, range(4096, 4104)), (8192, [5, 6]), (2000, range(1990, 2000)), (100003, range(0, 100003, 7))])
@pytest.mark.parametrize("shift", [0, 3])
def test_norm_of_gradients_whose_squares_are_binary32_numbers(aq, stage, dtype, n, at, shift):  # noqa: F811
    """Squares up to 3.4e38 each, whatever their sum; an element of 1.9e19, whose square is above, makes the norm infinite."""
    set_type(aq, stage, dtype)
    g = torch.zeros(n + shift, dtype=TYPES[dtype], device="cuda")[shift:]
    for value in (6.6e18, 1e19, 1.3e19, 1.8e19):
        g[list(at)] = value
        want = forms.clip([g.cpu()], 1.0, 1.0)
        norm, factor, step = norm_of(aq, stage, [g])
        # as in test_grad_norm: eight squares in binary32, halved by the root, and the roundings of the outputs
        assert abs(norm / want[0] - 1) < 6 * E and abs(factor / want[1] - 1) < 7 * E and step == 1, value
    for bad in (1.9e19, math.inf, math.nan):
        g[at[1]] = bad
        norm, factor, step = norm_of(aq, stage, [g])
        assert not math.isfinite(norm) and math.isnan(factor) and step == 0, bad


def test_a_norm_beyond_binary32_is_not_counted(aq, stage):  # noqa: F811
    """norm is infinite as it is returned, so the step is one to leave out, clipped or not."""
    set_type(aq, stage, "fp32")
    g = torch.full((4,), 1e10, device="cuda")
    for limit in (0.0, 1.0):
        norm, factor, step = norm_of(aq, stage, [g], 1e30, limit)
        assert norm == math.inf and math.isnan(factor) and step == 0
        norm, factor, step = norm_of(aq, stage, [g], 1e28, limit)
        assert math.isfinite(norm) and math.isfinite(factor) and factor > 0 and step == 1


@pytest.mark.parametrize("inv_scale", [3.4e38, 2e-38])
def test_scales_at_the_ends_of_binary32(aq, stage, inv_scale):  # noqa: F811
    set_type(aq, stage, "fp32")
    norm, factor, step = norm_of(aq, stage, [torch.full((4,), 0.25, device="cuda")], inv_scale, 0.0)
    assert abs(norm / (0.5 * inv_scale) - 1) < 3 * E and abs(factor / inv_scale - 1) < E and step == 1


@pytest.mark.parametrize("rows,d", [(1375000, 1600), (2000000, 64)])
def test_sums_over_very_many_rows(aq, stage, rows, d):  # noqa: F811
    """dw and db of 2.2e9 elements: a thread adds rows / 148 or fewer one by one, then come the CTA's warps and up to 148 CTAs' sums one
    by one: (rows / 148 + 200) e of the sum of magnitudes with the three roundings of n and of its product."""
    set_type(aq, stage, "bf16")
    chunks = [slice(r, min(r + 125000, rows)) for r in range(0, rows, 125000)]
    s, dy = (torch.empty((rows, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(d)
    want, size = [torch.zeros((2, d), dtype=torch.float64, device="cuda") for _ in range(2)]
    for c in chunks:
        s[c] = torch.randn(s[c].shape, generator=g, device="cuda") + 1.0
        dy[c] = torch.randn(s[c].shape, generator=g, device="cuda") + 0.25     # a sum that grows with the rows
        mean[c], rstd[c] = s[c].float().mean(1), 1 + 0.1 * torch.rand(s[c].shape[0], generator=g, device="cuda")
        y = dy[c].double()
        n = (s[c].double() - mean[c, None].double()) * rstd[c, None].double()
        for out, f in ((want, lambda x: x), (size, torch.abs)):
            out += torch.stack([f(y * n).sum(0), f(y).sum(0)])
        del y, n
    w, dw, db = torch.ones(d, device="cuda").bfloat16(), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dx = torch.empty_like(s) if d == 64 else None
    aq.aq_layer_norm_grad(stage, dy, d, None, 0, s, d, w, mean, rstd, rows, d, dx, d, dw, db)
    k = (rows / 148 + 200) * E
    for have, exact, magnitude in zip((dw, db), want, size):
        assert bool(((have.double() - exact).abs() <= k * magnitude).all())


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
@pytest.mark.parametrize("d", [1, 40, 64, 1021, 1600, 1601, 5000, 12001, 33000, 40001])
@pytest.mark.parametrize("with_w,with_b", [(True, False), (False, True)])
def test_layer_norm_with_one_of_weight_and_bias(aq, stage, dtype, d, with_w, with_b):  # noqa: F811
    set_type(aq, stage, dtype)
    for pad, offset in ((0, 0), (3, 0), (1, 5)):
        x, r, w, b, _, _ = norm_inputs(5, d, dtype, seed=12)
        w, b = w if with_w else None, b if with_b else None
        s, y, mean, rstd = run_norm(aq, stage, dtype, x, r, w, b, 1e-5, pad, offset)
        check_norm(dtype, s, torch.ones(d) if w is None else w, torch.zeros(d) if b is None else b, 1e-5, y, mean, rstd)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_gradient_whose_square_exceeds_binary32(aq, stage, bits):  # noqa: F811
    """v is infinite then and the element moves by its decay alone; in 8 bits its block's v is NaN from the next step on, and other blocks
    are as they would have been."""
    set_type(aq, stage, "fp32")
    one, two = (Set([1000], "fp32", "fp32", bits, False, False, seed=41, decay=0.0) for _ in range(2))
    one.grad[0][300] = 1e20
    old = one.param[0].clone()
    for s in (one, two):
        aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=3, state_bits=bits), s.table(aq, stage), 1, None, None, None)
    assert one.param[0][300] == old[300]
    keep = torch.arange(1000, device="cuda") != 300
    assert torch.equal(one.param[0][keep], two.param[0][keep])
    if bits == 32:
        assert one.v[0][300] == math.inf and torch.equal(one.v[0][keep], two.v[0][keep]) and torch.equal(one.m[0][keep], two.m[0][keep])
    else:
        assert one.v_scale[0].isnan().tolist() == [False, True, False, False] and not one.m_scale[0].isnan().any()
        others = torch.arange(1000, device="cuda") // 256 != 1
        for name in ("m", "v"):
            assert torch.equal(getattr(one, name)[0].view(torch.uint8)[others], getattr(two, name)[0].view(torch.uint8)[others])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("d", [3, 64, 250, 1021, 1600, 2045, 5001, 8190, 12000, 12001, 40001])
@pytest.mark.parametrize("pad", [0, 1])
def test_gradient_of_rows_very_far_from_zero(aq, stage, dtype, d, pad):  # noqa: F811
    """Rows of one value, whose mean times rstd is beyond binary32 though every element is at its mean: the places behind a row's end, which
    threads fill with zeros, count for nothing."""
    set_type(aq, stage, dtype)
    rows = 19
    s, _, w, _, dy, dsum = norm_inputs(rows, d, dtype, seed=13)
    s[::3] = torch.tensor([2.0 ** 115, -2.0 ** 120, 2.0 ** 127, 2.0 ** 100])[torch.arange(rows)[::3] % 4].to(s.dtype)[:, None]
    mean, rstd = statistics(s)
    mean[::3], rstd[::3] = s[::3, 0].float(), 1e5
    got = run_norm_grad(aq, stage, dtype, dy, dsum, s, w, mean, rstd, pad)
    check_norm_grad(dtype, dy, dsum, s, w, mean, rstd, got)


@pytest.mark.parametrize("d", [3, 64, 250, 1600, 2045, 8190, 12000, 12001, 40001])
@pytest.mark.parametrize("pad", [0, 1])
def test_gradient_of_rows_very_far_apart(aq, stage, d, pad):  # noqa: F811
    """Rows with elements of 3e38 on both sides of their mean, which have rstd 0: dx is the gradient along the stream."""
    set_type(aq, stage, "fp32")
    rows = 19
    s, _, w, _, dy, dsum = norm_inputs(rows, d, "fp32", seed=14)
    s[::3] = 3e38 * torch.sign(s[::3])
    dy[::3] *= 100
    mean, rstd = statistics(s)
    mean[::3], rstd[::3] = 0.0, 0.0
    got = run_norm_grad(aq, stage, "fp32", dy, dsum, s, w, mean, rstd, pad)
    check_norm_grad("fp32", dy, dsum, s, w, mean, rstd, got)
    assert torch.equal(got[0][::3].cpu(), dsum[::3])
