"""Stage operators without a GPU: what a handle-less call answers, and the plain forms the GPU tests compare with
against differences and hand-worked values."""
import ctypes
import math

import pytest
import torch

import paper_2206_01299_b200 as aq
from tests import stage_forms as forms

F64 = torch.float64


def test_calls_without_a_handle_are_refused():
    L = aq.lib()
    assert L.aq_stage_configure(None, aq.AQ_DTYPE, aq.AQ_FP16) == aq.AQ_EINVAL
    assert L.aq_stage_status(None, ctypes.byref(ctypes.c_uint32())) == aq.AQ_EINVAL
    assert L.aq_token_logprobs(None, None, 1, 1, 1, None, 1.0, 0, None, None, None, None, None) == aq.AQ_EINVAL
    assert L.aq_token_logprobs_grad(None, None, 1, 1, 1, None, 1.0, None, None, None, None, None, 1) == aq.AQ_EINVAL
    assert L.aq_gated_ffn(None, None, 8, None, None, 8, 1, 8, 8, 0, None, 8, None, None, 8) == aq.AQ_EINVAL
    assert L.aq_gated_ffn_grad(None, None, 8, None, 8, None, None, 8, None, None, 8, 1, 8, 8, 0, None, 8, None, None, 8) == aq.AQ_EINVAL
    assert L.aq_qk_norm_rope(None, None, 1, None, 8, None, 8, None, None, None, None, None, 8, None, 8) == aq.AQ_EINVAL
    assert L.aq_qk_norm_rope_grad(None, None, 1, None, 8, None, 8, None, 8, None, 8, None, None, None, None, None, 8, None, 8, None, None) == aq.AQ_EINVAL
    L.aq_stage_destroy(None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="says what happens without a device")
def test_create_without_a_device_says_why():
    with pytest.raises(aq.AqError) as e:
        aq.aq_stage_create()
    assert e.value.code == aq.AQ_ECUDA and "aq_stage_create" in str(e.value)


def test_constants_of_the_stage_operators():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "aq_b200.h")).read()
    for name in ("AQ_FP32", "AQ_ACT_SILU", "AQ_ACT_GELU", "AQ_ACT_GELU_TANH", "AQ_ST_STALLED"):
        assert getattr(aq, name) == int(re.search(rf"\b{name}\s*=\s*(\d+)", text).group(1))
    # int32 x 5, float, int64: no padding
    assert ctypes.sizeof(aq.QkShape) == 32 and aq.QkShape.n_positions.offset == 24


def _directional(f, x, v, h=1e-5):
    return ((f(x + h * v) - f(x - h * v)) / (2 * h)).item()


def test_plain_logprobs_by_hand():
    # probabilities 1/2, 1/4, 1/4: entropy 1.5 bits
    x = torch.log(torch.tensor([2.0, 1.0, 1.0], dtype=F64))
    lp, h, lse, ids, top = forms.logprobs(x, 1, 1.0, 3)
    assert abs(lp + math.log(4)) < 1e-15 and abs(h - 1.5 * math.log(2)) < 1e-15 and abs(lse - math.log(4)) < 1e-15
    assert ids.tolist() == [0, 1, 2] and torch.allclose(top, -torch.log(torch.tensor([2.0, 4.0, 4.0], dtype=F64)))


def test_plain_logprobs_gradient_against_differences():
    g = torch.Generator().manual_seed(1)
    x, v = torch.randn(33, generator=g, dtype=F64), torch.randn(33, generator=g, dtype=F64)

    def f(y):
        lp, h, *_ = forms.logprobs(y, 7, 0.8, 0)
        return torch.tensor(0.3 * lp - 0.2 * h, dtype=F64)
    assert abs(_directional(f, x, v) - (forms.logprobs_grad(x, 7, 0.8, 0.3, -0.2) @ v).item()) < 1e-8


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh"])
def test_plain_ffn_gradient_against_differences(name):
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, dtype=F64)  # noqa: E731
    x, wg, wu, dh = r(5, 8), r(6, 8), r(6, 8), r(5, 6)
    _, gg, u = forms.ffn(x, wg, wu, name)
    _, _, dx, dwg, dwu = forms.ffn_grad(dh, x, wg, wu, gg, u, name)
    for at, grad in ((0, dx), (1, dwg), (2, dwu)):
        args = [x, wg, wu]
        v = torch.randn(args[at].shape, generator=g, dtype=F64)
        f = lambda y: (forms.ffn(*[y if i == at else a for i, a in enumerate(args)], name)[0] * dh).sum()  # noqa: E731
        assert abs(_directional(f, args[at], v) - (grad * v).sum().item()) < 1e-7


@pytest.mark.parametrize("interleaved", [False, True])
def test_plain_rotation_keeps_lengths_and_turns_by_the_angle(interleaved):
    angle = torch.tensor([[0.3, 1.1]], dtype=F64)
    cs = torch.cat([angle.cos(), angle.sin()], 1)
    x = torch.tensor([[[3.0, 4.0, 0.0, 5.0]]], dtype=F64)
    w = torch.ones(4, dtype=F64)
    y = forms.qk(x, w, 0.0, cs, torch.tensor([0]), 4, interleaved)
    assert abs(y.square().mean().item() - 1) < 1e-14
    pair = (0, 1) if interleaved else (0, 2)
    n = x / x.square().mean().sqrt()
    a, b = n[0, 0, pair[0]], n[0, 0, pair[1]]
    assert abs(y[0, 0, pair[0]] - (a * math.cos(0.3) - b * math.sin(0.3))) < 1e-14
