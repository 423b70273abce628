"""The gradients' norm, the step and the layer norm at the ends of their ranges."""
import math

import pytest
import torch

from tests import step_forms as forms
from tests.stage_forms import TYPES
from tests.test_gpu_stage import E, set_type
from tests.test_gpu_step import aq, stage  # noqa: F401

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
