"""Layer norms and optimizer's steps one behind another in the same buffers: a kernel may start while the one before it still writes what it reads."""
import pytest
import torch

from tests.stage_forms import TYPES
from tests.test_gpu_stage import set_type
from tests.test_gpu_step import Set, aq, norm_inputs, stage  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp16", "fp32"])
@pytest.mark.parametrize("rows,d", [(700, 1600), (700, 1021), (3001, 40), (300, 5000), (70, 12000), (70, 12001), (9, 40001)])
def test_norms_in_place_one_behind_another(aq, stage, dtype, rows, d):  # noqa: F811
    """Eight norms whose sum and output take the inputs' places, each followed by its gradient in dy's place: without a wait in between
    the same bits as with one behind every call."""
    set_type(aq, stage, dtype)
    x, r, w, b, dy, dsum = (v.cuda() for v in norm_inputs(rows, d, dtype, seed=21))
    results = []
    for wait in (False, True):
        one, two, back = x.clone(), r.clone(), dy.clone()
        mean, rstd, dw, db = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
        torch.cuda.synchronize()
        for _ in range(8):
            aq.aq_layer_norm(stage, one, d, two, d, w, b, 1e-5, rows, d, two, d, one, d, mean, rstd)
            if wait:
                torch.cuda.synchronize()
            aq.aq_layer_norm_grad(stage, back, d, dsum, d, two, d, w, mean, rstd, rows, d, back, d, dw, db)
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        results.append([v.cpu() for v in (one, two, back, mean, rstd, dw, db)])
    assert all(torch.equal(p, q) for p, q in zip(*results))


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_whose_settings_the_kernel_before_writes(aq, stage, bits):  # noqa: F811
    """The factor and the step's number go from the norm's kernel to the step's, and the step's weights to a layer norm."""
    set_type(aq, stage, "bf16")
    d, results = 1600, []
    x = torch.randn((64, d), generator=torch.Generator().manual_seed(3)).to(TYPES["bf16"]).cuda()
    for wait in (False, True):
        s = Set([d, d, 30000], "bf16", "bf16", bits, True, False, seed=31)
        y, table, config = torch.empty_like(x), s.table(aq, stage), aq.AdamwConfig(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, state_bits=bits)
        norm, factor, step = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
        torch.cuda.synchronize()
        for _ in range(8):
            for call, *args in ((aq.aq_grad_norm, table, 3, 1.0, 0.5, norm, factor, step), (aq.aq_adamw, config, table, 3, factor, None, step),
                                (aq.aq_layer_norm, x, d, None, d, s.param[0], s.param[1], 1e-5, 64, d, None, d, y, d, None, None)):
                call(stage, *args)
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert step.item() == 8
        results.append([v.cpu().view(torch.uint8) for v in (y, norm, factor, *s.param, *s.master, *s.m, *s.v)])
    assert all(torch.equal(p, q) for p, q in zip(*results))
