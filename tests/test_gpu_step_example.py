"""The two-stage example with layer norms and the library's optimizer: it runs, and its norm's gradients are torch's."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("finetune_two_stages", os.path.join(ROOT, "examples", "finetune_two_stages.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("norm,optimizer", [("layer", "torch"), ("rms", "adamw"), ("layer", "adamw"), ("layer", "adamw8")])
def test_the_example_runs(example, norm, optimizer):
    losses = example.train(epochs=2, say=lambda *_: None, norm=norm, optimizer=optimizer)
    assert len(losses) == 2 * example.SAMPLES // example.BATCH and all(math.isfinite(x) for x in losses)


@pytest.mark.parametrize("residual", [False, True])
def test_gradients_of_the_examples_norm(example, residual):
    """bf16 outputs are off by half a step of 2^-8 each, sums of 96 rows in binary32 and rounded once: 2^-8 of the value and, for
    what cancels, of the largest one."""
    aq = example.aq
    st = aq.aq_stage_create()
    aq.aq_stage_configure(st, aq.AQ_DTYPE, aq.AQ_BF16)
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g).to(example.T).cuda()  # noqa: E731
    x, res, w, b, ds, dy = r(96, 200), r(96, 200) if residual else None, r(200), r(200), r(96, 200), r(96, 200)
    leaves = [v.clone().requires_grad_(True) for v in ([x, res, w, b] if residual else [x, w, b])]
    args = leaves if residual else [leaves[0], None, *leaves[1:]]
    s, y = example.LayerNorm.apply(st, *args)
    got = torch.autograd.grad([s, y], leaves, [ds, dy])
    wide = [v.detach().double().requires_grad_(True) for v in leaves]
    total = wide[0] + wide[1] if residual else wide[0]
    # the norm is that of the stored sum, whose rounding has no gradient
    total = total + ((total.detach().to(example.T).double() - total.detach()))
    z = torch.nn.functional.layer_norm(total, (200,), wide[-2], wide[-1], example.EPS)
    want = torch.autograd.grad([total, z], wide, [ds.double(), dy.double()])
    for a, c in zip((s, y, *got), (total.detach(), z.detach(), *want)):
        assert bool(((a.double() - c).abs() <= 2.0 ** -8 * c.abs() + 2.0 ** -16 * c.abs().max()).all())
    aq.aq_stage_destroy(st)


def test_the_examples_optimizer_against_torch(example):
    """Five clipped steps over tensors of its kinds, in binary64 by torch; each step moves a weight by up to lr, and is off by 24 roundings
    of that, the weight by two of its own: 5 * (24 * 0.005 + 2) * 2^-24 < 1e-6."""
    g = torch.Generator().manual_seed(3)
    params = [torch.randn(s, generator=g).cuda().requires_grad_(True) for s in ((96, 128), (128,), (7, 3), (5,))]
    wide = [p.detach().double().requires_grad_(True) for p in params]
    ours = example.AdamW(params, 0.005, 32)
    theirs = torch.optim.AdamW([{"params": [wide[0], wide[2]], "weight_decay": 0.01}, {"params": [wide[1], wide[3]], "weight_decay": 0.0}], lr=0.005)
    for _ in range(5):
        ours.zero_grad()
        for p, q in zip(params, wide):
            p.grad.add_(torch.randn(p.shape, generator=g).cuda())
            q.grad = p.grad.double()
        torch.nn.utils.clip_grad_norm_(wide, 1.0)
        ours.step()
        theirs.step()
    assert ours.count.item() == 5
    ours.close()
    for p, q in zip(params, wide):
        assert bool(((p.double() - q).abs() <= 2e-6).all())
