"""Calls of the optimizer's step that the documentation allows: betas of zero, a step's number below one, tensors off the grid of eight that
fill more than one launch, empty tensors at its end, one handle's calls in two captured graphs."""
import math

import pytest
import torch

from tests import step_forms as forms
from tests.stage_forms import TYPES
from tests.test_gpu_stage import E, set_type
from tests.test_gpu_step import Set, aq, close, laid_out, same, stage  # noqa: F401

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("beta1,beta2", [(0.0, 0.999), (0.9, 0.0), (0.0, 0.0), (0.5, 0.25)])
@pytest.mark.parametrize("on_device", [False, True])
def test_adamw_with_small_betas(aq, stage, bits, beta1, beta2, on_device):  # noqa: F811
    set_type(aq, stage, "fp32")
    s = Set([1000], "fp32", "fp32", bits, False, False, seed=51)
    before, step = s.snapshot(), 2
    m, v = forms.moments32(before["g"][0], *before["mv"][0], 1.0, beta1, beta2)
    count = torch.tensor([step], device="cuda") if on_device else None
    aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=beta1, beta2=beta2, eps=1e-8, step=0 if on_device else step, state_bits=bits), s.table(aq, stage), 1,
                None, None, count)
    if bits == 32:
        assert torch.equal(s.m[0].cpu(), m) and torch.equal(s.v[0].cpu(), v)
    else:
        um, uv = forms.random(1000, step)
        for name, x, u, kind in (("m", m, um, "e4m3"), ("v", v, uv, "e5m2")):
            z, scale = forms.store8(x, u, kind)
            assert torch.equal(getattr(s, name + "_scale")[0].cpu().double(), scale) and torch.equal(getattr(s, name)[0].cpu().double(), z)
    update = 1e-3 / (1 - beta1 ** step) * m.double() / (torch.sqrt(v.double() / (1 - beta2 ** step)) + 1e-8)
    want = before["p"][0] - update
    close(s.param[0], want, 24 * E * update.abs() + 2 * E * want.abs(), "param")


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("number", [0, -5, -2 ** 62])
def test_a_step_on_the_device_below_one_counts_as_one(aq, stage, bits, number):  # noqa: F811
    set_type(aq, stage, "bf16")
    one, two = (Set([777], "bf16", "bf16", bits, True, False, seed=52) for _ in range(2))
    c = lambda step: aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=step, state_bits=bits)  # noqa: E731
    aq.aq_adamw(stage, c(0), one.table(aq, stage), 1, None, None, torch.tensor([number], device="cuda"))
    aq.aq_adamw(stage, c(1), two.table(aq, stage), 1, None, None, None)
    for name in ("param", "master", "m", "v"):
        assert same(getattr(one, name)[0], getattr(two, name)[0]), name


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_more_tensors_off_the_grid_than_a_launch_takes(aq, stage, bits):  # noqa: F811
    """With 32-bit moments a tensor off the grid is two entries of a launch's 400; behind the last one lie empty ones."""
    set_type(aq, stage, "bf16")
    sizes = [(i * 37) % 700 for i in range(1203)] + [0] * 5
    s = Set(sizes, "bf16", "bf16", bits, True, True, seed=53)
    before = s.snapshot()
    aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=7, state_bits=bits), s.table(aq, stage), len(sizes), None, None, None)
    s.check(before, 1e-3, 7)
    s.check_between()


@pytest.mark.parametrize("n", [199, 200, 201, 399, 400, 401, 800])
@pytest.mark.parametrize("shift", [0, 1])
def test_grad_norm_of_as_many_tensors_as_launches_take(aq, stage, n, shift):  # noqa: F811
    """Exactly one launch, one more and one less, the last tensors empty; a gradient off the grid is two entries."""
    set_type(aq, stage, "fp16")
    g = torch.Generator().manual_seed(n)
    sizes = [20] * n + [0] * 3
    values = [torch.randn(k, generator=g).half() for k in sizes]
    parts = laid_out(sizes, TYPES["fp16"], shift, values)[1]
    norm, factor, step = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    aq.aq_grad_norm(stage, aq.aq_adam_table(stage, grads=parts), len(sizes), 0.5, 1.0, norm, factor, step)
    want = forms.clip(values, 0.5, 1.0)
    assert abs(norm.item() / want[0] - 1) < 6 * E and abs(factor.item() / want[1] - 1) < 7 * E and step.item() == 1


def test_two_captured_graphs_of_one_handle(aq, stage):  # noqa: F811
    """Norms and steps of two sets on one handle, captured apart and replayed in turn, do what eager calls do."""
    set_type(aq, stage, "fp16")
    sets = [[Set([3000, 77, 256], "fp16", "fp16", bits, True, False, seed=60 + bits) for bits in (32, 8)] for _ in range(2)]
    norm, factor = ([torch.zeros(1, device="cuda") for _ in range(4)] for _ in range(2))
    steps = [torch.zeros(1, dtype=torch.int64, device="cuda") for _ in range(4)]

    def call(s, i):
        table = s.table(aq, stage)
        aq.aq_grad_norm(stage, table, 3, 0.5, 0.1, norm[i], factor[i], steps[i])
        aq.aq_adamw(stage, aq.AdamwConfig(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, state_bits=s.bits), table, 3, factor[i], None, steps[i])
    graphs = []
    for i, s in enumerate(sets[0]):
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            aq.aq_stage_configure(stage, aq.AQ_STREAM, torch.cuda.current_stream().cuda_stream)
            try:
                call(s, i)
            finally:
                aq.aq_stage_configure(stage, aq.AQ_STREAM, 0)
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(5):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(sets[1]):
            call(s, 2 + i)
    torch.cuda.synchronize()
    for i, (s, t) in enumerate(zip(*sets)):
        assert steps[i].item() == steps[2 + i].item() == 5 and math.isfinite(norm[i].item()) and torch.equal(norm[i], norm[2 + i])
        for name in ("param", "master", "m", "v"):
            assert all(same(a, b) for a, b in zip(getattr(s, name), getattr(t, name))), name
    del graphs
