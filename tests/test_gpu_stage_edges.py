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
