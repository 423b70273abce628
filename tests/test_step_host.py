"""Layer norm and optimizer's step without a GPU: the plain forms the GPU tests compare with, the table of tensors, the thresholds."""
import ctypes
import math
import os
import re

import pytest
import torch

import paper_2206_01299_b200 as aq
from paper_2206_01299_b200 import binding
from tests import step_forms as forms
from tests.test_stage_binding import OnDevice, Recorder

F64 = torch.float64
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "aq_b200.h")


def test_calls_without_a_handle_are_refused():
    L = aq.lib()
    assert L.aq_layer_norm(None, None, 1, None, 1, None, None, 0.0, 1, 1, None, 1, None, 1, None, None) == aq.AQ_EINVAL
    assert L.aq_layer_norm_grad(None, None, 1, None, 1, None, 1, None, None, None, 1, 1, None, 1, None, None) == aq.AQ_EINVAL
    assert L.aq_grad_norm(None, None, 0, 1.0, 0.0, None, None, None) == aq.AQ_EINVAL
    assert L.aq_adamw(None, None, None, 0, None, None, None) == aq.AQ_EINVAL


@pytest.mark.parametrize("struct,name", [(aq.AdamTensor, "aq_adam_tensor"), (aq.AdamwConfig, "aq_adamw_config")])
def test_structures_have_the_headers_fields(struct, name):
    text = re.sub(r"/\*.*?\*/", " ", open(HEADER).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} " + name + ";", text).group(1)
    fields = re.findall(r"\*?\b(\w+)\s*(?=[,;])", body)
    assert fields == [f for f, _ in struct._fields_]
    assert ctypes.sizeof(aq.AdamTensor) == 72 and ctypes.sizeof(aq.AdamwConfig) == 48


# ---- plain forms ---------------------------------------------------------------------------------------------

def test_plain_layer_norm_by_hand():
    # 1, 3: mean 2, variance 1
    y, mean, rstd = forms.layer_norm(torch.tensor([[1.0, 3.0]], dtype=F64), torch.tensor([2.0, 5.0], dtype=F64), torch.tensor([0.5, -1.0], dtype=F64), 0.0)
    assert mean.item() == 2 and rstd.item() == 1 and y.tolist() == [[-1.5, 4.0]]


def test_plain_layer_norm_gradient_against_differences():
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, dtype=F64)  # noqa: E731
    s, w, b, dy, dsum, h = r(4, 7), r(7), r(7), r(4, 7), r(4, 7), 1e-5
    _, mean, rstd = forms.layer_norm(s, w, b, 1e-3)
    grads = dict(zip(("s", "w", "b"), forms.layer_norm_grad(dy, dsum, s, w, mean, rstd)))
    args = {"s": s, "w": w, "b": b}
    for name, x in args.items():
        u = torch.randn(x.shape, generator=g, dtype=F64)

        def f(t):
            a = dict(args, **{name: x + t * u})
            return ((forms.layer_norm(a["s"], a["w"], a["b"], 1e-3)[0] * dy).sum() + (a["s"] * dsum).sum()).item()
        assert abs((f(h) - f(-h)) / (2 * h) - (grads[name] * u).sum().item()) < 1e-7


def test_plain_step_agrees_with_torch():
    g = torch.Generator().manual_seed(4)
    p = torch.randn(50, generator=g, dtype=F64)
    q = p.clone().requires_grad_(True)
    adam = torch.optim.AdamW([q], lr=1e-2, weight_decay=0.1)
    m = v = torch.zeros(50, dtype=F64)
    for step in range(1, 6):
        grad = torch.randn(50, generator=g, dtype=F64)
        q.grad = grad.clone()
        adam.step()
        p, m, v = forms.adamw(p, grad, m, v, 1e-2, 0.1, step)
    assert torch.allclose(p, q.detach(), rtol=1e-12, atol=1e-14)


@pytest.mark.parametrize("kind,dtype", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_stored_moments_are_values_of_the_format_next_to_the_moment(kind, dtype):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(1000, generator=g) * torch.exp(6 * torch.randn(1000, generator=g))
    x = x if kind == "e4m3" else x.abs()
    below, scale = forms.store8(x, torch.zeros(1000, dtype=F64), kind)
    above, _ = forms.store8(x, torch.full((1000,), 65535.0, dtype=F64), kind)
    for z in (below, above):
        assert torch.equal(z, z.to(torch.float32).to(dtype).double())       # every one is a number of the format
    mag = x.double().abs() / scale.repeat_interleave(256)[:1000]
    # a threshold of 65535 leaves out places below a 65536th of the distance, which is at most mag / 4 or that of the subnormal numbers
    bits, low, _ = forms.FORMATS[kind]
    assert bool((above.abs() >= mag - torch.maximum(mag / 4, torch.tensor(2.0 ** (low - bits), dtype=F64)) / 65536).all())
    lower = below.abs() <= mag
    if kind == "e5m2":                                                       # what would vanish is held at the smallest value
        lower |= below == 2.0 ** -16
    assert bool(lower.all())
    for c, s in zip(x.double().abs().split(256), scale.tolist()):
        top = 1.75 * 2.0 ** forms.FORMATS[kind][2]
        assert top / 2 < c.max().item() / s <= top


def test_random_numbers_are_spread_evenly():
    """Of 64 elements over 4096 steps, and of 4096 elements at 64 steps: counts in 64 bins of an expected 64 each have a
    chi-square of 63 degrees of freedom, whose mean over 64 such rows is within 63 +- 4 sqrt(126 / 64) = 5.6; numbers of successive
    steps and of neighbouring elements have no correlation beyond 4 / sqrt(64 * 4096) = 0.008."""
    for rows in ([forms.random(64, t) for t in range(1, 4097)], [forms.random(4096, 1000 + t) for t in range(64)]):
        for which in (0, 1):
            x = torch.stack([r[which] for r in rows]) / 65536
            if x.shape[0] == 4096:
                x = x.T
            bins = torch.stack([torch.histc(r, 64, 0, 1) for r in x])
            assert abs(((bins - 64).square() / 64).sum(1).mean().item() - 63) < 5.6
            assert abs(torch.corrcoef(torch.stack([x[:, :-1].flatten(), x[:, 1:].flatten()]))[0, 1].item()) < 0.008
    lower, upper = forms.random(1, 1)
    k = 0x9E3779B9
    k = (k ^ k >> 16) * 0xBB67AE85 % 2 ** 32
    k = (k ^ k >> 15) * 0x9E3779B9 % 2 ** 32
    k ^= k >> 16
    u = k * 0xBB67AE85 % 2 ** 32
    u = (u ^ u >> 15) * 0x9E3779B9 % 2 ** 32
    u ^= u >> 16
    assert (lower.item(), upper.item()) == (u % 65536, u // 65536)


def test_stored_second_moment_follows_its_mean():
    """A v that falls by a thousandth per step, a hundredth of the format's distance: rounded to the nearest it would stay; here its mean
    follows.  A step adds a variance of at most place (1 - place) distance^2 <= 0.001 v * v / 4, which falls with v^2 as it is carried on: after n steps
    at most n * 0.00025 v^2, 0.375 v^2 after 1500.  The mean of 4096 elements is therefore within 4 sqrt(0.375 / 4096) = 0.038 of its place."""
    v = torch.linspace(0.5, 1.7, 4096)
    start = v.double().clone()
    for step in range(1, 1501):
        _, new = forms.moments32(torch.zeros(4096), torch.zeros(4096), v)
        z, scale = forms.store8(new, forms.random(4096, step)[1], "e5m2")
        v = (z * scale.repeat_interleave(256)).float()
    assert abs(v.double().mean() / (start * 0.999 ** 1500).mean() - 1) < 0.038


# ---- the wrappers --------------------------------------------------------------------------------------------

class Flat(OnDevice):
    """Stands for a contiguous CUDA tensor of n elements at an address."""

    def __init__(self, dtype, n, at):
        super().__init__(dtype)
        self.n, self.at = n, at

    def numel(self):
        return self.n

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def data_ptr(self):
        return self.at


@pytest.fixture
def stage(monkeypatch):
    recorder = Recorder()
    monkeypatch.setattr(binding, "_lib", recorder)
    st = aq.aq_stage_create()
    aq.aq_stage_configure(st, aq.AQ_DTYPE, aq.AQ_BF16)
    yield st, recorder
    aq.aq_stage_destroy(st)


def columns(narrow, n=300):
    b, f, blocks = torch.bfloat16, torch.float32, 2
    out = dict(params=[Flat(b, n, 1 << 20)], grads=[Flat(b, n, 2 << 20)], masters=[Flat(f, n, 3 << 20)],
               m=[Flat(torch.float8_e4m3fn if narrow else f, n, 4 << 20)], v=[Flat(torch.float8_e5m2 if narrow else f, n, 5 << 20)])
    if narrow:
        out.update(m_scale=[Flat(f, blocks, 6 << 20)], v_scale=[Flat(f, blocks, 7 << 20)])
    return out


@pytest.mark.parametrize("narrow", [False, True])
def test_table_of_tensors(stage, narrow):
    st, recorder = stage
    c = columns(narrow)
    t = aq.aq_adam_table(st, weight_decay=0.5, **c)
    assert t[0].numel == 300 and t[0].weight_decay == 0.5 and t[0].grad_dtype == aq.AQ_BF16 and t[0].param == 1 << 20 and t[0].v == 5 << 20
    assert t[0].m_scale == (6 << 20 if narrow else None)
    t = aq.aq_adam_table(st, **dict(c, grads=[Flat(torch.float32, 300, 2 << 20)]), weight_decay=[0.25])
    assert t[0].grad_dtype == aq.AQ_FP32 and t[0].weight_decay == 0.25
    aq.aq_adamw(st, aq.AdamwConfig(), t, 1, None, None, None)
    assert recorder.calls[-1] == "aq_adamw"
    with pytest.raises(AssertionError):
        aq.aq_adamw(st, aq.AdamwConfig(), t, 2, None, None, None)            # more than the array has
    for name, column in c.items():
        x = column[0]
        wrong = [Flat(torch.float64, x.n, x.at), Flat(x.dtype, x.n + 256, x.at), torch.zeros(x.n, dtype=x.dtype)]
        for y in wrong:
            with pytest.raises((AssertionError, KeyError)):
                aq.aq_adam_table(st, **dict(c, **{name: [y]}))
    with pytest.raises(AssertionError):
        aq.aq_adam_table(st, **dict(c, m=c["m"] * 2))


def test_a_tensor_listed_twice_is_refused(stage):
    st, _ = stage
    c = {n: x * 2 for n, x in columns(False).items()}
    with pytest.raises(AssertionError, match="overlap"):
        aq.aq_adam_table(st, **c)
    aq.aq_adam_table(st, grads=c["grads"])                                   # reading one twice is no race


T, F, L = "operand", torch.float32, torch.int64
CALLS = {
    "aq_layer_norm": [T, 8, T, 8, T, T, 1e-5, 8, 8, T, 8, T, 8, F, F],
    "aq_layer_norm_grad": [T, 8, T, 8, T, 8, T, F, F, 8, 8, T, 8, F, F],
    "aq_grad_norm": [1 << 20, 1, 1.0, 0.0, F, F, L],
    "aq_adamw": ["config", 1 << 20, 1, F, F, L],
}


@pytest.mark.parametrize("name", CALLS)
def test_operands_of_another_type_or_place_are_refused(stage, name):
    st, recorder = stage
    good = [OnDevice(torch.bfloat16) if k is T else aq.AdamwConfig() if k == "config" else OnDevice(k) if isinstance(k, torch.dtype) else k
            for k in CALLS[name]]
    getattr(aq, name)(st, *good)
    assert recorder.calls[-1] == name
    for at, x in enumerate(good):
        if not isinstance(x, OnDevice):
            continue
        others = {torch.float16, torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64} - {x.dtype}
        for wrong in [OnDevice(t) for t in others] + [torch.zeros((8, 8), dtype=x.dtype), OnDevice(x.dtype, contiguous=False)]:
            with pytest.raises(AssertionError):
                getattr(aq, name)(st, *good[:at], wrong, *good[at + 1:])
        getattr(aq, name)(st, *good[:at], None, *good[at + 1:])


def test_clip_form():
    assert forms.clip([torch.tensor([3.0]), torch.tensor([4.0])], 0.5, 0.0) == (2.5, 0.5)
    n, f = forms.clip([torch.tensor([3.0, 4.0])], 1.0, 1.0)
    assert n == 5 and abs(f - 0.2) < 1e-6 and math.isnan(forms.clip([torch.tensor([math.inf])], 1.0, 1.0)[1])
