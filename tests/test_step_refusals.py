"""What the calls of the optimizer's step refuse, and what the wrappers refuse before them.  The library's checks come before its first CUDA
call and read nothing of a handle but its element type, so a zeroed block (binary16) stands for a handle here, and addresses for tensors."""
import ctypes

import pytest
import torch

import paper_2206_01299_b200 as aq
from paper_2206_01299_b200 import binding
from tests.test_stage_binding import Recorder
from tests.test_step_host import Flat

no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that passes the checks has to end at the missing device")


@pytest.fixture
def handle():
    block = ctypes.create_string_buffer(4096)
    yield ctypes.addressof(block)


def one_tensor(**change):
    table = (aq.AdamTensor * 1)()
    for name in ("param", "grad", "m", "v"):
        setattr(table[0], name, 1 << 20)
    table[0].numel, table[0].grad_dtype = 300, aq.AQ_FP16
    for name, x in change.items():
        setattr(table[0], name, x)
    return table


def config(bits):
    return aq.AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, state_bits=bits)


@no_device
@pytest.mark.parametrize("scales", [dict(m_scale=1 << 20, v_scale=1 << 20), dict(m_scale=1 << 20), dict(v_scale=1 << 20)])
def test_a_table_of_8_bit_moments_is_refused_with_32(handle, scales):
    """Its codes would be read and written as binary32, four times their size."""
    L = aq.lib()
    assert L.aq_adamw(handle, ctypes.byref(config(32)), one_tensor(**scales), 1, None, None, None) == aq.AQ_EINVAL
    assert b"tensor 0" in L.aq_stage_last_error(handle) and b"m_scale" in L.aq_stage_last_error(handle)
    assert L.aq_adamw(handle, ctypes.byref(config(32)), one_tensor(numel=0, **scales), 1, None, None, None) == aq.AQ_OK      # nothing to read
    # what fits passes the checks
    assert L.aq_adamw(handle, ctypes.byref(config(32)), one_tensor(), 1, None, None, None) == aq.AQ_ECUDA
    assert L.aq_adamw(handle, ctypes.byref(config(8)), one_tensor(m_scale=1 << 20, v_scale=1 << 20), 1, None, None, None) == aq.AQ_ECUDA


@pytest.fixture
def stage(monkeypatch):
    recorder = Recorder()
    monkeypatch.setattr(binding, "_lib", recorder)
    st = aq.aq_stage_create()
    yield st, recorder
    aq.aq_stage_destroy(st)


def test_8_bit_moments_without_scales_are_refused(stage):
    st, _ = stage
    h, f = torch.float16, torch.float32
    c = dict(params=[Flat(h, 300, 1 << 20)], grads=[Flat(h, 300, 2 << 20)], m=[Flat(torch.float8_e4m3fn, 300, 4 << 20)], v=[Flat(torch.uint8, 300, 5 << 20)],
             m_scale=[Flat(f, 2, 6 << 20)], v_scale=[Flat(f, 2, 7 << 20)])
    assert aq.aq_adam_table(st, **c)[0].v_scale == 7 << 20
    for change in (dict(m_scale=[None]), dict(v_scale=[None]), dict(v_scale=None), dict(m_scale=[None], v_scale=[None])):
        with pytest.raises(AssertionError, match="scale"):
            aq.aq_adam_table(st, **dict(c, **change))
    empty = {n: [Flat(x[0].dtype, 0, 0)] for n, x in c.items()}
    aq.aq_adam_table(st, **dict(empty, m_scale=[None], v_scale=[None]))


def columns(t, grads, master=False):
    f = torch.float32
    out = dict(params=[Flat(t, 300, 1 << 20)], grads=[Flat(grads, 300, 2 << 20)], m=[Flat(f, 300, 4 << 20)], v=[Flat(f, 300, 5 << 20)])
    return dict(out, masters=[Flat(f, 300, 3 << 20)]) if master else out


TYPES = {aq.AQ_FP16: torch.float16, aq.AQ_BF16: torch.bfloat16, aq.AQ_FP32: torch.float32}


@pytest.mark.parametrize("laid_out", TYPES)
@pytest.mark.parametrize("taken", TYPES)
def test_a_table_of_another_element_type_is_refused(stage, laid_out, taken):
    """Binary32 gradients fit every handle, but the parameters' type is the handle's and stands nowhere in the array: 16-bit parameters would be
    taken for binary32 ones, twice their size."""
    st, recorder = stage
    aq.aq_stage_configure(st, aq.AQ_DTYPE, laid_out)
    table = aq.aq_adam_table(st, **columns(TYPES[laid_out], torch.float32))
    other = aq.aq_stage_create()
    for h in (st, other):
        aq.aq_stage_configure(h, aq.AQ_DTYPE, taken)
        n = len(recorder.calls)
        if laid_out == taken:
            aq.aq_adamw(h, config(32), table, 1, None, None, None)
            assert recorder.calls[n:] == ["aq_adamw"]
        else:
            with pytest.raises(aq.AqError) as e:
                aq.aq_adamw(h, config(32), table, 1, None, None, None)
            assert e.value.code == aq.AQ_EINVAL and str(TYPES[laid_out]) in str(e.value) and "aq_adamw" not in recorder.calls[n:]
        aq.aq_grad_norm(h, table, 1, 1.0, 1.0, None, None, None)              # the gradients' type is in the array
        assert recorder.calls[-1] == "aq_grad_norm"


def test_tables_whose_element_type_is_not_known_are_taken(stage):
    st, recorder = stage
    table = aq.aq_adam_table(77, **columns(torch.bfloat16, torch.float32))     # a handle that was not made by the wrappers
    aq.aq_adamw(st, config(32), table, 1, None, None, None)
    aq.aq_adamw(77, config(32), aq.aq_adam_table(st, **columns(torch.float16, torch.float32)), 1, None, None, None)
    aq.aq_adamw(st, config(32), (aq.AdamTensor * 1)(), 1, None, None, None)
    aq.aq_adamw(st, config(32), 1 << 20, 1, None, None, None)
    aq.aq_adamw(st, config(32), None, 0, None, None, None)
    grads = aq.aq_adam_table(st, grads=[Flat(torch.float32, 300, 2 << 20)])
    aq.aq_stage_configure(st, aq.AQ_DTYPE, aq.AQ_BF16)
    aq.aq_grad_norm(st, grads, 1, 1.0, 1.0, None, None, None)
    assert recorder.calls.count("aq_adamw") == 5 and recorder.calls[-1] == "aq_grad_norm"


@no_device
@pytest.mark.parametrize("inv_scale", [1e39, 3.5e38, 1e300, 1e-46, 5e-324])
def test_a_scale_outside_binary32_is_refused(handle, inv_scale):
    """The factor would be infinite or zero: a step that is counted but leaves the weights, or one without a gradient."""
    L = aq.lib()
    assert L.aq_grad_norm(handle, None, 0, inv_scale, 0.0, None, None, None) == aq.AQ_EINVAL
    assert b"inv_scale" in L.aq_stage_last_error(handle)
    for fine in (3.4e38, 1.0, 1e-38, 2e-45):
        assert L.aq_grad_norm(handle, None, 0, fine, 0.0, None, None, None) == aq.AQ_ECUDA


def test_a_tensor_without_a_gradient_is_refused(stage):
    st, _ = stage
    c = {n: x * 1 + [Flat(x[0].dtype, 300, x[0].at + (1 << 16))] for n, x in columns(torch.float16, torch.float16).items()}
    assert len(aq.aq_adam_table(st, **c)) == 2
    with pytest.raises(AssertionError, match="tensor 1 has no gradient"):
        aq.aq_adam_table(st, **dict(c, grads=[c["grads"][0], None]))
