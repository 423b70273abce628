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
