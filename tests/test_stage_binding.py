"""What the Python wrappers of the stage operators refuse before the library is called: element types, CPU tensors, layouts."""
import pytest
import torch

from paper_2206_01299_b200 import binding as aq


class Recorder:
    """In the library's place: notes the calls' names and answers 0."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            return 4242 if name == "aq_stage_create" else 0
        return call


class OnDevice:
    """Stands for a CUDA tensor, with what the wrappers ask of one."""

    device, is_cuda, shape = "cuda:0", True, (8, 8)

    def __init__(self, dtype, contiguous=True):
        self.dtype, self._contiguous = dtype, contiguous

    def is_contiguous(self):
        return self._contiguous

    def stride(self, dim=None):
        return 1 if self._contiguous else 2

    def data_ptr(self):
        return 1 << 20


T, I, F = "operand", torch.int32, torch.float32
CALLS = {  # the operands' types; N stands for the numbers between them
    "aq_token_logprobs": [T, "N", "N", "N", I, "N", "N", F, F, F, I, F],
    "aq_token_logprobs_grad": [T, "N", "N", "N", I, "N", F, F, F, F, T, "N"],
    "aq_gated_ffn": [T, "N", T, T, "N", "N", "N", "N", "N", T, "N", T, T, "N"],
    "aq_gated_ffn_grad": [T, "N", T, "N", T, T, "N", T, T, "N", "N", "N", "N", "N", T, "N", T, T, "N"],
    "aq_qk_norm_rope": ["S", "N", T, "N", T, "N", T, T, F, I, T, "N", T, "N"],
    "aq_qk_norm_rope_grad": ["S", "N", T, "N", T, "N", T, "N", T, "N", T, T, F, I, T, "N", T, "N", F, F],
}


@pytest.fixture
def stage(monkeypatch):
    recorder = Recorder()
    monkeypatch.setattr(aq, "_lib", recorder)
    st = aq.aq_stage_create()
    yield st, recorder
    aq.aq_stage_destroy(st)


def arguments(kinds, operand):
    return [8 if k == "N" else aq.QkShape() if k == "S" else OnDevice(operand if k is T else k) for k in kinds]


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("key,operand", [(aq.AQ_FP16, torch.float16), (aq.AQ_BF16, torch.bfloat16), (aq.AQ_FP32, torch.float32)])
def test_operands_of_another_type_or_place_are_refused(stage, name, key, operand):
    st, recorder = stage
    if key != aq.AQ_FP16:
        aq.aq_stage_configure(st, aq.AQ_DTYPE, key)
    good = arguments(CALLS[name], operand)
    getattr(aq, name)(st, *good)
    assert recorder.calls[-1] == name
    n = len(recorder.calls)
    for at, x in enumerate(good):
        if not isinstance(x, OnDevice):
            continue
        others = {torch.float16, torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64} - {x.dtype}
        for wrong in [OnDevice(t) for t in others] + [torch.zeros((8, 8), dtype=x.dtype), OnDevice(x.dtype, contiguous=False)]:
            with pytest.raises(AssertionError):
                getattr(aq, name)(st, *good[:at], wrong, *good[at + 1:])
        for fine in (None, 1 << 20):
            getattr(aq, name)(st, *good[:at], fine, *good[at + 1:])
            n += 1
        assert len(recorder.calls) == n, (name, at)


def test_a_handle_starts_with_fp16_and_forgets_its_type(stage):
    st, _ = stage
    aq.aq_stage_configure(st, aq.AQ_DTYPE, aq.AQ_BF16)
    aq.aq_stage_destroy(st)
    again = aq.aq_stage_create()
    aq.aq_gated_ffn(again, *arguments(CALLS["aq_gated_ffn"], torch.float16))
    with pytest.raises(AssertionError):
        aq.aq_gated_ffn(again, *arguments(CALLS["aq_gated_ffn"], torch.bfloat16))


def test_a_handle_made_past_the_wrappers_takes_any_type_but_no_cpu_tensor(stage):
    _, recorder = stage
    good = arguments(CALLS["aq_gated_ffn"], torch.bfloat16)
    aq.aq_gated_ffn(77, *good)
    assert recorder.calls[-1] == "aq_gated_ffn"
    with pytest.raises(AssertionError):
        aq.aq_gated_ffn(77, torch.zeros((8, 8), dtype=torch.bfloat16), *good[1:])
