"""The stage operators, the codec and torch's chain rule together: the two-stage example learns."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_two_stages_learn_a_small_language():
    spec = importlib.util.spec_from_file_location("finetune_two_stages", os.path.join(ROOT, "examples", "finetune_two_stages.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses = example.train(epochs=12, say=lambda *_: None)
    # the first loss is that of near-uniform guesses, ln 96 and what random logits add (about half their variance)
    assert abs(losses[0] - math.log(example.VOCAB)) < 1.0
    assert sum(losses[-4:]) / 4 < 0.75 * losses[0]
