"""The two-stage example's optimizer: every step is counted and every weight moves."""
import math

import pytest

from tests.test_gpu_step_example import example  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm,optimizer", [("rms", "adamw"), ("layer", "adamw"), ("layer", "adamw8")])
def test_every_weight_moves_and_every_step_counts(example, monkeypatch, norm, optimizer):  # noqa: F811
    made, finished = [], []

    class Watched(example.AdamW):
        def __init__(self, params, lr, state_bits):
            super().__init__(params, lr, state_bits)
            self.before = [p.detach().clone() for p in params]
            made.append(self)

        def close(self):
            finished.append((self.count.item(), self.factor.item(), self.norm.item()))
            super().close()

    monkeypatch.setattr(example, "AdamW", Watched)
    losses = example.train(epochs=2, say=lambda *_: None, norm=norm, optimizer=optimizer)
    (adam,), ((count, factor, norm_of_last),) = made, finished
    assert count == len(losses) and 0 < factor <= 1 and 0 < norm_of_last < math.inf
    assert all(p.grad is not None and bool((p.grad != 0).any()) for p in adam.params)
    moved = [int((p.detach() != q).sum()) / p.numel() for p, q in zip(adam.params, adam.before)]
    # Adam's first step moves a weight with a gradient by lr = 0.005, well above a rounding of weights of size 1
    assert all(x > 0.5 for x in moved), moved
    assert all(bool((m.float() != 0).any()) and bool((v.float() != 0).any()) for m, v in zip(adam.state["m"], adam.state["v"]))
