"""What holds for the sources of the layer norm and of the optimizer's step."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2206_01299_b200", "csrc")


@pytest.mark.parametrize("name", ["aq_layernorm.cu", "aq_adamw.cu", "aq_stage_device.cuh"])
def test_no_load_of_data_that_nothing_may_write(name):
    """Outputs may take the inputs' places, and a kernel may start while the one before still writes what it reads: neither goes with
    loads by way of the read-only path, whose data may not change while the kernel runs."""
    text = re.sub(r"//.*", "", open(os.path.join(CSRC, name)).read())
    assert not re.search(r"__ldg\b|\.nc\b|__restrict__", text)
