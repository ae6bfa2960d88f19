"""The example that runs prompts and decode steps of an attention block."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
def test_attention_block(window, sinks):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import attention_block
    # 8-bit keys and values: half a step of a row's largest magnitude / 127, uniform, and that magnitude is at most
    # sqrt(128) of the row's rms: 0.026 of the rms at worst, once through the weights and once through the values
    error, _ = attention_block.run(lengths=(300, 77, 1), steps=8, window=window, sinks=sinks)
    assert 0 < error <= 0.05
