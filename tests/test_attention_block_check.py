"""The example's own check of attention (no GPU): outputs that are not finite do not pass."""
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def checks():
    """The `check` of examples/attention_block.py, in a scope of its own, with its plain attention."""
    with open(os.path.join(ROOT, "examples", "attention_block.py")) as f:
        src = f.read()
    plain = re.search(r"^def plain\(.*?(?=\n\n\ndef )", src, re.S | re.M).group(0)
    check = re.search(r"^    def check\(.*?(?=\n\n)", src, re.S | re.M).group(0)
    scope = {"torch": torch, "HEADS": 4, "KV_HEADS": 2, "HEAD_DIM": 8}
    imports = "\n".join(l for l in src.splitlines() if re.fullmatch(r"import (math|os|sys)", l))
    exec(imports + "\n" + plain + "\n\ndef make(kept, window, sinks):\n    worst = 0.0\n\n" + check
         + "\n\n    return check, lambda: worst", scope)
    return scope["make"], scope["plain"]


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("first", [True, False])
def test_outputs_that_are_not_finite_are_refused(bad, first):
    make, plain = checks()
    check, worst = make([[], []], 0, 0)
    gen = torch.Generator().manual_seed(0)
    qkv = torch.randn((3, 8, 8), generator=gen)
    good = plain(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], 0, 0)
    if not first:
        check(0, qkv, good + 1e-3)
        assert 0 < worst() < 0.1
    broken = good.clone()
    broken[1, 2, 3] = bad
    with pytest.raises(FloatingPointError):
        check(1, qkv, broken)
