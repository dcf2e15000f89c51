"""The README's examples run as they stand, one after the other, and write results of about unit variance."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_examples_run():
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    names = {}
    for block in blocks:
        exec(compile(block, "README.md", "exec"), names)
        torch.cuda.synchronize()
        for n in ("Y", "dX"):
            v = float(names[n].double().square().mean())
            assert 0.5 < v < 2.0, (n, v)
    assert len(blocks) == 2 and names["dZ8"].shape == (names["T"], 2 * names["f"])
    for n in ("dWgu", "dWd", "dW1", "dW2"):
        v = float(names[n].double().square().mean())
        assert 0.5 < v < 2.0, (n, v)
