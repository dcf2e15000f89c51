"""The README's generation example runs after the others, as it stands."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_example_runs():
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```(?:python|py)\n(.*?)```", f.read(), re.S)
    assert len(blocks) == 3
    torch.manual_seed(0)
    names = {}
    for block in blocks:
        exec(compile(block, "README.md", "exec"), names)
        torch.cuda.synchronize()
    O, kept, weights = names["O"].double(), names["kept"], names["weights"]
    # queries and keys of unit variance share a row's weight unevenly: sum p^2 = e / n of 500 and more, so O's variance is near e
    assert 0.5 < float(O.square().mean()) < 4.0
    assert names["length"].tolist() == [names["keep"]] * names["batch"]
    assert bool((kept[:, :, 1:] > kept[:, :, :-1]).all()) and int(kept.min()) >= 0 and int(kept.max()) == names["prompt"] + 2
    # what three tokens of a key head's query heads gave out, less what the positions that went had
    mine = weights.sum((1, 2)).view(names["batch"], -1).sum(1)
    total = 3.0 * names["heads"]
    assert bool((mine < total).all()) and bool((mine > 0.8 * total).all())
