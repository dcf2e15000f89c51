"""What attention over the cache adds to accumulators that a long generation has made large; cases and definition are those of tests/test_gpu_cache.py."""
import pytest
import torch

from test_gpu_cache import Paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,heads,kv,max_len", [([100, 37], 16, 1, 100), ([1000, 3, 500], 32, 2, 1024), ([100, 37], 16, 1, 1100), ([40], 20, 1, 40)], ids=str)
def test_large_accumulators(lens, heads, kv, max_len, fp8):
    """Accumulators of 1e4 take sums of sixteen p of about 1/100: one rounding at their size (2^-24, which the bound allows), not one for each head."""
    c = Paged(lens, heads, kv, 64, 16, fp8, seed=9, wide=-(-max_len // 16), max_len=max_len)
    c.W = c.W * 1e4
    c.dev["W"].copy_(c.W)
    c.run()
    c.check()


@pytest.mark.parametrize("fp8", [False, True])
def test_the_bound_on_the_lengths_does_not_change_weights(fp8):
    """As many sequences as leave each key head one workgroup: up to 1024 positions it adds the weights itself, beyond them another launch does; the same bits."""
    got = []
    for max_len in (1024, 1025):
        c = Paged([(b * 53) % 300 for b in range(70)], 4 * 16, 16, 16, 16, fp8, seed=4, wide=65, max_len=max_len)
        c.W = c.W * 100
        c.dev["W"].copy_(c.W)
        c.run()
        torch.cuda.synchronize()
        got.append((c.dev["W"].clone(), c.O.clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
