"""What the backward pass of attention over another sequence's keys asks for: 16 bytes for each query row, and parts only where workgroups are few."""
import pytest

import paper_2303_11257_amd as us


@pytest.mark.parametrize("batch,heads,kv,sq,sk,dh", [(64, 512, 512, 1, 64, 32), (65535, 64, 64, 1, 1, 16), (4096, 16, 4, 3, 100, 128), (64, 256, 256, 33, 40, 64)])
def test_sixteen_bytes_a_row(batch, heads, kv, sq, sk, dh):
    rows = batch * heads * sq
    assert 16 * rows <= us.attention_cross_workspace_bytes(batch, heads, kv, sq, sk, dh) <= 16 * rows + 4096
