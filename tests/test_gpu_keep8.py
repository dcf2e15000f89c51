"""8-bit checkpoints on the GPU: codes, scales and loaded values equal the definition's, bit for bit."""
import numpy as np
import pytest
import torch

import gated_ref as R
import paper_2303_11257_amd as us
from gpu_util import DEV, ptr, stream, to_dev, to_np

pytestmark = pytest.mark.gpu


def store(x, ld, rows, n):
    """x: [rows, ld] FP16 device tensor; guard rows behind the outputs are checked."""
    nb = us.keep8_blocks(n)
    codes = torch.full((rows + 1, n), 77, dtype=torch.int8, device=DEV)
    scales = torch.full(((rows + 1) * nb,), 77, dtype=torch.uint8, device=DEV)
    us.keep8_store(ptr(x), ld, ptr(codes), ptr(scales), rows, n, stream())
    c, s = to_np(codes), to_np(scales)
    assert (c[rows] == 77).all() and (s[rows * nb:] == 77).all()
    return codes, scales, c[:rows], s[: rows * nb].reshape(rows, nb)


def values(rows, ld, seed):
    r = np.random.default_rng(seed)
    x = r.standard_normal((rows, ld)) * np.exp2(r.integers(-28, 18, (rows, 1)).astype(np.float64)) * np.exp(r.standard_normal((1, ld)))
    x[r.random((rows, ld)) < 0.02] = 0.0
    with np.errstate(over="ignore"):
        return x.astype(np.float16)


@pytest.mark.parametrize("rows,n,ld", [(1, 16, 16), (3, 16, 24), (1, 48, 48), (65, 1040, 1040), (257, 2048, 2056), (31, 4112, 8192), (70000, 32, 32), (5, 16384, 16384)])
def test_codes_scales_and_values(rows, n, ld):
    x = values(rows, ld, rows + n)
    t = to_dev(x)
    codes, scales, c, s = store(t, ld, rows, n)
    ec, es = R.keep8(x[:, :n].astype(np.float64))
    assert np.array_equal(s, es) and np.array_equal(c, ec)
    back = torch.full((rows + 1, ld), 7.0, dtype=torch.float16, device=DEV)
    us.keep8_load(ptr(codes), ptr(scales), ptr(back), ld, rows, n, stream())
    b = to_np(back)
    assert np.array_equal(b[:rows, :n].astype(np.float64), R.keep8_values(ec, es))
    assert (b[rows:] == 7).all() and (b[:, n:] == 7).all()                     # the columns between n and the row pitch, the rows behind


def test_every_fp16_value_and_specials():
    bits = np.arange(65536, dtype=np.uint16).view(np.float16)
    lone = np.zeros((65536, 32), dtype=np.float16)                             # each value as the largest of its block, beside a small one
    lone[:, 7] = bits
    lone[:, 19] = np.float16(2.0 ** -20)
    rows = np.concatenate([lone, bits.reshape(-1, 32), np.random.default_rng(1).permutation(bits).reshape(-1, 32)])
    codes, scales, c, s = store(to_dev(rows), 32, len(rows), 32)
    ec, es = R.keep8(rows.astype(np.float64))
    assert np.array_equal(s, es) and np.array_equal(c, ec)
    back = torch.empty((len(rows), 32), dtype=torch.float16, device=DEV)
    us.keep8_load(ptr(codes), ptr(scales), ptr(back), 32, len(rows), 32, stream())
    assert np.array_equal(to_np(back).astype(np.float64), R.keep8_values(ec, es), equal_nan=True)


def test_captured_and_replayed_on_another_stream():
    rows, n = 130, 528
    x = torch.zeros((rows, n), dtype=torch.float16, device=DEV)
    codes = torch.empty((rows, n), dtype=torch.int8, device=DEV)
    scales = torch.empty((rows, us.keep8_blocks(n)), dtype=torch.uint8, device=DEV)
    back = torch.empty_like(x)
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    us.keep8_store(ptr(x), n, ptr(codes), ptr(scales), rows, n, st.cuda_stream)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=st):
        us.keep8_store(ptr(x), n, ptr(codes), ptr(scales), rows, n, torch.cuda.current_stream().cuda_stream)
        us.keep8_load(ptr(codes), ptr(scales), ptr(back), n, rows, n, torch.cuda.current_stream().cuda_stream)
    for k in range(4):
        v = values(rows, n, 50 + k)
        x.copy_(to_dev(v))
        graph.replay()
        ec, es = R.keep8(v.astype(np.float64))
        assert np.array_equal(to_np(back).astype(np.float64), R.keep8_values(ec, es), equal_nan=True)


def test_the_error_of_a_value_is_within_the_stated_bound():
    """Every finite FP16 value as the largest of its block, next to values at the codes' borders (a half, one and a half ... steps of either candidate)."""
    bits = np.arange(65536, dtype=np.uint16).view(np.float16)
    big = np.abs(bits[np.isfinite(bits)]).astype(np.float64)
    x = np.concatenate([big[:, None] * np.array([1.0] + [k / 127.5 * h for k in (0.5, 1.0, 1.5, 63.5, 64.5, 126.5) for h in (0.5, 1.0, -1.0)])[None], np.zeros((len(big), 13))], 1)
    x = np.where(np.abs(x) <= big[:, None], x, big[:, None]).astype(np.float16)
    codes, scales, c, s = store(to_dev(x), 32, len(x), 32)
    back = torch.empty((len(x), 32), dtype=torch.float16, device=DEV)
    us.keep8_load(ptr(codes), ptr(scales), ptr(back), 32, len(x), 32, stream())
    x = x.astype(np.float64)
    off, most = np.abs(to_np(back).astype(np.float64) - x), np.abs(x).max(1)
    clipped = np.abs(x) > 127.5 * 512
    half = np.exp2(s.astype(np.float64) - 128.0)
    assert (off <= half)[~clipped].all() and (off[clipped] <= 480).all() and clipped.any()
    small = most < 127.5 * 2.0 ** -24
    assert (half[:, 0] <= most / 127.5)[~small].all() and (half[:, 0] == most / 127.5).any() and (off[small] == 0).all()
