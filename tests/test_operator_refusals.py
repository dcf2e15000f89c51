"""Argument checks of the gated block, the 8-bit checkpoints and the head calls: on the host, before anything is launched, so they need no
GPU; and the definitions that the GPU tests compare with."""
import ctypes
import math

import numpy as np
import pytest
import torch

import gated_ref as R
import paper_2303_11257_amd as us

OK = 16          # an aligned address that no refused call touches


def fwd(T=16, d=16, f=16, gate=0, mode=0, **kw):
    a = dict(X=OK, Wgu=OK, Wd=OK, Z=OK, Zs=None, H=OK, Y=OK)
    a.update(kw)
    us.ffn_gated_fwd(*a.values(), T, d, f, gate, mode)


def bwd(T=16, d=16, f=16, gate=0, mode=0, ws=None, wsb=0, **kw):
    a = dict(X=OK, Wgu=OK, Wd=OK, Z=OK, Zs=None, H=OK, G=OK, dZ=OK, dX=OK, dWgu=OK, dWd=OK)
    a.update(kw)
    us.ffn_gated_bwd(*a.values(), T, d, f, gate, mode, ws, wsb)


def heads(batch=1, s=4, h=4, kv=2, dh=32, rot=32, pairs=0, eps=0.0, ld=None, **kw):
    a = dict(QKV=OK, ld=(h + 2 * kv) * dh if ld is None else ld, wq=OK, wk=OK, pos=None, freq=OK, Q=OK, K=OK, V=OK)
    a.update(kw)
    us.qk_norm_rope_fwd(*a.values(), batch, s, h, kv, dh, rot, pairs, eps)


def heads_back(batch=1, s=4, h=4, kv=2, dh=32, rot=32, pairs=0, eps=0.0, ld=256, ld_d=256, ws=OK, wsb=1 << 20, **kw):
    a = dict(QKV=OK, ld=ld, wq=OK, wk=OK, pos=None, freq=OK, dQ=OK, dK=OK, dV=OK, dQKV=OK, ld_d=ld_d, dwq=OK, dwk=OK)
    a.update(kw)
    us.qk_norm_rope_bwd(*a.values(), batch, s, h, kv, dh, rot, pairs, eps, 0.0, 0.0, ws, wsb)


NULL, SHAPE, ALIGN, DTYPE, WORKSPACE, VALUE = 1, 2, 3, 4, 5, 7
CASES = [(lambda n=n: fwd(**{n: None}), NULL) for n in ("X", "Wgu", "Wd", "H", "Y")]
CASES += [(lambda n=n: fwd(**{n: 24}), ALIGN) for n in ("X", "Wgu", "Wd", "Z", "H", "Y")]
CASES += [(lambda: fwd(mode=us.FFN_KEEP8, Z=None, Zs=OK), NULL), (lambda: fwd(mode=us.FFN_KEEP8), NULL), (lambda: fwd(mode=us.FFN_KEEP8, Zs=8), ALIGN),
          (lambda: fwd(mode=us.FFN_TABLES_READY), VALUE), (lambda: fwd(mode=8), VALUE), (lambda: fwd(gate=4), DTYPE), (lambda: fwd(gate=-1), DTYPE),
          (lambda: fwd(T=-1), SHAPE), (lambda: fwd(d=0), SHAPE), (lambda: fwd(f=0), SHAPE), (lambda: fwd(d=24), SHAPE), (lambda: fwd(f=8), SHAPE),
          (lambda: fwd(f=(1 << 20) + 16), SHAPE), (lambda: fwd(d=1 << 40), SHAPE)]
CASES += [(lambda n=n: bwd(**{n: None}), NULL) for n in ("X", "Wgu", "Wd", "Z", "H", "G", "dZ")]
CASES += [(lambda n=n: bwd(**{n: 24}), ALIGN) for n in ("X", "Wgu", "Wd", "Z", "H", "G", "dZ", "dX", "dWgu", "dWd")]
CASES += [(lambda: bwd(mode=us.FFN_KEEP8), NULL), (lambda: bwd(mode=16), VALUE), (lambda: bwd(gate=9), DTYPE), (lambda: bwd(T=-5), SHAPE), (lambda: bwd(f=40), SHAPE),
          # 64 tiles of grad_W over 4096 tokens: slices, so a workspace is needed
          (lambda: bwd(T=4096, d=512, f=2048), WORKSPACE), (lambda: bwd(T=4096, d=512, f=2048, ws=OK, wsb=us.TABLE_AREA_BYTES), WORKSPACE)]
CASES += [(lambda: us.keep8_store(OK, 32, OK, OK, 1, 24), SHAPE), (lambda: us.keep8_store(OK, 16, OK, OK, 1, 32), SHAPE), (lambda: us.keep8_store(OK, 36, OK, OK, 1, 32), SHAPE),
          (lambda: us.keep8_store(OK, 32, OK, OK, -1, 32), SHAPE), (lambda: us.keep8_store(None, 32, OK, OK, 1, 32), NULL), (lambda: us.keep8_store(OK, 32, None, OK, 1, 32), NULL),
          (lambda: us.keep8_store(OK, 32, OK, None, 1, 32), NULL), (lambda: us.keep8_store(8, 32, OK, OK, 1, 32), ALIGN), (lambda: us.keep8_load(OK, 8, OK, 32, 1, 32), ALIGN),
          (lambda: us.keep8_load(OK, OK, None, 32, 1, 32), NULL), (lambda: us.keep8_load(OK, OK, OK, 31, 1, 32), SHAPE), (lambda: us.keep8_load(8, OK, OK, 32, 1, 32), ALIGN),
          (lambda: us.keep8_store(OK, 1 << 40, OK, OK, 1, 1 << 40), SHAPE)]
CASES += [(lambda n=n: heads(**{n: None}), NULL) for n in ("QKV", "freq", "Q", "K", "V")]
CASES += [(lambda n=n: heads(**{n: 8}), ALIGN) for n in ("QKV", "wq", "wk", "Q", "K", "V")]
CASES += [(lambda: heads(pos=2), ALIGN), (lambda: heads(freq=4), ALIGN), (lambda: heads(ld=255), SHAPE), (lambda: heads(ld=260), SHAPE), (lambda: heads(h=4, kv=3), SHAPE),
          (lambda: heads(h=0), SHAPE), (lambda: heads(kv=0), SHAPE), (lambda: heads(h=70000, kv=1), SHAPE), (lambda: heads(dh=24), SHAPE), (lambda: heads(dh=272), SHAPE),
          (lambda: heads(rot=8), SHAPE), (lambda: heads(rot=48), SHAPE), (lambda: heads(rot=-16), SHAPE), (lambda: heads(batch=-1), SHAPE), (lambda: heads(s=-1), SHAPE),
          (lambda: heads(s=1 << 31), SHAPE), (lambda: heads(pairs=2), VALUE), (lambda: heads(eps=-1.0), VALUE), (lambda: heads(eps=float("nan")), VALUE)]
CASES += [(lambda n=n: heads_back(**{n: None}), NULL) for n in ("QKV", "freq", "dQ", "dK", "dV", "dQKV")]
CASES += [(lambda n=n: heads_back(**{n: 8}), ALIGN) for n in ("QKV", "wq", "wk", "dQ", "dK", "dV", "dQKV", "ws")]
CASES += [(lambda: heads_back(dwq=17), ALIGN), (lambda: heads_back(dwk=17), ALIGN), (lambda: heads_back(ld_d=248), SHAPE), (lambda: heads_back(ld=248), SHAPE),
          (lambda: heads_back(ws=None), WORKSPACE), (lambda: heads_back(wsb=16), WORKSPACE), (lambda: heads_back(eps=-0.5), VALUE)]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_refused_before_anything_is_launched(i):
    call, status = CASES[i]
    with pytest.raises(us.UsError) as e:
        call()
    assert e.value.status == status


def test_nothing_to_do_is_no_error():
    us.ffn_gated_fwd(None, None, None, None, None, None, None, 0, 16, 16)
    us.keep8_store(None, 32, None, None, 0, 32)
    us.keep8_load(None, None, None, 0, 5, 0)
    heads(batch=0)
    heads_back(s=0)


def test_sizes_and_factors():
    assert [us.keep8_blocks(n) for n in (-3, 0, 1, 32, 33, 4096)] == [0, 0, 1, 1, 2, 128]
    assert [us.lib().us_keep8_blocks(n) for n in (-3, 0, 1, 32, 33, 4096)] == [0, 0, 1, 1, 2, 128]
    assert us.ffn_gated_workspace_bytes(0, 16, 16) == 0 and us.qk_norm_rope_workspace_bytes(1, 0, 1, 1, 16) == 0
    assert us.ffn_gated_workspace_bytes(4096, 512, 2048) >= us.workspace_bytes(4096, 512, 4096)
    assert us.ffn_gated_workspace_bytes(4096, 512, 2048) >= us.workspace_bytes(4096, 2048, 512)
    z = (torch.arange(400000, dtype=torch.float64) + 0.5) * (24 / 400000) - 12
    w = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) * (24 / 400000)
    for i, g in enumerate(R.GATES):
        a, b = us.gate_scales(i)
        # the midpoint rule's own error is below 1e-9 here (kinks and steps of relu lie between two points); the factors are floats, 2^-24
        assert abs(a * math.sqrt(float((R.gate_value(g, z) ** 2 * w).sum())) - 1) < 1e-7
        assert abs(b * math.sqrt(float((R.gate_slope(g, z) ** 2 * w).sum())) - 1) < 1e-7
    with pytest.raises(us.UsError):
        us.gate_scales(4)
    L = ctypes.CDLL(us.library_path())
    assert L.us_gate_scales(0, None, None) == NULL


def test_slopes_are_the_differences_of_the_gates():
    z = torch.linspace(-6, 6, 241, dtype=torch.float64) + 0.01
    h = 1e-5
    for g in R.GATES:
        d = (R.gate_value(g, z + h) - R.gate_value(g, z - h)) / (2 * h)
        assert float((d - R.gate_slope(g, z)).abs().max()) < 1e-9          # h^2 / 6 times a third derivative below 3


def test_blocks_by_definition():
    x = np.zeros((6, 48))
    x[0, 0], x[0, 5] = 127.0, 63.5                   # step 1; 63.5 lies between two codes: the even one
    x[1, 3] = -127.5                                 # reaches 127.5 steps of 1: step 2, 63.75 -> 64
    x[2, 40] = 2.0 ** -24                            # FP16's least value: the least step
    x[3, 1], x[3, 33] = np.inf, -65504.0             # clipped; 65504 is 127.9 steps of 512
    x[4, 2], x[4, 4] = np.nan, 1.0
    x[5, 47] = 3.0
    c, s = R.keep8(x)
    assert (c[0, 0], c[0, 5], s[0, 0]) == (127, 64, 127) and (c[1, 3], s[1, 0]) == (-64, 128) and (c[2, 40], s[2, 1]) == (1, 103)
    assert (c[3, 1], s[3, 0], c[3, 33], s[3, 1]) == (127, 136, -127, 136) and (c[4, 2], c[4, 4], s[4, 0]) == (-128, 64, 121 + 64)
    assert (c[5, 47], s[5, 1]) == (96, 122) and c[5, :32].any() == False and s[5, 0] == 103          # noqa: E712
    v = R.keep8_values(c, s)
    assert np.array_equal(v, v.astype(np.float16).astype(np.float64), equal_nan=True)               # FP16 holds every value
