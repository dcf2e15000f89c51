"""Query and key norms with the position rotation, into attention's heads and back, against the definition in 64 bits.

Tolerances: an output is rounded to FP16 once, half a step or 2^-11 of its value (2^-25 among subnormals).  Before that, in FP32: the norm's sum
of up to 256 squares in 16 steps and 4 exchanges, its root and division (24 roundings of 2^-24), two products, and the rotation with sines and
cosines whose absolute error is below 2^-18 (the device's v_sin / v_cos are within 2^-20 of the exact function over every phase, the phase
itself is exact to 2^-26 of a turn, 2.4e-8 * 2 pi): together below 2^-17 of the pair's length.  Gradients: the same terms once more through
the mean over the head, so 2^-15 of the largest magnitude of the head's gradient; sums of the weights' gradients: 2^-24 per addition of
a chain of at most (tokens / groups * heads + groups) terms, 2^-14 of the sum of magnitudes being far above it for the sizes here.
"""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import gated_ref as R
import paper_2303_11257_amd as us
from gpu_util import DEV, ptr, stream

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -11


def make(batch, s, h, kv, dh, rot, ld, seed, first=0, scale=1.5):
    g = torch.Generator().manual_seed(seed)
    T = batch * s
    x = (torch.randn((T, ld), generator=g) * scale).half()
    pos = (torch.randint(0, first + 1, (batch, 1), generator=g) + torch.arange(s)).reshape(T).int()
    freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) / max(1, rot // 2))
    wq, wk = (1 + 0.3 * torch.randn((2, dh), generator=g)).half()
    d = [torch.randn((batch * h, s, dh), generator=g).half() for _ in range(3)]
    return dict(x=x, pos=pos, freq=freq, wq=wq, wk=wk, dQ=d[0], dK=d[1], dV=d[2])


def reference(m, batch, s, h, kv, dh, rot, neighbours, eps, back):
    """Everything in float64, heads as [tokens, heads, dh]; the second value of a pair is the scale of the FP32 error."""
    T, rep = batch * s, h // kv
    x = m["x"][:, : (h + 2 * kv) * dh].double().view(T, h + 2 * kv, dh)
    out = lambda y: y.view(batch, s, -1, dh).permute(0, 2, 1, 3).repeat_interleave(h // y.shape[1], 1).reshape(batch * h, s, dh)      # noqa: E731
    res = {"V": out(x[:, h + kv:])}
    grads = []
    for name, part, w in (("Q", x[:, :h], m["wq"]), ("K", x[:, h: h + kv], m["wk"])):
        w = torch.ones(dh, dtype=torch.float64) if w is None else w.double()
        rstd = (part.square().mean(-1, keepdim=True) + eps) ** -0.5
        xh = part * rstd
        res[name] = out(R.turned(xh * w, m["pos"], m["freq"], rot, neighbours))
        if back:
            n = part.shape[1]
            g = m["d" + name].double().view(batch, n, h // n, s, dh).sum(2).permute(0, 2, 1, 3).reshape(T, n, dh) / math.sqrt(h // n)
            g = R.turned(g, m["pos"], m["freq"], rot, neighbours, back=True)
            res["dw" + name.lower()] = (g * xh).sum((0, 1)) / math.sqrt(T * n)
            res["dw" + name.lower() + "_size"] = (g * xh).abs().sum((0, 1)) / math.sqrt(T * n)
            g = g * w
            grads.append(rstd * (g - xh * (g * xh).mean(-1, keepdim=True)))
    if back:
        grads.append(m["dV"].double().view(batch, kv, rep, s, dh).sum(2).permute(0, 2, 1, 3).reshape(T, kv, dh) / math.sqrt(rep))
        res["dx"] = torch.cat(grads, 1)
    return res


def forward(m, batch, s, h, kv, dh, rot, ld, neighbours, eps, st=None, use_pos=True):
    n = batch * h * s * dh
    out = {k: torch.full((n + 64,), 7.0, dtype=torch.float16, device=DEV) for k in "QKV"}
    us.qk_norm_rope_fwd(ptr(m["x"]), ld, ptr(m["wq"]), ptr(m["wk"]), ptr(m["pos"]) if use_pos else None, ptr(m["freq"]), *(ptr(out[k]) for k in "QKV"),
                        batch, s, h, kv, dh, rot, us.ROPE_NEIGHBOURS if neighbours else us.ROPE_HALVES, eps, stream() if st is None else st)
    return out


def backward(m, batch, s, h, kv, dh, rot, ld, neighbours, eps, st=None):
    wsb = us.qk_norm_rope_workspace_bytes(batch, s, h, kv, dh)
    m["ws"] = torch.full((wsb,), 0xff, dtype=torch.uint8, device=DEV)                # NaN: nothing may be read before it is written
    out = dict(dx=torch.full((batch * s, ld), 7.0, dtype=torch.float16, device=DEV), dwq=torch.full((dh,), 7.0, dtype=torch.float16, device=DEV),
               dwk=torch.full((dh,), 7.0, dtype=torch.float16, device=DEV))
    us.qk_norm_rope_bwd(ptr(m["x"]), ld, ptr(m["wq"]), ptr(m["wk"]), ptr(m["pos"]), ptr(m["freq"]), ptr(m["dQ"]), ptr(m["dK"]), ptr(m["dV"]), ptr(out["dx"]), ld,
                        ptr(out["dwq"]), ptr(out["dwk"]), batch, s, h, kv, dh, rot, us.ROPE_NEIGHBOURS if neighbours else us.ROPE_HALVES, eps, 0.0, 0.0,
                        ptr(m["ws"]), wsb, stream() if st is None else st)
    return out


def to_gpu(m):
    return {k: None if v is None else v.to(DEV) for k, v in m.items()}


def check(got, ref, m, batch, s, h, kv, dh, rot, ld):
    n = batch * h * s * dh
    for k in "QKV":
        v = got[k].cpu().double()
        assert (v[n:] == 7).all()
        v, e = v[:n].view(batch * h, s, dh), ref[k]
        room = HALF * e.abs() + 2.0 ** -25
        if k != "V":
            room = room + 2.0 ** -17 * e.abs().amax(-1, keepdim=True) * 1.5
        else:
            room = torch.zeros_like(e)                       # a copy
        assert ((v - e).abs() <= room).all(), (k, float(((v - e).abs() - room).max()))


def check_back(got, ref, batch, s, h, kv, dh, ld):
    T, cols = batch * s, (h + 2 * kv) * dh
    d = got["dx"].cpu().double()
    assert (d[:, cols:] == 7).all()
    v, e = d[:, :cols].reshape(T, h + 2 * kv, dh), ref["dx"]
    room = HALF * e.abs() + 2.0 ** -15 * e.abs().amax(-1, keepdim=True) + 2.0 ** -25
    assert ((v - e).abs() <= room).all(), float(((v - e).abs() - room).max())
    for k in ("dwq", "dwk"):
        v, e = got[k].cpu().double(), ref[k]
        assert ((v - e).abs() <= HALF * e.abs() + 2.0 ** -14 * ref[k + "_size"] + 2.0 ** -25).all(), k


SHAPES = [(1, 1, 1, 1, 16, 16), (3, 1, 4, 4, 64, 64), (2, 7, 6, 2, 80, 32), (1, 33, 8, 1, 128, 128), (2, 65, 4, 2, 96, 96), (1, 19, 3, 3, 256, 256),
          (2, 5, 2, 1, 32, 0), (5, 40, 12, 4, 48, 16), (1, 2100, 2, 1, 32, 32),
          (1, 70, 70, 7, 16, 16), (3, 1400, 1, 1, 64, 64), (2, 5300, 3, 1, 16, 16)]       # more heads than lane groups; tokens for a wave each


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("batch,s,h,kv,dh,rot", SHAPES)
def test_forward_and_backward(batch, s, h, kv, dh, rot, neighbours):
    for pad, first in ((0, 0), (24, 100000)):
        ld = (h + 2 * kv) * dh + pad
        m = make(batch, s, h, kv, dh, rot, ld, seed=dh + s + pad, first=first)
        g = to_gpu(m)
        ref = reference(m, batch, s, h, kv, dh, rot, neighbours, 1e-6, True)
        check(forward(g, batch, s, h, kv, dh, rot, ld, neighbours, 1e-6), ref, m, batch, s, h, kv, dh, rot, ld)
        check_back(backward(g, batch, s, h, kv, dh, rot, ld, neighbours, 1e-6), ref, batch, s, h, kv, dh, ld)


def test_positions_over_all_of_32_bits_and_none():
    batch, s, h, kv, dh, rot = 1, 64, 2, 1, 64, 64
    ld = (h + 2 * kv) * dh
    m = make(batch, s, h, kv, dh, rot, ld, seed=5)
    m["pos"] = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 9, -123456789, 7] * 8, dtype=torch.int32)
    ref = reference(m, batch, s, h, kv, dh, rot, False, 0.0, False)
    check(forward(to_gpu(m), batch, s, h, kv, dh, rot, ld, False, 0.0), ref, m, batch, s, h, kv, dh, rot, ld)
    m["pos"] = torch.arange(s, dtype=torch.int32)
    ref = reference(m, batch, s, h, kv, dh, rot, False, 0.0, False)
    check(forward(to_gpu(m), batch, s, h, kv, dh, rot, ld, False, 0.0, use_pos=False), ref, m, batch, s, h, kv, dh, rot, ld)


def test_without_weights_and_frequencies_above_a_turn():
    batch, s, h, kv, dh, rot = 2, 9, 2, 2, 48, 48
    ld = (h + 2 * kv) * dh
    m = make(batch, s, h, kv, dh, rot, ld, seed=6)
    m["wq"] = m["wk"] = None
    m["freq"] = m["freq"] * 40.0 - 3.0                 # more than a turn per position, and negative ones
    ref = reference(m, batch, s, h, kv, dh, rot, True, 0.0, True)
    g = to_gpu(m)
    check(forward(g, batch, s, h, kv, dh, rot, ld, True, 0.0), ref, m, batch, s, h, kv, dh, rot, ld)
    check_back(backward(g, batch, s, h, kv, dh, rot, ld, True, 0.0), ref, batch, s, h, kv, dh, ld)


def test_heads_of_zeros_large_values_and_nan_stay_in_their_heads():
    batch, s, h, kv, dh, rot = 1, 4, 2, 1, 32, 32
    ld = (h + 2 * kv) * dh
    m = make(batch, s, h, kv, dh, rot, ld, seed=7)
    m["x"][0, :dh] = 0                                 # query head 0 of token 0: eps alone
    m["x"][1, dh: 2 * dh] = 60000.0                    # squares far beyond FP16, within FP32
    clean = {k: v.clone() for k, v in forward(to_gpu(m), batch, s, h, kv, dh, rot, ld, False, 1e-5).items()}
    ref = reference(m, batch, s, h, kv, dh, rot, False, 1e-5, False)
    check(clean, ref, m, batch, s, h, kv, dh, rot, ld)
    m["x"][2, 2 * dh + 3] = float("nan")               # the key head of token 2, shared by both query heads
    m["x"][3, 4] = float("inf")
    dirty = forward(to_gpu(m), batch, s, h, kv, dh, rot, ld, False, 1e-5)
    n = batch * h * s * dh
    for k, bad in (("Q", [(0, 3)]), ("K", [(0, 2), (1, 2)]), ("V", [])):
        a, b = clean[k][:n].view(batch * h, s, dh).cpu(), dirty[k][:n].view(batch * h, s, dh).cpu()
        hit = torch.zeros((batch * h, s), dtype=torch.bool)
        for i, t in bad:
            hit[i, t] = True
        assert torch.equal(a[~hit], b[~hit])
        if bad:
            assert torch.isnan(b[hit]).any(-1).all()


def test_gradient_against_differences():
    """<dx, v> against the central difference of <Q, dQ> + <K, dK> + <V, dV> in 64 bits along v: no shared heads, so every factor is 1.  Step
    h = 2^-10: the difference's own error, h^2 / 6 times a third derivative of order one, is below 2^-20 of the sums' size; the gradient's
    is 2^-11 per element of independent sign, below 2^-9 of <|dx|, |v|> / sqrt(n) times a generous 8."""
    batch, s, h, kv, dh, rot = 2, 6, 3, 3, 32, 32
    ld = (h + 2 * kv) * dh
    m = make(batch, s, h, kv, dh, rot, ld, seed=8, first=1000)
    dx = backward(to_gpu(m), batch, s, h, kv, dh, rot, ld, False, 1e-6)["dx"].cpu().double()
    v = torch.randn((batch * s, ld), generator=torch.Generator().manual_seed(9), dtype=torch.float64)
    step, vals = 2.0 ** -10, []
    for sign in (1, -1):
        r = reference(dict(m, x=m["x"].double() + sign * step * v), batch, s, h, kv, dh, rot, False, 1e-6, False)
        vals.append(sum(float((r[k] * m["d" + k].double()).sum()) for k in "QKV"))
    diff = (vals[0] - vals[1]) / (2 * step)
    size = float((dx.abs() * v.abs()).sum())
    assert abs(diff - float((dx * v).sum())) <= size * (8 * 2.0 ** -9 / math.sqrt(v.numel()) + 2.0 ** -18)


def test_captured_on_another_stream_and_two_at_once():
    batch, s, h, kv, dh, rot = 2, 30, 4, 2, 64, 64
    ld = (h + 2 * kv) * dh
    sets = [to_gpu(make(batch, s, h, kv, dh, rot, ld, seed=20 + i, first=50)) for i in range(2)]
    eager = [(forward(g, batch, s, h, kv, dh, rot, ld, False, 1e-6), backward(g, batch, s, h, kv, dh, rot, ld, False, 1e-6)) for g in sets]
    torch.cuda.synchronize()
    streams, graphs, outs = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for g, st in zip(sets, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            now = torch.cuda.current_stream().cuda_stream
            outs.append((forward(g, batch, s, h, kv, dh, rot, ld, False, 1e-6, now), backward(g, batch, s, h, kv, dh, rot, ld, False, 1e-6, now)))
        graphs.append(graph)
    for _ in range(4):
        for o in outs:
            o[1]["dx"].zero_()
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for (ef, eb), (of, ob) in zip(eager, outs):
            n, cols = batch * h * s * dh, (h + 2 * kv) * dh
            assert all(torch.equal(ef[k][:n], of[k][:n]) for k in "QKV")
            assert torch.equal(eb["dx"][:, :cols], ob["dx"][:, :cols]) and torch.equal(eb["dwq"], ob["dwq"]) and torch.equal(eb["dwk"], ob["dwk"])


PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")


@pytest.mark.parametrize("neighbours", [False, True])
def test_every_frequency_at_every_position(neighbours):
    """Large, negative, tiny and tiny negative frequencies at the ends of 32-bit positions, against angles from rational arithmetic (102 digits of pi)."""
    freqs = [37.0, 1e3, 1e6, -5.5e5, 2.0 ** 33 / 3, -2.0 ** 40, 1e-19, -1e-19, -4e-17, 1e-12, 2 * math.pi, -2 * math.pi, math.pi, 0.0, 0.1, 6.0]
    pos = [2 ** 31 - 1, -2 ** 31, 1234567891, -987654321, -1, 1, 0, 65537]
    batch, s, h, kv, dh, rot = 1, len(pos), 2, 1, 48, 32
    ld = (h + 2 * kv) * dh
    m = make(batch, s, h, kv, dh, rot, ld, seed=11)
    m["pos"], m["freq"] = torch.tensor(pos, dtype=torch.int32), torch.tensor(freqs, dtype=torch.float64)
    turns = [[p * Fraction(f) / (2 * PI) % 1 for f in freqs] for p in pos]
    angle = torch.tensor([[float(t if t <= Fraction(1, 2) else t - 1) * 2 * math.pi for t in row] for row in turns], dtype=torch.float64)
    ref = reference(m, batch, s, h, kv, dh, 0, neighbours, 1e-6, False)
    i = torch.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
    for k in "QK":
        y = ref[k].clone()
        ref[k][..., a] = y[..., a] * angle.cos() - y[..., b] * angle.sin()
        ref[k][..., b] = y[..., b] * angle.cos() + y[..., a] * angle.sin()
    check(forward(to_gpu(m), batch, s, h, kv, dh, rot, ld, neighbours, 1e-6), ref, m, batch, s, h, kv, dh, rot, ld)
