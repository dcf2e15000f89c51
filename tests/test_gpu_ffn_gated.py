"""The gated feed-forward block against its definition in 64 bits, stage by stage on the tensors that the GPU stored.

Products with FP16 results (Z, Y, dX, dWgu, dWd) go by the matmul metric of the other tests (gpu_util.assert_close).  Codes: an E4M3 / E5M2 code is the
nearest value to a number that may be off by `slack`, so it is within half a step (2^-4, 2^-3 of the value; half of the least step among
subnormals) plus slack; an 8-bit block's code within half a step plus slack, and its step is the definition's but where the block's largest
magnitude lies within slack of a border.  slack: what the matrix core's sums are off (parity.py: FP8 operands 2e-4 of a unit; FP16 2^-20 sqrt(K)
of a unit, FP32 sums in any order) times the derivative towards it, at most |f| + |f'||zu| <= 1.13 |zu| + |zg| + 1, times the factor.

The metric's absolute part for FP8 operands, 2e-4 of a unit, was measured on normal operands.  H and dZ are products of two and three normal
numbers, with tails to match, and the matrix core's adder keeps about 14 bits below the largest product of a group: where a group
holds a product P, its sum may be off by 2^-13 P, and all groups together by 2^-12 of the sum of all magnitudes, which is therefore what products with
such an operand are allowed per element (as the range-stress products are).  That bound is wide, so their error's 2-norm is held as well: rounding to
FP16 is off by at most 2^-11 with a uniform distribution, 2^-11 / sqrt(3) = 2.82e-4 of the values' rms, the adder by 1.4e-5 rms of a unit on normal
operands and at most five times that on these, and (2.82e-4^2 + 7e-5^2)^1/2 < 3e-4.
"""
import math

import numpy as np
import pytest
import torch

import gated_ref as R
import paper_2303_11257_amd as us
from gpu_util import DEV, assert_close, ptr, stream

pytestmark = pytest.mark.gpu


class Block:
    """Operands and buffers of one block; outputs have a guard row behind them."""

    def __init__(self, T, d, f, fp8, keep8, gate, seed=1, sigma=1.0):
        g = torch.Generator().manual_seed(seed)
        self.T, self.d, self.f, self.fp8, self.keep8, self.gate = T, d, f, fp8, keep8, gate
        self.mode = (us.FFN_FP8 if fp8 else 0) | (us.FFN_KEEP8 if keep8 else 0)
        rnd = lambda *s: (torch.randn(s, generator=g) * sigma).half()      # noqa: E731
        self.X, self.Wgu, self.Wd, self.G = rnd(T, d), rnd(d, 2 * f), rnd(f, d), rnd(T, d)
        if fp8:
            self.X, self.Wgu, self.Wd = (x.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for x in (self.X, self.Wgu, self.Wd))
            self.G = self.G.float().clamp(-57344, 57344).to(torch.float8_e5m2).view(torch.uint8)
        self.g = {k: getattr(self, k).to(DEV) for k in ("X", "Wgu", "Wd", "G")}
        el = torch.uint8 if fp8 else torch.float16
        new = lambda r, c, t: torch.full((r + 1, c), 7, dtype=t, device=DEV)      # noqa: E731
        self.Z = new(T, 2 * f, torch.int8 if keep8 else torch.float16)
        self.Zs = new(T, 2 * us.keep8_blocks(f), torch.uint8) if keep8 else None
        self.H, self.Y, self.dZ, self.dX = new(T, f, el), new(T, d, torch.float16), new(T, 2 * f, el), new(T, d, torch.float16)
        self.dWgu, self.dWd = new(d, 2 * f, torch.float16), new(f, d, torch.float16)
        self.wsb = us.ffn_gated_workspace_bytes(T, d, f, self.mode)
        self.ws = torch.full((max(16, self.wsb),), 0xff, dtype=torch.uint8, device=DEV)

    def forward(self, st=None, keep=True, ws=True, **kw):
        us.ffn_gated_fwd(ptr(self.g["X"]), ptr(self.g["Wgu"]), ptr(self.g["Wd"]), ptr(self.Z) if keep else None, ptr(self.Zs), ptr(self.H), ptr(self.Y), self.T, self.d,
                         self.f, self.gate, self.mode, ptr(self.ws) if ws else None, self.wsb if ws else 0, stream() if st is None else st, **kw)
        return self

    def backward(self, st=None, skip=(), **kw):
        us.ffn_gated_bwd(ptr(self.g["X"]), ptr(self.g["Wgu"]), ptr(self.g["Wd"]), ptr(self.Z), ptr(self.Zs), ptr(self.H), ptr(self.g["G"]), ptr(self.dZ),
                         *(None if n in skip else ptr(getattr(self, n)) for n in ("dX", "dWgu", "dWd")), self.T, self.d, self.f, self.gate, self.mode, ptr(self.ws),
                         self.wsb, stream() if st is None else st, **kw)
        return self

    def outputs(self):
        torch.cuda.synchronize()
        return {n: getattr(self, n).cpu() for n in ("Z", "Zs", "H", "Y", "dZ", "dX", "dWgu", "dWd") if getattr(self, n) is not None}


def operand(x, e5m2=False):
    return R.fp8_values(x, e5m2) if x.dtype == torch.uint8 else x.double()


def product_close(b, got, A, B, factor, what):
    want = A @ B * factor
    if not b.fp8:
        assert_close(got.numpy(), want.numpy(), what, scale=max(1.0, float(want.square().mean().sqrt())))
        return
    scale = float(want.square().mean().sqrt())
    assert_close(got.numpy(), want.numpy(), what, fp8=True, scale=scale, allow=(A.abs() @ B.abs() * (factor * 2.0 ** -12)).numpy())
    assert float((got.double() - want).square().mean().sqrt()) <= 3e-4 * scale + 2.0 ** -25, what


def slack_of(b, zg, zu, factor):
    unit = (2e-4 if b.fp8 else 2.0 ** -20 * math.sqrt(b.d))
    return factor * unit * (2 + zg.abs() + 1.2 * zu.abs())


def near_codes(codes, e5m2, want, slack, what):
    v = R.fp8_values(codes, e5m2)
    least, rel, top = (2.0 ** -17, 2.0 ** -3, 57344.0) if e5m2 else (2.0 ** -10, 2.0 ** -4, 448.0)
    w = want.clamp(-top, top)
    bad = (v - w).abs() > torch.clamp(w.abs() * rel, min=least) + slack
    assert not bad.any(), (what, int(bad.sum()), float((v - w).abs()[bad].max()))


def kept(b, out):
    """The values that the backward pass reads, [T, f] each."""
    z = out["Z"][: b.T]
    if not b.keep8:
        return z[:, : b.f].double(), z[:, b.f:].double()
    nb = us.keep8_blocks(b.f)
    s = out["Zs"][: b.T].numpy()
    return tuple(torch.from_numpy(R.keep8_values(z[:, i * b.f: (i + 1) * b.f].numpy(), s[:, i * nb: (i + 1) * nb])) for i in (0, 1))


def check_forward(b, out, alpha=None):
    gate = R.GATES[b.gate]
    a = us.gate_scales(b.gate)[0] if alpha is None else alpha
    X, Wgu, Wd = (operand(getattr(b, n)) for n in ("X", "Wgu", "Wd"))
    Z = X @ Wgu / math.sqrt(b.d)
    zg, zu = Z[:, : b.f], Z[:, b.f:]
    if not b.keep8:
        assert_close(out["Z"][: b.T].numpy(), Z.numpy(), "Z", fp8=b.fp8)
    else:
        nb = us.keep8_blocks(b.f)
        unit = slack_of(b, torch.zeros(()), torch.zeros(()), 1.0).item()
        for i, z in enumerate((zg, zu)):
            codes, scales = out["Z"][: b.T, i * b.f: (i + 1) * b.f].numpy(), out["Zs"][: b.T, i * nb: (i + 1) * nb].numpy()
            lo, hi = R.keep8(z.numpy() * (1 - 1e-6) - np.sign(z.numpy()) * unit)[1], R.keep8(z.numpy() * (1 + 1e-6) + np.sign(z.numpy()) * unit)[1]
            assert ((scales >= lo) & (scales <= hi)).all()
            step = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, axis=1)[:, : b.f]
            assert (np.abs(codes * step - z.numpy()) <= step / 2 + unit * (1 + np.abs(z.numpy()))).all()
    H = a * R.gate_value(gate, zg) * zu
    if b.fp8:
        near_codes(out["H"][: b.T], False, H, slack_of(b, zg, zu, a), "H")
    else:
        d = (out["H"][: b.T].double() - H).abs()
        assert (d <= 2.0 ** -11 * H.abs() + 2.0 ** -25 + 1e-5 * H.abs() + slack_of(b, zg, zu, a)).all()
    product_close(b, out["Y"][: b.T], operand(out["H"][: b.T]), Wd, b.f ** -0.5, "Y")
    for n in ("Z", "Zs", "H", "Y"):
        if n in out:
            assert (out[n][b.T].float() == 7).all(), n


def check_backward(b, out, alpha=None, beta_gate=None, beta_up=None):
    gate = R.GATES[b.gate]
    da, db = us.gate_scales(b.gate)
    a, bg, bu = (d if x is None else x for x, d in ((alpha, da), (beta_gate, db), (beta_up, da)))
    X, Wgu, Wd, G = operand(b.X), operand(b.Wgu), operand(b.Wd), operand(b.G, True)
    zg, zu = kept(b, out)
    dH = G @ Wd.t() / math.sqrt(b.d)
    F, S = R.gate_value(gate, zg), R.gate_slope(gate, zg)
    want = torch.cat([bg * S * zu * dH, bu * F * dH], 1)
    unit = 2e-4 if b.fp8 else 2.0 ** -20 * math.sqrt(b.d)
    # dH's own error, and the gate functions' 2e-5 (the fitted tail of gelu 4e-6 of the probability, exponentials and reciprocals 2^-22)
    room = unit * torch.cat([bg * (S * zu).abs(), bu * F.abs()], 1) + 2e-5 * torch.cat([bg * (zu * dH).abs(), bu * (1 + zg.abs()) * dH.abs()], 1)
    if b.fp8:
        near_codes(out["dZ"][: b.T], True, want, room, "dZ")
    else:
        assert ((out["dZ"][: b.T].double() - want).abs() <= 2.0 ** -11 * want.abs() + 2.0 ** -25 + room).all()
    if b.keep8:
        H = a * F * zu
        if b.fp8:
            near_codes(out["H"][: b.T], False, H, 2e-5 * a * (1 + zg.abs()) * zu.abs(), "H again")
        else:
            assert ((out["H"][: b.T].double() - H).abs() <= 2.0 ** -11 * H.abs() + 2.0 ** -25 + 2e-5 * a * (1 + zg.abs()) * zu.abs()).all()
    dZ, H = operand(out["dZ"][: b.T], True), operand(out["H"][: b.T])
    product_close(b, out["dX"][: b.T], dZ, Wgu.t(), (2 * b.f) ** -0.5, "dX")
    product_close(b, out["dWgu"][: b.d], X.t(), dZ, b.T ** -0.5, "dWgu")
    product_close(b, out["dWd"][: b.f], H.t(), G, b.T ** -0.5, "dWd")
    for n, r in (("dZ", b.T), ("dX", b.T), ("dWgu", b.d), ("dWd", b.f), ("H", b.T)):
        assert (out[n][r].float() == 7).all(), n


# one token, a few, odd numbers; widths that end inside a block of 32, a tile's half and a tile; all kernels' tiles
SHAPES = [(1, 16, 16), (1, 256, 688), (5, 48, 32), (33, 64, 80), (64, 528, 144), (65, 512, 2064), (130, 256, 272), (600, 512, 1040), (1999, 272, 528), (2048, 128, 2064), (1300, 64, 4112),
          (4095, 256, 4112), (5001, 128, 272)]            # an odd number of tokens as reduction: of wave groups in one launch, and in slices


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,d,f", SHAPES)
def test_forward_and_backward(T, d, f, fp8, keep8):
    b = Block(T, d, f, fp8, keep8, us.GATE_SILU, seed=T + f)
    b.forward()
    first = b.outputs()
    check_forward(b, first)
    if keep8:
        b.H.view(torch.uint8)[: b.T].fill_(0x3c)             # the forward call's H is not read again
    b.backward()
    if T == 4095:
        assert "pair:" in us.last_launch() or fp8, us.last_launch()
    if T == 5001:
        assert "partial" in us.last_launch(), us.last_launch()
    out = b.outputs()
    assert torch.equal(out["Z"], first["Z"])
    check_backward(b, out)


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("gate", range(4))
@pytest.mark.parametrize("T,d,f", [(40, 96, 208), (700, 96, 1296)])
def test_gates_and_factors(T, d, f, gate, fp8, keep8):
    b = Block(T, d, f, fp8, keep8, gate, seed=gate)
    b.forward().backward()
    out = b.outputs()
    if not keep8:
        check_forward(b, out)
    check_backward(b, out)
    kw = dict(alpha=1.25, beta_gate=0.75, beta_up=0.5)
    b.forward(alpha=1.25)
    check_forward(b, b.outputs(), alpha=1.25)
    b.backward(**kw)
    check_backward(b, b.outputs(), **kw)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,d,f", [(1, 1024, 4400), (16, 256, 688), (300, 256, 1040)])
def test_serving_keeps_nothing_and_answers_the_same(T, d, f, fp8):
    b = Block(T, d, f, fp8, False, us.GATE_GELU)
    y = b.forward().outputs()
    b.Y.fill_(7), b.H.fill_(7), b.Z.fill_(3)
    z = b.forward(keep=False).outputs()
    assert (z["Z"] == 3).all()
    assert torch.equal(y["H"], z["H"]) and torch.equal(y["Y"], z["Y"])
    c = Block(T, d, f, fp8, True, us.GATE_GELU)              # what is kept does not change the answer either
    k = c.forward().outputs()
    assert torch.equal(y["H"], k["H"]) and torch.equal(y["Y"], k["Y"])
    w = Block(T, d, f, fp8, False, us.GATE_GELU)             # without a workspace the sums may be taken in another order
    check_forward(w, w.forward(ws=False).outputs())


# (tokens, d, f): the streams of weights, every row count they take and the next; slices of several steps, the last one shorter; f and d that end inside a strip
@pytest.mark.parametrize("fp8,T", [(False, t) for t in (1, 2, 3, 4, 5, 8, 9)] + [(True, t) for t in (1, 2, 3, 4, 5)])
def test_a_few_rows(T, fp8):
    for d, f, keep8 in (((2064, 10896, False), (11024, 2032, True)) if fp8 else ((1040, 4400, False), (4112, 1040, True))):
        b = Block(T, d, f, fp8, keep8, us.GATE_SILU, seed=T * d)
        check_forward(b, b.forward().outputs())
        assert ("stream" in us.last_launch()) == (T <= (4 if fp8 else 8))
        w = Block(T, d, f, fp8, keep8, us.GATE_SILU, seed=T * d)      # without a workspace the sums are taken in another order
        check_forward(w, w.forward(ws=False).outputs())
        assert "stream" not in us.last_launch()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,d,f,up,down", [(9, 2064, 5648, False, True), (32, 4112, 5136, True, True), (33, 2048, 5632, False, True), (64, 1040, 4112, False, True),
                                           (65, 1040, 4112, False, False), (17, 512, 1376, False, False)])
def test_a_few_rows_in_slices(T, d, f, up, down, fp8):
    """Up to 64 rows: reductions in slices on either side of the rule, the last slice shorter than the others."""
    for keep8 in (False, True):
        b = Block(T, d, f, fp8, keep8, us.GATE_SIGMOID, seed=T)
        check_forward(b, b.forward().outputs())
        launches = us.last_launch().split(" + ")
        if not fp8:
            assert ["partial" in n for n in launches] == [up, down], launches
        check_forward(b, b.forward(ws=False).outputs())
        assert "partial" not in us.last_launch()


def test_single_gradients_and_none_of_no_tokens():
    b = Block(130, 64, 96, False, True, us.GATE_SILU)
    full = b.forward().backward().outputs()
    for n in ("dX", "dWgu", "dWd"):
        c = Block(130, 64, 96, False, True, us.GATE_SILU)
        o = c.forward().backward(skip=[n]).outputs()
        assert (o[n] == 7).all()
        for other in {"dX", "dWgu", "dWd"} - {n}:
            assert_close(o[other][:-1].numpy(), full[other][:-1].double().numpy(), other)
    e = Block(0, 64, 96, True, False, us.GATE_SILU)
    o = e.forward().backward().outputs()
    assert (o["dWgu"][:64] == 0).all() and (o["dWd"][:96] == 0).all() and (o["dX"] == 7).all()


@pytest.mark.parametrize("T", [3, 700])
def test_infinities_and_nan_stay_in_their_rows(T):
    """A NaN and an infinity in X reach their own rows of Z, H, Y and dX only; 8-bit blocks hold NaN and clip infinities."""
    for keep8 in (False, True):
        b = Block(T, 64, 2080 if T > 3 else 96, False, keep8, us.GATE_SILU)
        clean = b.forward().backward().outputs()
        b.g["X"][1, 5] = float("nan")
        b.g["X"][2, 9] = float("inf")
        dirty = b.forward().backward().outputs()
        others = [r for r in range(T) if r not in (1, 2)]
        for n in ("Z", "H", "Y", "dZ", "dX"):
            assert torch.equal(clean[n][others], dirty[n][others]), n
        assert torch.isnan(dirty["Y"][1]).all() and torch.isnan(dirty["dX"][1]).all()
        if keep8:
            assert (dirty["Z"][1] == -128).all() and (dirty["Z"][2].abs() == 127).all() and (dirty["Zs"][2] == 136).all() and (dirty["Zs"][1] == 103 + 64).all()
        else:
            assert torch.isnan(dirty["Z"][1]).all() and torch.isinf(dirty["Z"][2]).all()


@pytest.mark.parametrize("T,f", [(3, 80), (9, 4112), (300, 1040), (700, 2064), (3000, 4112)])
def test_an_infinity_marks_no_block(T, f):
    """An infinite X makes infinities, which are clipped; the columns that a last block of 16 lacks are NaN on the way and must not show."""
    b = Block(T, 1024 if T == 9 else 64, f, False, True, us.GATE_SILU)
    b.g["X"][2, 9] = float("inf")
    b.forward()
    out = b.outputs()
    assert (out["Z"][2].abs() == 127).all() and (out["Zs"][2] == 136).all()
    rest = [r for r in range(T) if r != 2]
    assert (out["Zs"][rest] <= 136).all()


def test_gradients_against_differences():
    """With one factor for both halves of dZ the gradients are those of <Y, G> up to known factors: dX (2f)^1/2 (f/d)^-1/2 ... all products' factors
    divided out.  Central difference in 64 bits along a direction v, step 2^-8: its error, h^2 / 6 times a third derivative of order one per
    element, is below 2^-17 of the sums' size; the FP16 roundings of Z, dZ and dX are 2^-11 each per element with independent signs: below
    3 * 2^-10 of <|dX|, |v|> / sqrt(n), times a generous 8."""
    T, d, f = 24, 48, 64
    b = Block(T, d, f, False, False, us.GATE_SILU, seed=3)
    a = us.gate_scales(us.GATE_SILU)[0]
    b.forward().backward(alpha=a, beta_gate=a, beta_up=a)
    out = b.outputs()
    X, Wgu, Wd, G = (getattr(b, n).double() for n in ("X", "Wgu", "Wd", "G"))

    def value(X, Wgu, Wd):
        Z = X @ Wgu / math.sqrt(d)
        return float((((a * R.gate_value("silu", Z[:, :f]) * Z[:, f:]) @ Wd / math.sqrt(f)) * G).sum())

    # true gradient / stored one: dH f^-1/2 instead of d^-1/2; dX d^-1/2 instead of (2f)^-1/2; weights d^-1/2 (f^-1/2) instead of T^-1/2
    hs = math.sqrt(d / f)
    gen = torch.Generator().manual_seed(4)
    for name, at, factor in (("dX", 0, hs * math.sqrt(2 * f / d)), ("dWgu", 1, hs * math.sqrt(T / d)), ("dWd", 2, math.sqrt(T / f))):
        g = out[name][:-1].double() * factor
        v = torch.randn(g.shape, generator=gen, dtype=torch.float64)
        h, p = 2.0 ** -8, [X, Wgu, Wd]
        p[at] = p[at] + h * v
        up = value(*p)
        p[at] = p[at] - 2 * h * v
        diff = (up - value(*p)) / (2 * h)
        size = float((g.abs() * v.abs()).sum())
        assert abs(diff - float((g * v).sum())) <= size * (24 * 2.0 ** -10 / math.sqrt(v.numel()) + 2.0 ** -14), name


def test_captured_replayed_and_two_streams():
    blocks = [Block(70, 128, 272, fp8, True, us.GATE_SILU, seed=s) for s, fp8 in ((1, False), (2, True))]
    eager = [b.forward().backward().outputs() for b in blocks]
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for b, st in zip(blocks, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            now = torch.cuda.current_stream().cuda_stream
            b.forward(now).backward(now)
        graphs.append(graph)
    for _ in range(4):
        for b in blocks:
            for n in ("Z", "H", "Y", "dZ", "dX"):
                getattr(b, n)[: b.T].zero_()
        torch.cuda.synchronize()
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for b, e in zip(blocks, eager):
            o = b.outputs()
            assert all(torch.equal(o[n], e[n]) for n in e)


def test_unit_variance():
    """Unit-normal operands: the tensors that the factors are for have unit variance (5 %, the bound of the other layers' tests)."""
    b = Block(2048, 256, 704, False, False, us.GATE_SILU)
    out = b.forward().backward().outputs()
    for n in ("Z", "H", "Y", "dX", "dWgu", "dWd"):
        assert abs(float(out[n][:-1].double().square().mean()) - 1) < 0.05, n
    assert abs(float(out["dZ"][:-1].double().square().mean()) - 1) < 0.05


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,d,f,forward,dz,grads", [
    (100, 256, 688, "32x64", "32x64", "three:32x64"),            # few tiles everywhere
    (700, 1040, 1552, "128x128:wk2", "128x128", None),           # two wave groups where the reduction has 2048 bytes (FP16)
    (1900, 256, 2064, "128x128", "128x128", None),
    (2064, 784, 2080, "256x256", "128x128", None),               # one round of large tiles instead of two of small ones
    (1333, 1248, 2496, None, None, "three:128x128"),
    (11000, 272, 2064, "256x256", "128x128", None),               # dZ with a short reduction: two workgroups per CU
])
def test_tiles_by_rule(T, d, f, forward, dz, grads, fp8):
    """One block inside every window of the choice of tiles; the results go by the definition whichever is taken."""
    for keep8 in (False, True):
        b = Block(T, d, f, fp8, keep8, us.GATE_SILU, seed=5)
        first = b.forward().outputs()
        taken = us.last_launch().split(" + ")[0]
        if forward and not (fp8 and ":wk2" in forward):
            assert forward in taken, taken
        check_forward(b, first)
        out = b.backward().outputs()
        launches = us.last_launch().split(" + ")
        if dz and not keep8:
            assert dz in launches[0], launches
        if grads:
            assert len(launches) == 4 and all(n.startswith(grads) for n in launches[1:]), launches
        check_backward(b, out)


@pytest.mark.parametrize("fp8", [False, True])
def test_wide_gradients_on_large_tiles(fp8):
    """dZ on large tiles (a long reduction in FP8 bytes, or 8-bit blocks), rows and columns that end inside a tile."""
    for T, d, f, keep8 in ((3000, 2576, 4112, False), (3000, 144, 4112, True)):
        b = Block(T, d, f, fp8, keep8, us.GATE_GELU, seed=6)
        b.forward().backward()
        assert us.last_launch().startswith("direct:256x256"), us.last_launch()
        check_backward(b, b.outputs())


@pytest.mark.parametrize("T,d,f", [(5, 1040, 4112), (16, 1040, 4112), (130, 528, 1040), (700, 512, 1552), (1024, 528, 2064)])
def test_codes_of_few_tokens_go_by_exact_sums(T, d, f):
    """FP8 with up to 1024 tokens: the sums of Z and dH are as good as FP32's, so that hardly a code of dZ falls on the other side of a border.

    Sums of FP16 products in FP32 are off by less than e = 4e-7 of a unit.  A value is rounded to the other neighbour with probability
    error / step: of Z (FP16, |z| >= 1/4, step 2^-12 and more) at most e / 2^-12 + 2^-24 / 2^-11 < 2e-3, where the FP8 adder's mean error of 1.05e-5 gives 1.5 % and
    more; of dZ (E5M2, relu: five FP32 roundings, |dH| >= 1/4, step an eighth of the value and more) at most (5 * 2^-24 + 4 e) * 8 < 2e-5, where the
    adder gives 8e-5.  Counts of a few are allowed three more.
    """
    b = Block(T, d, f, True, False, us.GATE_RELU, seed=11)
    b.forward().backward()
    out = b.outputs()
    X, Wgu, Wd, G = operand(b.X), operand(b.Wgu), operand(b.Wd), operand(b.G, True)
    Z = X @ Wgu / math.sqrt(d)
    at = Z.abs() >= 0.25
    moved = (out["Z"][:T] != Z.half()) & at
    assert int(moved.sum()) <= 2e-3 * int(at.sum()) + 3, (int(moved.sum()), int(at.sum()))
    zg, zu = kept(b, out)
    alpha, beta = us.gate_scales(us.GATE_RELU)
    alpha, beta = float(np.float32(alpha)), float(np.float32(beta))
    dH = G @ Wd.t() / math.sqrt(d)
    dZ = torch.cat([beta * (zg > 0) * zu * dH, alpha * zg.clamp(min=0) * dH], 1)
    at = (dZ.abs() >= 2.0 ** -14) & (torch.cat([dH, dH], 1).abs() >= 0.25)
    want = dZ.clamp(-57344, 57344).to(torch.float32).to(torch.float8_e5m2).view(torch.uint8)
    moved = (out["dZ"][:T] != want) & at
    assert int(moved.sum()) <= 2e-5 * int(at.sum()) + 3, (int(moved.sum()), int(at.sum()))


@pytest.mark.parametrize("T", [1024, 1025])
def test_the_launch_record_tells_how_codes_are_added(T):
    """The sums of Z and dH go by FP16 instructions up to 1024 tokens and by the FP8 ones beyond; the other products by the FP8 ones."""
    b = Block(T, 64, 96, True, False, us.GATE_SILU)
    for run in (b.forward, b.backward):
        run()
        first, *others = us.last_launch().split(" + ")
        assert ":fp8:" in first and first.endswith(":as16") == (T <= 1024), first
        assert others and not any(":as16" in n for n in others), others


@pytest.mark.parametrize("T,d,f,up,down", [(9, 2064, 5648, False, True), (32, 4112, 5136, True, True), (33, 2048, 5632, False, True), (64, 1040, 4112, False, True),
                                           (65, 1040, 4112, False, False), (17, 512, 1376, False, False)])
def test_a_few_rows_of_codes_in_slices(T, d, f, up, down):
    """... the same rule in FP8, whose weights have half of the bytes."""
    b = Block(T, d, f, True, False, us.GATE_SILU, seed=T)
    b.forward()
    launches = us.last_launch().split(" + ")
    assert ["partial" in n for n in launches] == [up, down], launches
    assert [n.endswith(":as16") for n in launches] == [True, False], launches


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("T,d,f,forward,dz", [
    (1100, 2048, 1600, "128x128:wk2", "128x128:wk2"),            # two wave groups in both directions
    (1027, 2064, 1616, "128x128:wk2", "128x128:wk2"),            # ... tokens, reduction and widths that end inside a tile and a block of 32
    (1100, 256, 416, "64x64", "32x64"),                          # few tiles
    (1100, 272, 800, "128x128:wk1", "64x64"),
    (1040, 144, 208, "32x64", "32x64"),
])
def test_tiles_of_the_fp8_adder(T, d, f, forward, dz, keep8):
    """FP8 with more than 1024 tokens: every tile of few rows of tiles, whose sums are the matrix core's FP8 sums."""
    b = Block(T, d, f, True, keep8, us.GATE_GELU, seed=T + f)
    first = b.forward().outputs()
    taken = us.last_launch().split(" + ")[0]
    assert forward in taken and ":as16" not in taken, taken
    check_forward(b, first)
    out = b.backward().outputs()
    taken = us.last_launch().split(" + ")[0]
    assert dz in taken and ":as16" not in taken, taken
    check_backward(b, out)


def nearest_codes(v, bits, least, top):
    """Values of the nearest FP8 codes (`bits` behind the leading one, exponents from `least`, clipped at `top`), and the step at each."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** least))) - bits)
    return ((v / step).round() * step).clamp(-top, top), step


@pytest.mark.parametrize("T", [512, 1024, 1025, 1400])
def test_gradients_end_to_end_on_both_sides_of_1024_tokens(T):
    """dX, dWgu and dWd against 64 bits from the operands' codes on, no tensor of the GPU's in between.

    What separates them are codes of dZ and H that fall on the other side of a border, each of which moves a value by its step, and Zg next to zero whose
    relu' comes out for the other sign, which moves dZ by all of its value; next to FP16's rounding of the results and the products' sums (3e-4 of the
    2-norm together, see above).  A sum that is off by e moves a code with probability |e| / step and a sign with |e| times a unit normal's density at
    zero.  |e| is on average 4/5 of the sum's rms error (normal), 1.3e-5 for the FP8 adder and 4e-8 for sums of exact products, times the derivative
    towards Zg, Zu and dH (kept Z's own rounding passes a shift on, on average); for dZ and H themselves five roundings of 2^-25 on average.  The
    moved energy therefore has the mean sum p E and the variance sum p E^2 over all elements (p: probability, E: the move's square): four standard deviations
    are allowed.  A product of independent operands keeps the ratio of 2-norms.
    Single elements: a code from 8 to 16 of dZ (step 2; larger ones are a few per tensor) next to an operand of 4 moves an element of dWgu by
    8 T^-1/2 of a unit, an eighth of that for dX, whose sum has 2f terms; H's steps are half as large.  Signs: no sum is off by more than 2e-4 of a
    unit with FP8 operands (parity.py), 2e-6 being 50 times the rms error of exact products' sums; whatever lies closer to zero may move."""
    d, f = 528, 1040
    b = Block(T, d, f, True, False, us.GATE_RELU, seed=T)
    b.forward()
    assert ":as16" in us.last_launch() or T > 1024
    out = b.backward().outputs()
    X, Wgu, Wd, G = operand(b.X), operand(b.Wgu), operand(b.Wd), operand(b.G, True)
    alpha, beta = (float(np.float32(v)) for v in us.gate_scales(us.GATE_RELU))
    Z = X @ Wgu / math.sqrt(d)
    on, near = (Z[:, :f] > 0).double(), (Z[:, :f].abs() <= (2e-6 if T <= 1024 else 2e-4)).double()
    H, h_step = nearest_codes(alpha * on * Z[:, :f] * Z[:, f:], 3, -6, 448.0)
    zg, zu = (z.half().double() for z in (Z[:, :f], Z[:, f:]))
    dH = G @ Wd.t() / math.sqrt(d)
    dZ, z_step = nearest_codes(torch.cat([beta * on * zu * dH, alpha * on * zg * dH], 1), 2, -14, 57344.0)
    unit = 0.8 * (4e-8 if T <= 1024 else 1.3e-5)
    e_z = unit * torch.cat([beta * on * (zu.abs() + dH.abs()), alpha * on * (zg.abs() + dH.abs())], 1) + 5 * 2.0 ** -25 * dZ.abs()
    e_h = unit * alpha * on * (zg.abs() + zu.abs()) + 5 * 2.0 ** -25 * H.abs()
    sign = beta * zu * dH

    def most_energy(*moves):
        mean, var = (sum(float((p * e.square() ** k).sum()) for p, e in moves) for k in (1, 2))
        return mean + 4 * math.sqrt(var)

    of_z = math.sqrt(most_energy((e_z / z_step, z_step), (unit * (2 * math.pi) ** -0.5, sign)) / float(dZ.square().sum()))
    of_h = math.sqrt(most_energy((e_h / h_step, h_step)) / float(H.square().sum()))
    jump = torch.cat([sign.abs() * near, torch.zeros_like(sign)], 1)
    for name, want, moved, jumps in (("dX", dZ @ Wgu.t() / math.sqrt(2 * f), of_z, jump @ Wgu.abs().t() / math.sqrt(2 * f)),
                                     ("dWgu", X.t() @ dZ / math.sqrt(T), of_z, X.abs().t() @ jump / math.sqrt(T)), ("dWd", H.t() @ G / math.sqrt(T), of_h, 0.0)):
        diff, rms = (out[name][:-1].double() - want).abs(), float(want.square().mean().sqrt())
        off = float(diff.square().mean().sqrt()) / rms
        assert off <= 3e-4 + moved, (name, off, moved)
        assert (diff <= 8 / math.sqrt(T) * rms + jumps).all(), (name, float((diff - jumps).max()) / rms)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("gate", range(4))
@pytest.mark.parametrize("T,f", [(5, 80), (700, 2064)])
def test_a_nan_of_the_gate_is_one_in_its_column(T, f, gate, fp8):
    """A NaN weight of the gate's half makes its columns of Z, H and dZ NaN, whatever the gate, and no other column of Z and dZ."""
    for keep8 in (False, True):
        b = Block(T, 64, f, fp8, keep8, gate, seed=2)
        b.g["Wgu"][3, 7] = 0x7f if fp8 else float("nan")
        out = b.forward().backward().outputs()
        zg, zu = kept(b, out)
        H, dZ = operand(out["H"][:T]), operand(out["dZ"][:T], True)
        hit = torch.zeros(2 * f, dtype=torch.bool)
        hit[7] = hit[f + 7] = True
        assert torch.isnan(zg[:, 7]).all() and not torch.isnan(zg[:, ~hit[:f]]).any() and not torch.isnan(zu).any()
        assert torch.isnan(H[:, 7]).all() and not torch.isnan(H[:, ~hit[:f]]).any()
        assert torch.isnan(dZ[:, hit]).all() and not torch.isnan(dZ[:, ~hit]).any(), [int(torch.isnan(dZ[:, c]).sum()) for c in (7, f + 7)]
