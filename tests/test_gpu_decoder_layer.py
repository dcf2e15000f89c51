"""The operators as a layer uses them: projection -> norms, rotation and heads (shared keys and values) -> attention -> projection with residual ->
gated block with 8-bit checkpoints -> backward through all of it, the layer's input and attention's input kept in 8 bits meanwhile."""
import math

import numpy as np
import pytest
import torch

import gated_ref as R
import paper_2303_11257_amd as us
from gpu_util import DEV, ptr, stream

pytestmark = pytest.mark.gpu


def rms(x):
    return float(x.double().square().mean().sqrt())


def test_layer_forward_and_backward():
    batch, s, h, kv, dh, f = 3, 48, 4, 2, 32, 352
    d, T, cols = h * dh, batch * s, (h + 2 * kv) * dh
    gen = torch.Generator().manual_seed(11)
    host = {n: torch.randn(sh, generator=gen).half() for n, sh in dict(X=(T, d), Wqkv=(d, cols), Wo=(d, d), Wgu=(d, 2 * f), Wd=(f, d), G=(T, d)).items()}
    t = {n: v.to(DEV) for n, v in host.items()}
    new = lambda *sh, dt=torch.float16: torch.empty(sh, dtype=dt, device=DEV)      # noqa: E731
    freq = 10000.0 ** (-torch.arange(dh // 2, dtype=torch.float64) / (dh // 2))
    t["freq"] = freq.to(DEV)
    st, F16 = stream(), us.F16

    def keep(x, rows, n):
        codes, scales = new(rows, n, dt=torch.int8), new(rows, us.keep8_blocks(n), dt=torch.uint8)
        us.keep8_store(ptr(x), n, ptr(codes), ptr(scales), rows, n, st)
        return codes, scales, n

    def load(k):
        codes, scales, n = k
        x = new(codes.shape[0], n)
        us.keep8_load(ptr(codes), ptr(scales), ptr(x), n, codes.shape[0], n, st)
        return x

    # forward
    qkv = new(T, cols)
    us.linear_fwd(ptr(t["X"]), ptr(t["Wqkv"]), ptr(qkv), T, d, cols, F16, F16, stream=st)
    Q, K, V = new(batch * h, s, dh), new(batch * h, s, dh), new(batch * h, s, dh)
    us.qk_norm_rope_fwd(ptr(qkv), cols, None, None, None, ptr(t["freq"]), ptr(Q), ptr(K), ptr(V), batch, s, h, kv, dh, dh, us.ROPE_HALVES, 1e-6, st)
    A, P, O = new(batch * h, s, s), new(batch * h, s, s), new(batch * h, s, dh)
    us.attention_fwd(ptr(Q), ptr(K), ptr(V), ptr(A), ptr(P), ptr(O), batch * h, s, dh, st)
    merged = O.view(batch, h, s, dh).transpose(1, 2).reshape(T, d).contiguous()
    mid = new(T, d)
    us.linear_fwd(ptr(merged), ptr(t["Wo"]), ptr(mid), T, d, d, F16, F16, stream=st)
    us.weighted_add(ptr(mid), ptr(t["X"]), ptr(mid), T * d, F16, math.sqrt(0.5), math.sqrt(0.5), st)
    Z, Zs, H, Y = new(T, 2 * f, dt=torch.int8), new(T, 2 * us.keep8_blocks(f), dt=torch.uint8), new(T, f), new(T, d)
    us.ffn_gated_fwd(ptr(mid), ptr(t["Wgu"]), ptr(t["Wd"]), ptr(Z), ptr(Zs), ptr(H), ptr(Y), T, d, f, us.GATE_SILU, us.FFN_KEEP8, None, 0, st)
    kept = dict(X=keep(t["X"], T, d), qkv=keep(qkv, T, cols), mid=keep(mid, T, d))
    ref_mid, ref_qkv = mid.clone(), qkv.clone()
    qkv.zero_(), mid.zero_(), H.zero_()                        # what is not kept is gone

    # backward
    mid_, qkv_, X_ = load(kept["mid"]), load(kept["qkv"]), load(kept["X"])
    wsb = max(us.ffn_gated_workspace_bytes(T, d, f, us.FFN_KEEP8), us.workspace_bytes(T, d, cols), us.qk_norm_rope_workspace_bytes(batch, s, h, kv, dh), 16)
    ws = new(wsb, dt=torch.uint8)
    dZ, dmid, dWgu, dWd = new(T, 2 * f), new(T, d), new(d, 2 * f), new(f, d)
    us.ffn_gated_bwd(ptr(mid_), ptr(t["Wgu"]), ptr(t["Wd"]), ptr(Z), ptr(Zs), ptr(H), ptr(t["G"]), ptr(dZ), ptr(dmid), ptr(dWgu), ptr(dWd), T, d, f, us.GATE_SILU,
                     us.FFN_KEEP8, ptr(ws), wsb, st)
    dmerged, dWo = new(T, d), new(d, d)
    us.linear_bwd(ptr(merged), ptr(t["Wo"]), ptr(dmid), ptr(dmerged), ptr(dWo), T, d, d, F16, F16, F16, workspace=ptr(ws), workspace_bytes=wsb, stream=st)
    dO = dmerged.view(batch, s, h, dh).transpose(1, 2).reshape(batch * h, s, dh).contiguous()
    dP, dA, dQ, dK, dV = new(batch * h, s, s), new(batch * h, s, s), *(new(batch * h, s, dh) for _ in range(3))
    us.attention_bwd(ptr(Q), ptr(K), ptr(V), ptr(A), ptr(P), ptr(dO), ptr(dP), ptr(dA), ptr(dQ), ptr(dK), ptr(dV), batch * h, s, dh, st)
    dqkv, dX, dWqkv = new(T, cols), new(T, d), new(d, cols)
    us.qk_norm_rope_bwd(ptr(qkv_), cols, None, None, None, ptr(t["freq"]), ptr(dQ), ptr(dK), ptr(dV), ptr(dqkv), cols, None, None, batch, s, h, kv, dh, dh,
                        us.ROPE_HALVES, 1e-6, 0.0, 0.0, ptr(ws), wsb, st)
    us.linear_bwd(ptr(X_), ptr(t["Wqkv"]), ptr(dqkv), ptr(dX), ptr(dWqkv), T, d, cols, F16, F16, F16, workspace=ptr(ws), workspace_bytes=wsb, stream=st)
    torch.cuda.synchronize()

    # the same layer in 64 bits
    X, Wqkv, Wo, Wgu, Wd, G = (host[n].double() for n in ("X", "Wqkv", "Wo", "Wgu", "Wd", "G"))
    q8 = lambda x: torch.from_numpy(R.keep8_values(*R.keep8(x.numpy())))      # noqa: E731
    pos = torch.arange(s).repeat(batch)
    heads_out = lambda y: y.view(batch, s, -1, dh).permute(0, 2, 1, 3).repeat_interleave(h // y.shape[1], 1).reshape(batch * h, s, dh)      # noqa: E731
    r_qkv = X @ Wqkv / math.sqrt(d)

    def norm(x):
        return (x.square().mean(-1, keepdim=True) + 1e-6) ** -0.5

    x = r_qkv.view(T, h + 2 * kv, dh)
    q, k = (R.turned(y * norm(y), pos, freq, dh, False) for y in (x[:, :h], x[:, h: h + kv]))
    q, k, v = heads_out(q), heads_out(k), heads_out(x[:, h + kv:])
    p = torch.softmax(q @ k.transpose(1, 2) / math.sqrt(dh), -1)
    o = math.sqrt(s) * p @ v                                   # P = s softmax, O = s^-1/2 P V
    r_merged = o.view(batch, h, s, dh).transpose(1, 2).reshape(T, d)
    r_mid = (r_merged @ Wo / math.sqrt(d) + X) * math.sqrt(0.5)
    a, bg = us.gate_scales(us.GATE_SILU)
    r_z = r_mid @ Wgu / math.sqrt(d)
    r_y = (a * R.gate_value("silu", r_z[:, :f]) * r_z[:, f:]) @ Wd / math.sqrt(f)
    zg, zu = q8(r_z[:, :f]), q8(r_z[:, f:])
    dh_ = G @ Wd.t() / math.sqrt(d)
    r_dz = torch.cat([bg * R.gate_slope("silu", zg) * zu * dh_, a * R.gate_value("silu", zg) * dh_], 1)
    r_dmid = r_dz @ Wgu.t() / math.sqrt(2 * f)
    r_dWgu, r_dWd = q8(r_mid).t() @ r_dz / math.sqrt(T), (a * R.gate_value("silu", zg) * zu).t() @ G / math.sqrt(T)
    r_do = (r_dmid @ Wo.t() / math.sqrt(d)).view(batch, s, h, dh).transpose(1, 2).reshape(batch * h, s, dh)
    r_dv = s ** -0.5 * s * p.transpose(1, 2) @ r_do
    dp = r_do @ v.transpose(1, 2) / math.sqrt(dh)
    da = s * p * (dp - (p * dp).sum(-1, keepdim=True))
    r_dq, r_dk = da @ k / math.sqrt(s), da.transpose(1, 2) @ q / math.sqrt(s)
    xk = q8(r_qkv).view(T, h + 2 * kv, dh)
    parts = []
    for g, y in ((r_dq, xk[:, :h]), (r_dk, xk[:, h: h + kv])):
        n = y.shape[1]
        g = g.view(batch, n, h // n, s, dh).sum(2).permute(0, 2, 1, 3).reshape(T, n, dh) / math.sqrt(h // n)
        g = R.turned(g, pos, freq, dh, False, back=True)
        r = norm(y)
        parts.append(r * (g - y * r * (g * y * r).mean(-1, keepdim=True)))
    parts.append(r_dv.view(batch, kv, h // kv, s, dh).sum(2).permute(0, 2, 1, 3).reshape(T, kv, dh) / math.sqrt(h // kv))
    r_dqkv = torch.cat(parts, 1).reshape(T, cols)
    r_dX, r_dWqkv = r_dqkv @ Wqkv.t() / math.sqrt(cols), q8(X).t() @ r_dqkv / math.sqrt(T)

    # Every FP16 tensor of the chain adds a rounding of at most 2^-11 / sqrt(3) = 2.8e-4 rms of independent sign; in front of the gated block there are
    # six of them (qkv, Q, K, A, P, O, mid), passed on with factors of about one: below 2^-10 rms of qkv, mid and, with Z's and H's, 2^-9 of Y.
    # A kept value takes its neighbour's code where an error e moves it across a border: probability 0.8 e / step, error one step, so
    # (0.8 e step)^1/2 rms.  Blocks of 32 normal values reach 2 to 4 sigma, step 2^-5: with e = 2^-10, 5e-3.  H and dZ hold two such factors,
    # 7e-3 < 2^-7; what comes after is made from dmid (2^-7), the kept qkv (5e-3) and the softmax's two products with dmid's error: (7e-3^2 +
    # 7e-3^2 + 5e-3^2)^1/2 = 1.1e-2 < 2^-6.
    bounds = dict(qkv=2.0 ** -10, mid=2.0 ** -10, Y=2.0 ** -9, dWd=2.0 ** -7, dWgu=2.0 ** -7, dmid=2.0 ** -7, dqkv=2.0 ** -6, dX=2.0 ** -6, dWqkv=2.0 ** -6)
    for name, got, want in (("qkv", ref_qkv, r_qkv), ("mid", ref_mid, r_mid), ("Y", Y, r_y), ("dWd", dWd, r_dWd), ("dWgu", dWgu, r_dWgu), ("dmid", dmid, r_dmid),
                            ("dqkv", dqkv, r_dqkv), ("dX", dX, r_dX), ("dWqkv", dWqkv, r_dWqkv)):
        e = rms(got.cpu().double() - want) / rms(want)
        print(name, "rms error", e)
        assert e <= bounds[name], (name, e)
