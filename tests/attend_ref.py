"""Attention over another sequence's keys, over a paged cache, and the cache's eviction, by their definitions in 64 bits on the CPU, each computed value
with the bound that the kernels' roundings allow it.

Roundings counted (u = 2^-11, half a step of FP16; v = 2^-24, of FP32):
  scores     s = c q k, FP32 sums of dh exact products: at most (dh + 4) v c sum |q k| off, as is the exponent that is made of s and its row's maximum or L (whose
             own rounding is v |L|): e of a probability, relative, twice for its sum, with n v for the sum's additions
  p, a p     rounded to FP16: u relative, 2^-25 absolute below FP16's normal numbers (of the largest p, which is 1 there)
  ds         u of itself; p's e of itself; the error of dp and of D = dO O / a, O being rounded (u |O|), times a p; 2^-25 absolute
  products   FP32 sums of at most m terms: m v of the sum of magnitudes;  the result's rounding: u of itself, or 2^-25
"""
import math

import torch

U, V, TINY = 2.0 ** -11, 2.0 ** -24, 2.0 ** -25


def _scores(q, k, n, dh):
    c = dh ** -0.5
    s = q @ k[:n].t() * c
    worst = (q.abs() @ k[:n].abs().t()).amax(1, keepdim=True) * c
    return s, (dh + 8) * V * worst + 4 * V * worst


def _rounded(x, error):
    return error + U * (x.abs() + error) + TINY


def rows_forward(q, k, v, n, alpha):
    """q [rows, dh], k, v [n.., dh] -> O, its bound, p, lse, e (p's relative error) of one head."""
    rows, dh = q.shape
    if n == 0:
        z = torch.zeros(rows, v.shape[1], dtype=torch.float64)
        return z, z, torch.zeros(rows, 0, dtype=torch.float64), torch.full((rows,), -math.inf, dtype=torch.float64), torch.zeros(rows, 1, dtype=torch.float64)
    a = alpha if alpha > 0 else math.sqrt(n)
    s, es = _scores(q, k, n, dh)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    top = p.amax(1, keepdim=True)
    e = 2 * es + (n + 40) * V
    o = a * (p @ v[:n])
    mag = a * (p @ v[:n].abs())
    err = (U + e + (n + 40) * V) * mag + a * TINY * top * v[:n].abs().sum(0)
    return o, _rounded(o, err), p, lse, e + V * lse.abs()[:, None] * 3


def cross(Q, K, V_, klen, alpha=0.0, dO=None, beta_q=0.0, beta_kv=0.0):
    """Q [batch, heads, sq, dh], K, V [batch, kv, sk, dh] (any type) -> {"O": (value, bound), "lse": .., "dQ", "dK", "dV"}."""
    B, h, sq, dh = Q.shape
    kv, sk = K.shape[1:3]
    r = h // kv
    bq = beta_q if beta_q > 0 else 1.0
    bkv = beta_kv if beta_kv > 0 else math.sqrt(sk / sq * kv / h) if sq else 1.0
    z = lambda *sh: torch.zeros(sh, dtype=torch.float64)      # noqa: E731
    out = {"O": (z(B, h, sq, dh), z(B, h, sq, dh)), "lse": (z(B, h, sq), z(B, h, sq))}
    if dO is not None:
        out.update({n: (z(*x.shape), z(*x.shape)) for n, x in (("dQ", Q), ("dK", K), ("dV", V_))})
    c = dh ** -0.5
    for b in range(B):
        n = sk if klen is None else max(0, min(sk, int(klen[b])))
        for hd in range(h):
            q, k, v = Q[b, hd].double(), K[b, hd // r, :n].double(), V_[b, hd // r, :n].double()
            o, eo, p, lse, e = rows_forward(q, k, v, n, alpha)
            out["O"][0][b, hd], out["O"][1][b, hd] = o, eo
            out["lse"][0][b, hd], out["lse"][1][b, hd] = lse, (e[:, 0] + 8 * V * lse.abs()) if n else 0.0
            if dO is None or n == 0:
                continue
            a = alpha if alpha > 0 else math.sqrt(n)
            g = dO[b, hd].double()
            P = a * p
            dp = g @ v.t()
            D = (p * dp).sum(1, keepdim=True)
            edp = (dh + 4) * V * (g.abs() @ v.abs().t()) + ((g.abs() * (U * o.abs() + TINY)).sum(1, keepdim=True) + (dh + 4) * V * (g.abs() * o.abs()).sum(1, keepdim=True)) / a
            # (O that the backward pass reads is itself within its bound of o)
            edp = edp + (g.abs() * eo).sum(1, keepdim=True) / a
            ds = P * (dp - D)
            eds = (U + e) * ds.abs() + P * (1 + e) * edp * (1 + U) + TINY
            if n == 1:
                ds, eds = ds * 0, eds * 0
            eP = (U + e) * P + TINY
            m = sq * r + 40
            dq = bq * c * (ds @ k)
            out["dQ"][0][b, hd] = dq
            out["dQ"][1][b, hd] = _rounded(dq, bq * c * ((eds + (n + 40) * V * ds.abs()) @ k.abs()))
            for name, x, ex, y, f in (("dK", ds, eds, q, bkv * c), ("dV", P, eP, g, bkv)):
                out[name][0][b, hd // r, :n] += f * (x.t() @ y)
                out[name][1][b, hd // r, :n] += f * ((ex + m * V * x.abs()).t() @ y.abs())
    if dO is not None:
        for name in ("dK", "dV"):
            x, e = out[name]
            out[name] = (x, torch.where(e > 0, _rounded(x, e), e))
    return out


def close(got, want, what):
    """Every value within its bound; NaN where NaN is due."""
    value, bound = want
    got = got.detach().cpu().double()
    assert got.shape == value.shape, what
    same = (got == value) | (got.isnan() & value.isnan())
    off = torch.where(same, torch.zeros_like(value), (got - value).abs())
    worst = float((off / bound.clamp_min(1e-300)).max()) if off.numel() else 0.0
    print(f"{what}: largest error {float(off.max()) if off.numel() else 0.0:.2e}, {worst:.3f} of its bound")
    assert bool(((off <= bound) | same).all()), (what, worst)


# ---- the cache -------------------------------------------------------------------------------------------------------------

def position(table, b, i, page, pages):
    """Page and slot of a position, or None."""
    if i < 0 or i // page >= table.shape[1]:
        return None
    p = int(table[b, i // page])
    return (p, i % page) if 0 <= p < pages else None


def evict(W, table, lens, page, max_len, keep, recent):
    """kept [batch][kv head] lists of positions, by sorting; W [pages, kv, page]."""
    pages, kv, _ = W.shape
    kept = []
    for b in range(table.shape[0]):
        n = max(0, min(int(lens[b]), max_len, table.shape[1] * page))
        heads = []
        for h in range(kv):
            if n <= keep:
                heads.append(list(range(n)))
                continue

            def rank(i):
                at = position(table, b, i, page, pages)
                w = -math.inf if at is None else float(W[at[0], h, at[1]])
                return (0 if at is None else 2 if math.isnan(w) else 1, 0.0 if math.isnan(w) else w)
            first = sorted(range(n - recent), key=lambda i: (-rank(i)[0], -rank(i)[1], i))[: keep - recent]
            heads.append(sorted(first) + list(range(n - recent, n)))
        kept.append(heads)
    return kept
