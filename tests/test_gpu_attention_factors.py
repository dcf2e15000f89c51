"""us_attention_cross_bwd with factors that the caller gives, far below the default of n^1/2: a p and a dS would be subnormal in FP16.

The gradients of a factor a are a / f times those of any other factor f, so that the definition with f, whose roundings tests/attend_ref.py counts, and with the other
factors times a / f bounds what the kernels may be off that round f p and f dS.  f = max(a, min(n^1/2, n / 2048)).  One error is a's own: O is rounded with it, 2^-25 at
least, which D = dO O / a takes over."""
import math

import pytest
import torch

import attend_ref as R
import paper_2303_11257_amd as us
from gpu_util import DEV, ptr, stream

pytestmark = pytest.mark.gpu


def gradients(Q, K, V, G, alpha, beta_q, beta_kv):
    batch, heads, sq, dh = Q.shape
    kv, sk = K.shape[1:3]
    q, k, v, g = (x.to(DEV) for x in (Q, K, V, G))
    o, dq, dk, dv = (torch.empty_like(x) for x in (q, q, k, v))
    lse = torch.empty(batch * heads, sq, device=DEV)
    wsb = us.attention_cross_workspace_bytes(batch, heads, kv, sq, sk, dh)
    ws = torch.empty(max(16, wsb), dtype=torch.uint8, device=DEV)
    us.attention_cross_fwd(ptr(q), ptr(k), ptr(v), None, ptr(o), ptr(lse), batch, heads, kv, sq, sk, dh, alpha, None, None, None, ptr(ws), wsb, stream())
    us.attention_cross_bwd(ptr(q), ptr(k), ptr(v), None, ptr(o), ptr(lse), ptr(g), ptr(dq), ptr(dk), ptr(dv), batch, heads, kv, sq, sk, dh, alpha, beta_q, beta_kv,
                           None, None, None, ptr(ws), wsb, stream())
    torch.cuda.synchronize()
    return dict(dQ=dq, dK=dk, dV=dv)


@pytest.mark.parametrize("dh,heads,kv", [(16, 1, 1), (64, 4, 2), (80, 2, 2), (128, 2, 1), (160, 1, 1)])
@pytest.mark.parametrize("inputs", ["equal queries", "signs", "normal"])
@pytest.mark.parametrize("sq,sk", [(48, 1000), (20, 6000), (2000, 1000)])
def test_small_factors(sq, sk, inputs, dh, heads, kv):
    """a p = 100.5 steps of FP16's subnormal numbers: rounded so it is off by 5e-3 of itself, and so are gradients whose terms are all alike; two roundings of normal numbers
    allow them 2^-10.  "equal queries": no key stands out and all queries are one; "signs": no query prefers a key, keys and values are one row and its negative."""
    g = torch.Generator().manual_seed(sk + dh)
    r = lambda *s: torch.randn(*s, generator=g).half()      # noqa: E731
    Q, K, V, G = r(1, heads, sq, dh), r(1, kv, sk, dh), r(1, kv, sk, dh), r(1, heads, sq, dh)
    if inputs == "equal queries":
        K.zero_()
        Q[:], G[:] = Q[:, :, :1].clone(), G[:, :, :1].clone()
    elif inputs == "signs":
        Q.zero_()
        sign = torch.where(torch.arange(sk) % 2 == 0, 1.0, -1.0).half()[None, None, :, None]
        K[:] = sign * K[:, :, :1].clone()
        V[:], G[:] = sign * 0.25, 4.0 / dh                  # dO v = +-1 (dh = 80, 160: within 2^-11)
    alpha = 100.5 * 2.0 ** -24 * sk
    beta_q, beta_kv = 0.5 * dh ** 0.5 / alpha, sk / (alpha * sq)
    f = max(alpha, min(math.sqrt(sk), sk / 2048))
    assert f > alpha
    got = gradients(Q, K, V, G, alpha, beta_q, beta_kv)
    want = R.cross(Q, K, V, None, f, G, beta_q * alpha / f, beta_kv * alpha / f)
    # O's roundings to steps of 2^-24, half a step each, in the forward pass and in what the bound takes O to be
    rep, c = heads // kv, dh ** -0.5
    for h in range(heads):
        q, k = Q[0, h].double(), K[0, h // rep].double()
        p = torch.softmax(q @ k.t() * c, 1)
        off = 2 * R.TINY / alpha * G[0, h].double().abs().sum(1, keepdim=True)
        want["dQ"][1][0, h] += alpha * beta_q * c * ((p * off) @ k.abs())
        want["dK"][1][0, h // rep] += alpha * beta_kv * c * ((p * off).t() @ q.abs())
    for n in ("dQ", "dK", "dV"):
        R.close(got[n], want[n], f"{inputs} {n}")


@pytest.mark.parametrize("alpha,sk", [(1.0, 131072), (0.125, 16384)])
def test_rounding_of_long_rows(alpha, sk):
    """2-norm errors of unit normal inputs.  A rounding to FP16 is off by at most 2^-11 / 3^1/2 of a 2-norm, evenly spread over half a step on either side of numbers at the
    lower end of their power of two; three of them (f p or f dS, the result, O within D), independent: 2^-11."""
    heads, sq, dh = 2, 24, 32
    g = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(*s, generator=g).half()      # noqa: E731
    Q, K, V, G = r(1, heads, sq, dh), r(1, 1, sk, dh), r(1, 1, sk, dh), r(1, heads, sq, dh)
    betas = 32.0 / alpha, sk / 8 / alpha
    got = gradients(Q, K, V, G, alpha, *betas)
    c = dh ** -0.5
    q, k, v, d = Q[0].double(), K[0, 0].double(), V[0, 0].double(), G[0].double()
    P = torch.softmax(torch.matmul(q, k.t()) * c, -1)
    dp = torch.matmul(d, v.t())
    ds = P * (dp - (P * dp).sum(-1, keepdim=True)) * alpha
    want = dict(dQ=torch.matmul(ds, k) * c * betas[0], dK=torch.matmul(ds.transpose(1, 2).contiguous(), q).sum(0) * c * betas[1],
                dV=torch.matmul(P.transpose(1, 2).contiguous(), d).sum(0) * alpha * betas[1])
    for n, w in want.items():
        e = float((got[n].cpu().double().view(w.shape) - w).norm() / w.norm())
        print(n, e)
        assert e < 2.0 ** -11, (n, e)
