"""2-norm error of dQ where sum p dp is taken from the products themselves instead of the rounded O: heads of up to 32 columns over any keys that one workgroup has, up to 64
columns over 256 keys, wider ones over 128.  Peaked rows (queries of 3), in which O's rounding weighs most.  Both forms' errors are worked out here on the CPU, in 64 bits but for the roundings:
dS (and O) to FP16, then dQ; the kernel has to lie on the products' side of their middle."""
import pytest
import torch

import paper_2303_11257_amd as us
from test_gpu_attention_cross import Call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh,sk", [(16, 100), (16, 700), (16, 2000), (32, 130), (32, 1024), (48, 256), (64, 256), (80, 128), (96, 100), (128, 128), (192, 128), (256, 90)])
def test_few_keys_and_narrow_heads(dh, sk):
    batch, heads, sq = 8, 64, 32
    assert us.attention_cross_workspace_bytes(batch, heads, heads, sq, sk, dh) <= 16 * batch * heads * sq + 4096       # no parts
    c = Call(batch, heads, heads, sq, sk, dh, seed=dh + sk, sigma=3.0)
    c.fwd()
    c.bwd()
    got = c.t["dQ"].cpu().double()
    half = lambda x: x.half().double()      # noqa: E731
    Q, K, V, G = (x.double() for x in (c.Q, c.K, c.V, c.G))
    p = torch.softmax(torch.matmul(Q, K.transpose(2, 3).contiguous()) * dh ** -0.5, -1)
    a = sk ** 0.5
    dp = torch.matmul(G, V.transpose(2, 3).contiguous())
    D = (p * dp).sum(-1, keepdim=True)
    D_of_O = (G * half(a * torch.matmul(p, V))).sum(-1, keepdim=True) / a
    P = a * p
    want = torch.matmul(P * (dp - D), K) * dh ** -0.5
    error = lambda x: float((x - want).norm() / want.norm())      # noqa: E731
    products, from_o = (error(half(torch.matmul(half(P * (dp - d)), K) * dh ** -0.5)) for d in (D, D_of_O))
    mine = error(got)
    print(f"{dh} columns, {sk} keys: {mine:.3e}; from the products {products:.3e}, from O {from_o:.3e}")
    assert from_o > 1.15 * products
    assert mine < (products + from_o) / 2
