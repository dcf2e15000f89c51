"""us_attention_cross_fwd / _bwd against the definition in 64 bits (tests/attend_ref.py, where the bounds are derived)."""
import math

import pytest
import torch

import attend_ref as R
import paper_2303_11257_amd as us
from gpu_util import DEV, ptr, stream

pytestmark = pytest.mark.gpu
F = torch.float16


def heads_view(buf, batch, heads, s, dh, lay, offset=0):
    """[batch, heads, s, dh] view of a flat buffer by a layout."""
    return torch.as_strided(buf, (batch, heads, s, dh), (lay.batch, lay.head, lay.row, 1), offset)


class Call:
    """One set of tensors, laid out as asked, guards around and between what is written."""

    def __init__(self, batch, heads, kv, sq, sk, dh, klen=None, layout="packed", seed=0, sigma=1.0, alpha=0.0, beta_q=0.0, beta_kv=0.0, fill=0.0):
        g = torch.Generator().manual_seed(seed)
        self.dims, self.alpha, self.betas = (batch, heads, kv, sq, sk, dh), alpha, (beta_q, beta_kv)
        r = lambda *s, f=1.0: (torch.randn(*s, generator=g) * f).half()      # noqa: E731
        self.Q, self.K, self.V, self.G = r(batch, heads, sq, dh, f=sigma), r(batch, kv, sk, dh), r(batch, kv, sk, dh), r(batch, heads, sq, dh)
        self.klen = klen
        if klen is not None and fill is not None:
            for b, n in enumerate(klen):                 # what no result may see
                self.K[b, :, max(0, n):], self.V[b, :, max(0, n):] = fill, fill
        pad = 0
        if layout == "packed":
            self.lq = self.lkv = self.lo = None
            q = o = us.HeadsLayout(heads * sq * dh, sq * dh, dh)
            k = us.HeadsLayout(kv * sk * dh, sk * dh, dh)
        elif layout == "tokens":                         # a token's heads side by side
            q = o = us.HeadsLayout(sq * heads * dh, dh, heads * dh)
            k = us.HeadsLayout(sk * 2 * kv * dh, dh, 2 * kv * dh)
            self.lq, self.lkv, self.lo = q, k, o
        else:                                            # gaps everywhere, another order for each
            pad = 24
            q = us.HeadsLayout(dh + 8, batch * (dh + 8), heads * batch * (dh + 8) + pad)
            k = us.HeadsLayout(kv * (sk * (dh + 16) + 8) + 40, sk * (dh + 16) + 8, dh + 16)
            o = us.HeadsLayout(sq * (heads * dh + 16), dh, heads * dh + 16)
            self.lq, self.lkv, self.lo = q, k, o
        size = lambda lay, n, s: lay.batch * max(0, batch - 1) + lay.head * (n - 1) + lay.row * max(0, s - 1) + dh + 64      # noqa: E731
        nq, nk, no = size(q, heads, sq), size(k, kv, sk), size(o, heads, sq)
        two = k.row >= 2 * kv * dh and layout == "tokens"
        mark = float("nan") if layout == "gaps" else 0.0
        self.bufs = {n: torch.full((m,), mark, dtype=F, device=DEV) for n, m in (("Q", nq), ("K", nk), ("V", nk), ("dO", no))}
        for n, m in (("O", no), ("dQ", nq), ("dK", nk), ("dV", nk)):
            self.bufs[n] = torch.full((m,), 7.0, dtype=F, device=DEV)
        lay = dict(Q=(q, heads, sq), dQ=(q, heads, sq), K=(k, kv, sk), V=(k, kv, sk), dK=(k, kv, sk), dV=(k, kv, sk), O=(o, heads, sq), dO=(o, heads, sq))
        self.t = {n: heads_view(self.bufs[n], batch, x[1], x[2], dh, x[0]) for n, x in lay.items()} if batch else {}
        for n, x in (("Q", self.Q), ("K", self.K), ("V", self.V), ("dO", self.G)):
            self.t[n].copy_(x)
        self.two = two
        self.kl = None if klen is None else torch.tensor(klen, dtype=torch.int32, device=DEV)
        self.lse = torch.full((batch * heads, max(1, sq)), 5.0, dtype=torch.float32, device=DEV)
        self.wsb = us.attention_cross_workspace_bytes(batch, heads, kv, sq, sk, dh)
        self.ws = torch.full((max(16, self.wsb) + 64,), 0xEE, dtype=torch.uint8, device=DEV)

    def fwd(self, workspace=True, lse=True, st=None):
        p, d = {n: ptr(x) for n, x in self.bufs.items()}, self.dims
        us.attention_cross_fwd(p["Q"], p["K"], p["V"], ptr(self.kl), p["O"], ptr(self.lse) if lse else None, *d, self.alpha, self.lq, self.lkv, self.lo,
                               ptr(self.ws) if workspace else None, self.wsb if workspace else 0, stream() if st is None else st)

    def bwd(self, st=None):
        p, d = {n: ptr(x) for n, x in self.bufs.items()}, self.dims
        us.attention_cross_bwd(p["Q"], p["K"], p["V"], ptr(self.kl), p["O"], ptr(self.lse), p["dO"], p["dQ"], p["dK"], p["dV"], *d, self.alpha, *self.betas,
                               self.lq, self.lkv, self.lo, ptr(self.ws), self.wsb, stream() if st is None else st)

    def reference(self, back=True):
        klen = self.klen
        return R.cross(self.Q, self.K, self.V, klen, self.alpha, self.G if back else None, *self.betas)

    def check(self, back=True, what=""):
        torch.cuda.synchronize()
        want = self.reference(back)
        R.close(self.t["O"], want["O"], what + "O")
        R.close(self.lse.view(*want["lse"][0].shape), want["lse"], what + "lse")
        for n in ("dQ", "dK", "dV") if back else ():
            R.close(self.t[n], want[n], what + n)
        # nothing beside the rows was written
        for n in ("O", "dQ", "dK", "dV") if back else ("O",):
            rest = self.bufs[n].clone()
            heads_view(rest, self.dims[0], self.t[n].shape[1], self.t[n].shape[2], self.dims[5], us.HeadsLayout(*self.t[n].stride()[:3])).fill_(7.0)
            assert bool((rest == 7.0).all()), what + n
        assert bool((self.ws[max(16, self.wsb):] == 0xEE).all())


SHAPES = [
    # batch, heads, kv, sq, sk, dh
    (1, 1, 1, 1, 1, 16), (2, 2, 1, 3, 2, 32), (1, 2, 2, 17, 63, 64), (1, 2, 2, 33, 64, 64), (2, 4, 2, 31, 65, 48), (1, 3, 3, 129, 127, 80), (1, 8, 2, 128, 130, 96),
    (1, 2, 1, 100, 257, 112), (1, 2, 2, 65, 193, 128), (1, 2, 1, 40, 97, 160), (1, 2, 2, 70, 66, 192), (1, 1, 1, 35, 129, 208), (1, 4, 1, 50, 70, 256),
    # one and a few queries: the rows of a key head's sharing heads together
    (3, 4, 4, 1, 300, 64), (2, 8, 1, 1, 129, 128), (1, 16, 1, 1, 1000, 96), (2, 4, 2, 7, 31, 80), (1, 2, 1, 8, 515, 256), (1, 6, 3, 5, 33, 16), (2, 3, 3, 16, 200, 192),
    # up to 128 keys and just beyond, every width, many queries over them (sums in parts)
    (1, 2, 1, 70, 128, 32), (1, 2, 2, 33, 128, 64), (2, 2, 2, 100, 128, 96), (1, 4, 2, 65, 128, 128), (1, 2, 2, 40, 127, 16), (1, 1, 1, 32, 16, 128), (1, 2, 1, 70, 129, 32),
    (1, 2, 1, 1100, 128, 64), (1, 1, 1, 2000, 77, 128), (2, 2, 1, 700, 5, 80), (1, 1, 1, 64, 128, 144), (2, 3, 3, 2, 100, 112),
    # few queries over many keys, and the other way round: reductions in parts
    (1, 1, 1, 40, 3000, 64), (1, 2, 1, 20, 2500, 128), (1, 1, 1, 2900, 40, 64), (1, 4, 1, 1500, 33, 80), (1, 1, 1, 1, 5001, 32), (1, 1, 1, 30, 1400, 256),
]


@pytest.mark.parametrize("dims", SHAPES, ids=str)
def test_forward_and_backward(dims):
    c = Call(*dims, seed=hash(dims) % 1000)
    c.fwd()
    c.bwd()
    c.check(what=f"{dims} ")


@pytest.mark.parametrize("klen", [[0, 1, 2, 70], [70, 69, 64, 63], [65, 33, 0, 200], [-5, 1, 1, 1], [0, 0, 0, 0]], ids=str)
@pytest.mark.parametrize("sq,heads,dh", [(1, 2, 64), (37, 4, 80), (140, 2, 128), (37, 2, 160)])
@pytest.mark.parametrize("fill", [float("nan"), float("inf"), -65504.0])
def test_lengths_hide_what_lies_behind(klen, sq, heads, dh, fill):
    """Keys and values behind an item's length are NaN, infinite or FP16's lowest; lengths beyond sk are cut to it; no key, one key."""
    c = Call(4, heads, 2, sq, 70, dh, klen=klen, seed=sq + klen[0], fill=fill)
    c.fwd()
    c.bwd()
    c.check(what=f"{klen} ")
    for b, n in enumerate(klen):
        if n <= 1:
            assert bool((c.t["dQ"][b] == 0).all()) and bool((c.t["dK"][b] == 0).all())
        assert bool((c.t["dK"][b, :, max(0, min(70, n)):] == 0).all()) and bool((c.t["dV"][b, :, max(0, min(70, n)):] == 0).all())
        if n <= 0:
            assert bool((c.t["O"][b] == 0).all()) and bool((c.lse.view(4, heads, sq)[b] == -math.inf).all())


@pytest.mark.parametrize("layout", ["tokens", "gaps"])
@pytest.mark.parametrize("dims", [(2, 4, 2, 37, 83, 80), (3, 2, 2, 1, 200, 64), (2, 2, 1, 130, 300, 128), (1, 2, 1, 24, 2000, 64), (2, 2, 2, 1300, 20, 64)], ids=str)
def test_layouts(dims, layout):
    c = Call(*dims, klen=[dims[4] - 3 * b for b in range(dims[0])], layout=layout, seed=5, fill=float("nan"))
    c.fwd()
    c.bwd()
    c.check(what=f"{layout} ")


@pytest.mark.parametrize("sigma", [0.0, 8.0, 60.0])
@pytest.mark.parametrize("dims", [(1, 2, 1, 50, 150, 64), (2, 2, 2, 1, 150, 128)], ids=str)
def test_even_and_peaked_rows(dims, sigma):
    """All scores equal; one key with nearly all of the weight; scores of several hundred."""
    c = Call(*dims, seed=3, sigma=sigma)
    c.fwd()
    c.bwd()
    c.check(what=f"sigma {sigma} ")


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("sq", [1, 40])
def test_scores_far_from_zero(sign, sq):
    """All scores near +-700: exponentials of them as they are would be infinite or zero; so would those of the columns that fill a tile."""
    c = Call(1, 2, 1, sq, 77, 64, seed=9)
    c.Q.fill_(sign * 8.0)
    c.K.copy_((c.K.float() * 0.05 + 11.0).half())
    c.t["Q"].copy_(c.Q), c.t["K"].copy_(c.K)
    c.fwd()
    c.bwd()
    c.check(what=f"{sign} ")


def test_factors():
    c = Call(2, 4, 2, 45, 90, 64, klen=[90, 33], alpha=0.5, beta_q=2.0, beta_kv=0.25, seed=11)
    c.fwd()
    c.bwd()
    c.check()


@pytest.mark.parametrize("dims", [(1, 2, 1, 64, 3000, 64), (1, 2, 2, 1, 3000, 128), (2, 2, 2, 50, 60, 80)], ids=str)
def test_forward_without_workspace_or_lse(dims):
    c = Call(*dims, seed=1)
    c.fwd(workspace=False)
    c.check(back=False)
    c.lse.fill_(5.0), c.bufs["O"].fill_(7.0)
    c.fwd(lse=False)
    torch.cuda.synchronize()
    assert bool((c.lse == 5.0).all())
    R.close(c.t["O"], c.reference(False)["O"], "O")


@pytest.mark.parametrize("layout", ["packed", "tokens", "gaps"])
@pytest.mark.parametrize("dims", [(3, 10, 5, 37, 300, 64), (2, 12, 3, 21, 150, 160), (1, 9, 3, 43, 700, 256), (3, 30, 2, 3, 260, 96), (5, 14, 2, 33, 90, 16), (1, 24, 1, 129, 40, 128)], ids=str)
def test_heads_that_share_keys_also_share_tiles(dims, layout):
    """Queries of a key head's heads in the same tiles, a tile over two and over many heads, key heads that no number of XCDs divides, ragged keys."""
    c = Call(*dims, klen=[dims[4] - 57 * b % dims[4] for b in range(dims[0])], layout=layout, seed=8, fill=float("nan"))
    c.fwd()
    c.bwd()
    c.check(what=f"{layout} ")


@pytest.mark.parametrize("batch", [64, 65])
@pytest.mark.parametrize("lens", ["mixed", "equal"])
def test_batches_that_are_ranked_and_larger_ones(batch, lens):
    """Up to 64 items are taken by their numbers of keys, equal ones among them; more in order."""
    klen = [(b * 37) % 150 - 3 for b in range(batch)] if lens == "mixed" else [90] * batch
    c = Call(batch, 2, 1, 19, 141, 32, klen=klen, seed=batch, fill=float("nan"))
    c.fwd()
    c.bwd()
    c.check(what=f"{lens} ")


def test_heads_too_far_apart_to_share_tiles():
    """Shared key heads whose query heads lie more than 31 bits apart: the workspace that is asked for, without layouts, serves this call too."""
    heads, sq, sk, dh, far = 64, 2, 128, 64, (1 << 23) + 8
    near = Call(1, heads, 1, sq, sk, dh, seed=12)
    near.fwd()
    near.bwd()
    size = far * (heads - 1) + sq * dh
    lay = us.HeadsLayout(size, far, dh)
    Q, O, G, dQ = (torch.empty(size, dtype=F, device=DEV) for _ in range(4))
    at = lambda t: t.as_strided((heads, sq, dh), (far, dh, 1))      # noqa: E731
    at(Q).copy_(near.Q[0]), at(G).copy_(near.G[0])
    K, V = near.t["K"], near.t["V"]
    dK, dV = torch.empty(sk * dh, dtype=F, device=DEV), torch.empty(sk * dh, dtype=F, device=DEV)
    lse = torch.empty(heads * sq, dtype=torch.float32, device=DEV)
    wsb = us.attention_cross_workspace_bytes(1, heads, 1, sq, sk, dh)
    ws = torch.empty(wsb, dtype=torch.uint8, device=DEV)
    us.attention_cross_fwd(ptr(Q), ptr(K), ptr(V), None, ptr(O), ptr(lse), 1, heads, 1, sq, sk, dh, 0.0, lay, None, lay, ptr(ws), wsb, stream())
    us.attention_cross_bwd(ptr(Q), ptr(K), ptr(V), None, ptr(O), ptr(lse), ptr(G), ptr(dQ), ptr(dK), ptr(dV), 1, heads, 1, sq, sk, dh, 0.0, 0.0, 0.0, lay, None, lay, ptr(ws), wsb, stream())
    want = near.reference(True)
    for name, got in (("O", at(O)[None]), ("dQ", at(dQ)[None]), ("dK", dK.view(1, 1, sk, dh)), ("dV", dV.view(1, 1, sk, dh))):
        R.close(got, want[name], name)


def test_a_bad_query_beside_other_heads_in_its_tile():
    c = Call(1, 8, 2, 20, 150, 64, seed=6)
    c.Q[0, 5, 13, 5] = float("nan")
    c.t["Q"].copy_(c.Q)
    c.fwd()
    c.bwd()
    bad = torch.zeros(1, 8, 20, dtype=torch.bool)
    bad[0, 5, 13] = True
    for name in ("O", "dQ"):
        got = c.t[name].float().cpu()
        assert bool(got[bad].isnan().all()) and bool(got[~bad].isfinite().all()), name
    for name in ("dK", "dV"):
        got = c.t[name].float().cpu()
        assert bool(got[0, 1].isnan().all()) and bool(got[0, 0].isfinite().all()), name


def test_items_that_share_keys():
    """A batch stride of zero: several sequences over one encoder's states."""
    batch, heads, sq, sk, dh = 3, 2, 21, 100, 64
    one = Call(1, heads, heads, sq, sk, dh, seed=2)
    Q = torch.randn(batch, heads, sq, dh, generator=torch.Generator().manual_seed(8)).half()
    q, o = Q.to(DEV), torch.empty(batch, heads, sq, dh, dtype=F, device=DEV)
    lay = us.HeadsLayout(0, sk * dh, dh)
    us.attention_cross_fwd(ptr(q), ptr(one.bufs["K"]), ptr(one.bufs["V"]), None, ptr(o), None, batch, heads, heads, sq, sk, dh, 0.0, None, lay, None, None, 0, stream())
    want = R.cross(Q, one.K.expand(batch, -1, -1, -1), one.V.expand(batch, -1, -1, -1), None)
    R.close(o, want["O"], "O")


def test_no_queries_and_no_keys():
    t = lambda *s: torch.full(s, 7.0, dtype=F, device=DEV)      # noqa: E731
    dK, dV, K = t(2, 2, 9, 32), t(2, 2, 9, 32), t(2, 2, 9, 32)
    us.attention_cross_bwd(None, ptr(K), ptr(K), None, None, None, None, None, ptr(dK), ptr(dV), 2, 4, 2, 0, 9, 32, stream=stream())
    assert bool((dK == 0).all()) and bool((dV == 0).all())
    O, Q, dQ, lse = t(2, 4, 5, 32), t(2, 4, 5, 32), t(2, 4, 5, 32), torch.zeros(8, 5, device=DEV)
    us.attention_cross_fwd(ptr(Q), None, None, None, ptr(O), ptr(lse), 2, 4, 2, 5, 0, 32, stream=stream())
    assert bool((O == 0).all()) and bool((lse == -math.inf).all())
    n = us.attention_cross_workspace_bytes(2, 4, 2, 5, 0, 32)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device=DEV)
    us.attention_cross_bwd(ptr(Q), None, None, None, ptr(O), ptr(lse), ptr(Q), ptr(dQ), None, None, 2, 4, 2, 5, 0, 32, workspace=ptr(ws), workspace_bytes=n, stream=stream())
    assert bool((dQ == 0).all())


@pytest.mark.parametrize("at,value", [("Q", float("nan")), ("K", float("nan")), ("V", float("nan")), ("Q", float("inf"))])
def test_what_is_not_finite_stays_in_its_row(at, value):
    """A NaN in one query (or in a key or value of one head) reaches that row (that head) and nothing else; infinite scores are NaN rows."""
    c = Call(2, 2, 2, 40, 70, 64, seed=6)
    getattr(c, at)[1, 1, 13, 5] = value
    c.t[at].copy_(getattr(c, at))
    c.fwd()
    got = c.t["O"].float().cpu()
    bad = torch.zeros(2, 2, 40, dtype=torch.bool)
    bad[1, 1] = True if at != "Q" else torch.arange(40) == 13
    if at == "V":
        assert bool(got[1, 1, :, 5].isnan().all()) and bool(got[1, 1, :, :5].isfinite().all())
    else:
        assert bool(got[bad].isnan().all())
    assert bool(got[~bad].isfinite().all())


@pytest.mark.parametrize("dims", [(2, 4, 2, 37, 83, 80), (1, 2, 1, 40, 3000, 64), (1, 1, 1, 1500, 40, 64), (2, 8, 1, 1, 3000, 128)], ids=str)
def test_the_same_bits_again_on_another_stream_and_in_a_graph(dims):
    c = Call(*dims, klen=[dims[4] - 5] * dims[0], seed=4)
    names = ("O", "dQ", "dK", "dV")
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    first = {n: c.bufs[n].clone() for n in names}

    def again(run):
        for n in names:
            c.bufs[n].fill_(7.0)
        c.ws.fill_(0x77)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        for n in names:
            assert torch.equal(first[n], c.bufs[n]), n

    def go(st=None):
        c.fwd(st=st)
        c.bwd(st=st)
    again(go)
    side = torch.cuda.Stream()
    again(lambda: go(side.cuda_stream))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        again(graph.replay)
        other = Call(*dims, seed=40)
        other.fwd()
        other.bwd()


def test_offsets_beyond_32_bits():
    """Rows 8 MB apart over 5 GB, and two batch items 6 GB apart."""
    batch, heads, sq, sk, dh = 2, 1, 20, 600, 32
    row = 1 << 22
    lay = us.HeadsLayout(3 * 2 ** 30, 0, row)
    K = torch.empty(lay.batch + row * (sk - 1) + 64, dtype=F, device=DEV)
    V = torch.empty_like(K)
    c = Call(batch, heads, heads, sq, sk, dh, seed=12)
    heads_view(K, batch, heads, sk, dh, lay).copy_(c.K)
    heads_view(V, batch, heads, sk, dh, lay).copy_(c.V)
    O = torch.empty(batch, heads, sq, dh, dtype=F, device=DEV)
    lse = torch.empty(batch * heads, sq, device=DEV)
    us.attention_cross_fwd(ptr(c.bufs["Q"]), ptr(K), ptr(V), None, ptr(O), ptr(lse), batch, heads, heads, sq, sk, dh, 0.0, None, lay, None, ptr(c.ws), c.wsb, stream())
    want = c.reference()
    R.close(O, want["O"], "O")
    dK, dV, dQ = torch.empty_like(K), torch.empty_like(K), torch.empty_like(O)
    us.attention_cross_bwd(ptr(c.bufs["Q"]), ptr(K), ptr(V), None, ptr(O), ptr(lse), ptr(c.bufs["dO"]), ptr(dQ), ptr(dK), ptr(dV), batch, heads, heads, sq, sk, dh, 0.0, 0.0,
                           0.0, None, lay, None, ptr(c.ws), c.wsb, stream())
    R.close(dQ, want["dQ"], "dQ")
    R.close(heads_view(dK, batch, heads, sk, dh, lay), want["dK"], "dK")
    R.close(heads_view(dV, batch, heads, sk, dh, lay), want["dV"], "dV")
    # one query takes the other kernel
    us.attention_cross_fwd(ptr(c.bufs["Q"]), ptr(K), ptr(V), None, ptr(O), None, batch, heads, heads, 1, sk, dh, 0.0, us.HeadsLayout(sq * dh, sq * dh, dh), lay,
                           us.HeadsLayout(sq * dh, sq * dh, dh), None, 0, stream())
    R.close(O[:, :, :1], tuple(x[:, :, :1] for x in want["O"]), "O of one query")


def test_equal_lengths_agree_with_the_unmasked_attention():
    """us_attention_fwd / _bwd of the same tensors: its rounded scores, probabilities and their gradients make it the less exact of the two: each rounding to
    FP16 is 2^-11 of a score of up to 6 (3e-3 of p), P, dP and dA 2^-11 each, which many keys average out; within 2 % of the RMS everywhere."""
    heads, s, d = 4, 128, 64
    c = Call(1, heads, heads, s, s, d, seed=21)
    c.fwd()
    c.bwd()
    new = lambda *sh: torch.empty(sh, dtype=F, device=DEV)      # noqa: E731
    A, P, O, dP, dA, dQ, dK, dV = new(heads, s, s), new(heads, s, s), new(heads, s, d), new(heads, s, s), new(heads, s, s), new(heads, s, d), new(heads, s, d), new(heads, s, d)
    q, k, v, g = (ptr(c.bufs[n]) for n in ("Q", "K", "V", "dO"))
    us.attention_fwd(q, k, v, ptr(A), ptr(P), ptr(O), heads, s, d, stream())
    us.attention_bwd(q, k, v, ptr(A), ptr(P), g, ptr(dP), ptr(dA), ptr(dQ), ptr(dK), ptr(dV), heads, s, d, stream())
    for a, n in ((O, "O"), (dQ, "dQ"), (dK, "dK"), (dV, "dV")):
        b = c.t[n][0].float()
        assert float((a.float() - b).abs().max()) < 0.02 * max(1.0, float(b.abs().max())), n
