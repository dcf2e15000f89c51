"""Argument checks of attention over another sequence's keys, of the paged cache and of its eviction: on the host, before anything is launched; and the
definitions that the GPU tests compare with, held to differences and to elementary cases."""
import math

import pytest
import torch

import attend_ref as R
import paper_2303_11257_amd as us

OK = 16          # an aligned address that no refused call touches
L = us.HeadsLayout
BIG = 1 << 40


def fwd(batch=2, heads=4, kv=2, sq=5, sk=7, dh=32, lq=None, lkv=None, lo=None, ws=None, wsb=0, **kw):
    a = dict(Q=OK, K=OK, V=OK, klen=OK, O=OK, lse=OK)
    a.update(kw)
    us.attention_cross_fwd(*a.values(), batch, heads, kv, sq, sk, dh, 0.0, lq, lkv, lo, ws, wsb)


def bwd(batch=2, heads=4, kv=2, sq=5, sk=7, dh=32, lq=None, lkv=None, lo=None, ws=OK, wsb=BIG, **kw):
    a = dict(Q=OK, K=OK, V=OK, klen=OK, O=OK, lse=OK, dO=OK, dQ=OK, dK=OK, dV=OK)
    a.update(kw)
    us.attention_cross_bwd(*a.values(), batch, heads, kv, sq, sk, dh, 0.0, 0.0, 0.0, lq, lkv, lo, ws, wsb)


def store(dt=us.F16, pages=4, page=16, ld=3, batch=2, kv=2, s=5, dh=32, layout=None, **kw):
    a = dict(K=OK, V=OK, kc=OK, vc=OK, table=OK, len=OK, count=OK)
    a.update(kw)
    us.cache_store(a["K"], a["V"], layout, a["kc"], a["vc"], dt, pages, page, a["table"], ld, a["len"], a["count"], batch, kv, s, dh)


def paged(dt=us.F16, pages=4, page=16, ld=3, batch=2, heads=4, kv=2, dh=32, max_len=40, ldq=128, ldo=128, ws=OK, wsb=BIG, **kw):
    a = dict(Q=OK, kc=OK, vc=OK, table=OK, len=OK, W=OK, O=OK)
    a.update(kw)
    us.attention_paged(a["Q"], ldq, a["kc"], a["vc"], dt, pages, page, a["table"], ld, a["len"], a["W"], a["O"], ldo, batch, heads, kv, dh, max_len, 0.0, ws, wsb)


def evict(dt=us.F16, pages=4, page=16, ld=3, ld_to=3, batch=2, kv=2, dh=32, max_len=40, keep=20, recent=4, **kw):
    a = dict(kc=OK, vc=OK, W=OK, table=OK, to=OK, len=OK, new=OK, kept=OK)
    a.update(kw)
    us.cache_evict(a["kc"], a["vc"], a["W"], dt, pages, page, a["table"], ld, a["to"], ld_to, a["len"], a["new"], a["kept"], batch, kv, dh, max_len, keep, recent)


NULL, SHAPE, ALIGN, DTYPE, WORKSPACE = 1, 2, 3, 4, 5
CASES = [(lambda n=n: fwd(**{n: None}), NULL) for n in ("Q", "K", "V", "O")]
CASES += [(lambda n=n: fwd(**{n: 24}), ALIGN) for n in ("Q", "K", "V", "O")] + [(lambda: fwd(klen=18), ALIGN), (lambda: fwd(lse=18), ALIGN), (lambda: fwd(ws=8), ALIGN)]
SHAPES = [dict(batch=-1), dict(batch=65536), dict(heads=0), dict(kv=0), dict(heads=4, kv=3), dict(heads=70000, kv=1), dict(sq=-1), dict(sk=-1), dict(dh=8), dict(dh=24),
          dict(dh=272), dict(dh=0), dict(sq=1 << 29), dict(sk=1 << 29), dict(batch=65535, heads=65535, kv=1)]
CASES += [(lambda k=k: f(**k), SHAPE) for k in SHAPES for f in (fwd, bwd)]
LAYOUTS = [L(-8, 32, 32), L(1000, 33, 32), L(1004, 64, 64), L(1000, 200, 24), L(1000, 200, 36), L(1000, 200, (1 << 22) + 8)]
CASES += [(lambda k=k, n=n: f(**{n: k}), SHAPE) for k in LAYOUTS for n in ("lq", "lkv", "lo") for f in (fwd, bwd)]
# what is written must not overlap: heads on one another, items on one another, rows interleaved into the next head
APART = [L(0, 160, 32), L(640, 0, 32), L(640, 64, 32), L(640, 32, 64), L(320, 32, 128)]
CASES += [(lambda k=k: fwd(lo=k), SHAPE) for k in APART] + [(lambda k=k: bwd(lq=k), SHAPE) for k in APART] + [(lambda: bwd(lkv=L(0, 224, 32)), SHAPE), (lambda: bwd(lkv=L(448, 0, 32)), SHAPE)]
CASES += [(lambda n=n: bwd(**{n: None}), NULL) for n in ("Q", "K", "V", "O", "lse", "dO", "dQ", "dK", "dV")]
CASES += [(lambda n=n: bwd(**{n: 24}), ALIGN) for n in ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV", "ws")] + [(lambda: bwd(klen=17), ALIGN), (lambda: bwd(lse=17), ALIGN)]
CASES += [(lambda: bwd(sk=200, ws=None), WORKSPACE), (lambda: bwd(sk=200, wsb=16), WORKSPACE), (lambda: fwd(batch=1, heads=1, kv=1, sq=100, sk=9000, ws=OK, wsb=64), WORKSPACE)]
CACHE = [dict(batch=-1), dict(batch=65536), dict(kv=0), dict(dh=8), dict(dh=40), dict(dh=272), dict(page=8), dict(page=24), dict(page=2048), dict(page=0), dict(pages=-1),
         dict(pages=1 << 31), dict(ld=-1)]
CASES += [(lambda k=k: f(**k), SHAPE) for k in CACHE for f in (store, paged, evict)]
CASES += [(lambda d=d: f(dt=d), DTYPE) for d in (us.F32, us.E5M2, 9) for f in (store, paged, evict)]
CASES += [(lambda: store(s=-1), SHAPE), (lambda: store(s=1 << 28), SHAPE), (lambda: store(layout=L(160, 160, 24)), SHAPE), (lambda: store(layout=L(160, 161, 32)), SHAPE), (lambda: paged(heads=3), SHAPE),
          (lambda: paged(heads=0), SHAPE), (lambda: paged(max_len=-1), SHAPE), (lambda: paged(max_len=1 << 31), SHAPE), (lambda: paged(ldq=120), SHAPE), (lambda: paged(ldq=132), SHAPE),
          (lambda: paged(ldo=64), SHAPE), (lambda: paged(ldo=129), SHAPE), (lambda: evict(keep=-1), SHAPE), (lambda: evict(recent=-1), SHAPE), (lambda: evict(recent=21), SHAPE),
          (lambda: evict(max_len=-1), SHAPE), (lambda: evict(keep=(1 << 20) + 1), SHAPE), (lambda: evict(ld_to=2), SHAPE), (lambda: evict(to=32, ld_to=-1), SHAPE)]
CASES += [(lambda n=n: store(**{n: None}), NULL) for n in ("K", "V", "kc", "vc", "table", "len")] + [(lambda n=n: store(**{n: 24}), ALIGN) for n in ("K", "V", "kc", "vc")]
CASES += [(lambda n=n: store(**{n: 18}), ALIGN) for n in ("table", "len", "count")]
CASES += [(lambda n=n: paged(**{n: None}), NULL) for n in ("Q", "kc", "vc", "table", "len", "O")] + [(lambda n=n: paged(**{n: 24}), ALIGN) for n in ("Q", "kc", "vc", "O", "ws")]
CASES += [(lambda n=n: paged(**{n: 18}), ALIGN) for n in ("table", "len", "W")] + [(lambda: paged(ws=None), WORKSPACE), (lambda: paged(wsb=15), WORKSPACE)]
CASES += [(lambda n=n: evict(**{n: None}), NULL) for n in ("kc", "vc", "W", "table", "to", "len", "kept")] + [(lambda n=n: evict(**{n: 24}), ALIGN) for n in ("kc", "vc")]
CASES += [(lambda n=n: evict(**{n: 18}), ALIGN) for n in ("W", "table", "to", "len", "new", "kept")]

# what one launch cannot hold: 2^22 tiles of rows, 2^23 pieces of 256 positions, 2^20 key heads to choose for
CASES += [(lambda k=k: f(batch=65535, kv=1, **k), SHAPE) for k in (dict(heads=65, sq=1), dict(heads=1, sq=8200), dict(heads=1, sq=1, sk=8200)) for f in (fwd, bwd)]
CASES += [(lambda: paged(batch=65535, heads=65, kv=1, ldq=65 * 32, ldo=65 * 32), SHAPE), (lambda: paged(batch=65535, heads=1, kv=1, max_len=33000), SHAPE), (lambda: evict(batch=65535, kv=17), SHAPE)]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_refused_before_anything_is_launched(i):
    call, status = CASES[i]
    with pytest.raises(us.UsError) as e:
        call()
    assert e.value.status == status


def test_nothing_to_do_is_no_error():
    us.attention_cross_fwd(None, None, None, None, None, None, 0, 4, 2, 5, 7, 32)
    us.attention_cross_fwd(None, None, None, None, None, None, 2, 4, 2, 0, 7, 32)
    us.attention_cross_bwd(None, None, None, None, None, None, None, None, None, None, 2, 4, 2, 0, 0, 32)
    store(batch=0), store(s=0), store(pages=0, kc=None, vc=None), store(ld=0)
    paged(batch=0)
    evict(batch=0)


def test_sizes():
    assert us.attention_cross_workspace_bytes(0, 4, 2, 5, 7, 32) == 0 and us.attention_cross_workspace_bytes(2, 4, 3, 5, 7, 32) == 0
    assert us.attention_cross_workspace_bytes(2, 4, 2, 5, 200, 32) >= 2 * 4 * 64 * 8
    assert us.attention_paged_workspace_bytes(0, 4, 2, 32, 100, True) == 0 and us.attention_paged_workspace_bytes(2, 4, 3, 32, 100, True) == 0
    assert us.attention_paged_workspace_bytes(2, 4, 2, 32, 100, True) >= 2 * 4 * 100 * 4
    assert us.attention_cross_workspace_bytes(2, 4, 2, 0, 7, 32) == us.attention_cross_workspace_bytes(2, 4, 2, 0, 0, 32) == 0
    assert us.attention_cross_workspace_bytes(2, 4, 2, 5, 0, 32) >= 2 * 4 * 32 * 8 and us.attention_paged_workspace_bytes(2, 4, 2, 32, 0, False) == 0
    assert us.HeadsLayout(1, 2, 3).row == 3


@pytest.mark.parametrize("n,alpha", [(6, 0.0), (3, 0.7), (1, 0.0), (2, 0.0)])
def test_definition_against_differences(n, alpha):
    """The gradients of sum(G O) in 64 bits: central differences of step h are h^2 / 6 of a third derivative off, which stays below 1e3 here, and 2^-52 |sum| / h."""
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)      # noqa: E731
    x = dict(Q=r(1, 4, 3, 16), K=r(1, 2, 6, 16), V=r(1, 2, 6, 16))
    G = r(1, 4, 3, 16)
    f = lambda: float((R.cross(x["Q"], x["K"], x["V"], [n], alpha)["O"][0] * G).sum())      # noqa: E731
    got = R.cross(x["Q"], x["K"], x["V"], [n], alpha, G, 1.0, 1.0)
    h = 1e-4
    for name, t in x.items():
        flat, grad = t.view(-1), got["d" + name][0].reshape(-1)
        for i in range(0, flat.numel(), 7):
            keep = float(flat[i])
            flat[i] = keep + h
            up = f()
            flat[i] = keep - h
            down = f()
            flat[i] = keep
            assert abs((up - down) / (2 * h) - float(grad[i])) < 2e-5, (name, i)


def test_definition_has_unit_variance():
    """The default factors: outputs and gradients of independent unit normal inputs have a variance near one (64 keys of 64 columns: the softmax is not
    quite even, its sum of squares e rather than 1 over n, so up to e^1/2 in O and more in the gradients)."""
    g = torch.Generator().manual_seed(4)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)      # noqa: E731
    Q, K, V, G = r(1, 8, 32, 64), r(1, 2, 64, 64), r(1, 2, 64, 64), r(1, 8, 32, 64)
    out = R.cross(Q, K, V, None, 0.0, G)
    for name in ("O", "dQ", "dK", "dV"):
        rms = float(out[name][0].square().mean().sqrt())
        assert 0.8 < rms < 2.2, (name, rms)


def test_definition_of_eviction():
    W = torch.tensor([[[3.0, 1, 9, 1, 0, 5, 5, math.nan]]])                # one page of 8
    table = torch.tensor([[0]])
    assert R.evict(W, table, [8], 8, 100, 3, 1)[0][0] == [2, 5, 7]         # 9, the first 5, the last one
    assert R.evict(W, table, [8], 8, 100, 3, 0)[0][0] == [2, 5, 7]         # NaN above all, 9, the first 5
    assert R.evict(W, table, [5], 8, 100, 3, 2)[0][0] == [2, 3, 4]
    assert R.evict(W, table, [3], 8, 100, 3, 2)[0][0] == [0, 1, 2] and R.evict(W, table, [-2], 8, 100, 3, 2)[0][0] == []
    assert R.evict(W, torch.tensor([[5]]), [8], 8, 100, 3, 1)[0][0] == [0, 1, 7]       # a page that there is not
