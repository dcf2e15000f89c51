"""The paged cache: storing into it, attention of one token over it, eviction from it, against the definitions of tests/attend_ref.py; and a generation that uses them
together with the norms, the rotation and attention over an encoder's states."""
import math

import pytest
import torch

import attend_ref as R
import paper_2303_11257_amd as us
from gpu_util import DEV, ptr, stream

pytestmark = pytest.mark.gpu
F, F8 = torch.float16, torch.float8_e4m3fn


def tables(lens, page, g, spare=3, wide=0):
    each = [max(0, -(-n // page)) for n in lens]
    wide = max(wide, max(each), 1)
    pages = sum(each) + spare
    ids = torch.randperm(pages, generator=g).int()
    t = torch.full((len(lens), wide), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(each):
        t[b, :n] = ids[at: at + n]
        at += n
    return t, pages


def pool(pages, kv, page, dh, fp8, g):
    x = torch.randn(pages, kv, page, dh, generator=g).half()
    return x.float().to(F8) if fp8 else x


def dt(fp8):
    return us.E4M3 if fp8 else us.F16


def bits(x):
    return x.view(torch.uint8) if x.dtype == F8 else x


def rows(x, table, b, head, n, page):
    """The n rows of a sequence's key head (zeros on pages that there are not), and which there are."""
    out, there = torch.zeros(n, x.shape[-1], dtype=torch.float64), torch.zeros(n, dtype=torch.bool)
    for i in range(0, n, page):
        at = R.position(table, b, i, page, x.shape[0])
        m = min(page, n - i)
        if at:
            out[i: i + m], there[i: i + m] = x[at[0], head, :m].double(), True
    return out, there


# ---- store -------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("batch,kv,s,dh,page,rep,layout", [(3, 2, 1, 64, 16, 1, "packed"), (2, 3, 45, 80, 32, 1, "packed"), (4, 1, 100, 16, 16, 4, "heads"), (2, 4, 33, 128, 64, 2, "fused"),
                                                          (1, 2, 7, 256, 1024, 1, "fused"), (5, 2, 130, 48, 128, 3, "heads")])
def test_store(batch, kv, s, dh, page, rep, layout, fp8):
    g = torch.Generator().manual_seed(batch * s)
    count = [s if b == 0 else max(0, s - 13 * b) for b in range(batch)]
    before = [0 if b == 0 else 5 * b + page // 2 for b in range(batch)]
    lens = [c + n for c, n in zip(count, before)]
    table, pages = tables(lens, page, g)
    old = {n: pool(pages, kv, page, dh, fp8, g) for n in "KV"}
    if layout == "packed":
        new, lay = torch.randn(2, batch, kv, s, dh, generator=g).half(), None
        x = {n: new[i] for i, n in enumerate("KV")}
        at = (0, new[0].numel())
    elif layout == "heads":
        new, lay = torch.randn(2, batch, kv * rep, s, dh, generator=g).half(), us.HeadsLayout(kv * rep * s * dh, rep * s * dh, dh)
        x = {n: new[i, :, ::rep] for i, n in enumerate("KV")}
        at = (0, new[0].numel())
    else:
        new = torch.randn(batch, s, (rep + 2) * kv, dh, generator=g).half()
        lay = us.HeadsLayout(s * (rep + 2) * kv * dh, dh, (rep + 2) * kv * dh)
        x = {n: new[:, :, kv * (rep + i): kv * (rep + i + 1)].transpose(1, 2) for i, n in enumerate("KV")}
        at = (kv * rep * dh, kv * (rep + 1) * dh)
    new.view(-1)[3], new.view(-1)[at[1] + 2] = 700.0, float("nan")          # clipped in E4M3; NaN's code
    dev = {n: v.to(DEV) for n, v in old.items()}
    nd, td, ld, cd = new.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), torch.tensor(count, dtype=torch.int32, device=DEV)
    us.cache_store(ptr(nd) + 2 * at[0], ptr(nd) + 2 * at[1], lay, ptr(dev["K"]), ptr(dev["V"]), dt(fp8), pages, page, ptr(td), table.shape[1], ptr(ld), ptr(cd), batch, kv, s, dh,
                   stream())
    for n in "KV":
        want = bits(old[n].clone())
        for b in range(batch):
            for t in range(count[b]):
                p, slot = R.position(table, b, before[b] + t, page, pages)
                row = x[n][b, :, t]
                if fp8:
                    row = row.float().clamp(-448, 448).to(F8).view(torch.uint8)
                want[p, :, slot] = row
        got = bits(dev[n].cpu())
        if fp8:       # either NaN code
            want, got = (torch.where((v & 0x7F) == 0x7F, 0x7F, v) for v in (want, got))
            assert torch.equal(got, want), n
        else:
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)), n


def test_store_leaves_out_what_has_no_place():
    """Pages outside the pool, positions before the first and behind the table: nothing is written for them, everything else is."""
    g = torch.Generator().manual_seed(1)
    batch, kv, s, dh, page, pages = 4, 2, 40, 32, 16, 6
    table = torch.tensor([[0, -1, 1], [2, 6, 3], [4, 5, -7], [2 ** 31 - 1, 0, 0]], dtype=torch.int32)
    lens = [48, 40, 60, 20]          # the third's last positions have no column in the table, the fourth's first would be before the first
    K = torch.randn(batch, kv, s, dh, generator=g).half()
    kc, vc = torch.full((pages + 2, kv, page, dh), 7.0, dtype=F, device=DEV), torch.full((pages + 2, kv, page, dh), 7.0, dtype=F, device=DEV)
    kd, td, ld = K.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    inner = lambda x: ptr(x) + 2 * kv * page * dh          # noqa: E731          (a guard page on either side)
    us.cache_store(ptr(kd), ptr(kd), None, inner(kc), inner(vc), us.F16, pages, page, ptr(td), 3, ptr(ld), None, batch, kv, s, dh, stream())
    want = torch.full((pages, kv, page, dh), 7.0, dtype=F)
    for b in range(3):
        for t in range(s):
            at = R.position(table, b, lens[b] - s + t, page, pages)
            if at:
                want[at[0], :, at[1]] = K[b, :, t]
    # (the fourth sequence stores its positions 0 .. 19: on a page that there is not, then on page 0, whose slots 0 .. 3 it shares with the first here)
    got, gv = kc.cpu(), vc.cpu()
    mine = torch.ones_like(want, dtype=torch.bool)
    mine[0, :, :4] = False
    assert torch.equal(got[1:-1][mine], want[mine]) and torch.equal(gv[1:-1][mine], want[mine])
    for x in (got, gv):
        assert bool((x[0] == 7.0).all()) and bool((x[-1] == 7.0).all())


# ---- attention ---------------------------------------------------------------------------------------------------------------

class Paged:
    def __init__(self, lens, heads, kv, dh, page, fp8, weights=True, seed=0, sigma=1.5, wide=0, max_len=None, ldq=0, alpha=0.0, break_pages=()):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.alpha = lens, page, alpha
        self.B, self.h, self.kv, self.dh, self.fp8 = len(lens), heads, kv, dh, fp8
        self.table, pages = tables(lens, page, g, wide=wide)
        for b, i, v in break_pages:
            self.table[b, i] = v
        self.K, self.V = pool(pages, kv, page, dh, fp8, g), pool(pages, kv, page, dh, fp8, g)
        self.W = torch.rand(pages, kv, page, generator=g)
        self.ldq = ldq or heads * dh
        self.Q = (torch.randn(self.B, self.ldq, generator=g) * sigma).half()
        self.max_len = max(max(lens), 0) if max_len is None else max_len
        self.dev = {n: getattr(self, n).to(DEV) for n in ("table", "K", "V", "W", "Q")}
        self.len = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.O = torch.full((self.B, self.ldq), 7.0, dtype=F, device=DEV)
        self.weights = weights
        self.wsb = us.attention_paged_workspace_bytes(self.B, heads, kv, dh, self.max_len, weights)
        self.ws = torch.full((max(16, self.wsb) + 64,), 0xEE, dtype=torch.uint8, device=DEV)

    def run(self, st=None):
        d, K = self.dev, self.K
        us.attention_paged(ptr(d["Q"]), self.ldq, ptr(d["K"]), ptr(d["V"]), dt(self.fp8), K.shape[0], self.page, ptr(d["table"]), self.table.shape[1], ptr(self.len),
                           ptr(d["W"]) if self.weights else None, ptr(self.O), self.ldq, self.B, self.h, self.kv, self.dh, self.max_len, self.alpha, ptr(self.ws), self.wsb,
                           stream() if st is None else st)

    def check(self, what=""):
        rep, dh, page = self.h // self.kv, self.dh, self.page
        O, eO = (torch.zeros(self.B, self.h, dh, dtype=torch.float64) for _ in range(2))
        W, eW = self.W.double(), torch.zeros(self.W.shape, dtype=torch.float64)
        for b, n in enumerate(self.lens):
            n = max(0, min(n, self.max_len, self.table.shape[1] * page))
            a = self.alpha if self.alpha > 0 else math.sqrt(max(n, 1))
            for k in range(self.kv):
                (kr, there), (vr, _) = rows(self.K, self.table, b, k, n, page), rows(self.V, self.table, b, k, n, page)
                m = int(there.sum())
                q = self.Q[b, k * rep * dh: (k + 1) * rep * dh].view(rep, dh).double()
                o, e, p, _, ep = R.rows_forward(q, kr[there], vr[there], m, a)
                O[b, k * rep: (k + 1) * rep], eO[b, k * rep: (k + 1) * rep] = o, e
                if m:
                    for j, i in enumerate(there.nonzero().view(-1).tolist()):
                        at = R.position(self.table, b, i, page, self.K.shape[0])
                        W[at[0], k, at[1]] += p[:, j].sum()
                        eW[at[0], k, at[1]] += ((ep[:, 0] + (rep + 8) * R.V) * p[:, j]).sum() + 2.0 ** -126
        got = self.O.cpu()
        R.close(got[:, : self.h * dh].reshape(self.B, self.h, dh), (O, eO), what + "O")
        assert bool((got[:, self.h * dh:] == 7.0).all())
        if self.weights:
            R.close(self.dev["W"], (W, torch.where(eW > 0, eW + R.V * W.abs(), eW)), what + "weights")
        else:
            assert torch.equal(self.dev["W"].cpu(), self.W)
        assert bool((self.ws[max(16, self.wsb):] == 0xEE).all())
        for n in ("K", "V"):
            assert torch.equal(bits(self.dev[n]).cpu(), bits(getattr(self, n)))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,heads,kv,dh,page", [([1], 1, 1, 16, 16), ([0, 1, 2, 17], 4, 2, 32, 16), ([100, 33, 128, 129], 8, 2, 64, 32), ([31, 500, 1000], 4, 4, 80, 64), ([700, 0, 65], 6, 1, 96, 16),
                                                 ([300, 301], 16, 1, 128, 256), ([260, 7], 20, 1, 64, 128), ([140, 200], 40, 2, 32, 16), ([129, 77], 2, 1, 160, 1024), ([513, 40], 4, 2, 192, 32),
                                                 ([257, 90, 1], 8, 1, 256, 16), ([3000], 2, 2, 112, 64), ([-3, 40], 2, 1, 48, 16), ([9000, 64], 8, 1, 128, 128)], ids=str)
def test_attention(lens, heads, kv, dh, page, fp8):
    for weights in (True, False):
        c = Paged(lens, heads, kv, dh, page, fp8, weights, seed=len(lens) * dh)
        c.run()
        c.check(f"{lens} ")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("batch", [64, 70])
def test_attention_of_many_sequences(batch, fp8):
    """Up to 64 sequences are taken by their lengths, equal ones among them; more in order."""
    c = Paged([(b * 29) % 90 - 1 for b in range(batch)], 4, 2, 32, 16, fp8, True, seed=batch)
    c.run()
    c.check()


@pytest.mark.parametrize("fp8", [False, True])
def test_attention_rows_apart_factor_and_bounds(fp8):
    Paged([50, 60], 4, 2, 64, 16, fp8, ldq=4 * 64 + 40, alpha=0.75).run()
    c = Paged([50, 60], 4, 2, 64, 16, fp8, ldq=4 * 64 + 40, alpha=0.75, wide=9)
    c.run()
    c.check()
    c = Paged([50, 400, 10], 4, 2, 64, 16, fp8, max_len=200)            # the second is cut off at max_len
    c.run()
    c.check()
    c = Paged([50, 400, 10], 4, 2, 64, 16, fp8, max_len=5000)           # far fewer than there might be
    c.run()
    c.check()
    c = Paged([48, 32], 4, 2, 64, 16, fp8)                              # longer than the table
    c.lens = [1000, 32]
    c.len.copy_(torch.tensor(c.lens))
    c.table, c.max_len = c.table.clone(), 48
    c.run()
    c.check()


@pytest.mark.parametrize("fp8", [False, True])
def test_pages_that_there_are_not(fp8):
    """Entries outside the pool: no attention goes there; a sequence with no page at all has a result of zeros."""
    c = Paged([100, 64, 40, 33], 4, 2, 64, 16, fp8, break_pages=[(0, 2, -1), (0, 6, 10 ** 6), (1, 0, 2 ** 31 - 1), (2, 0, -5), (2, 1, -5), (2, 2, 999), (3, 2, -1)])
    c.run()
    c.check()
    assert bool((c.O[2, : 4 * 64] == 0).all())


def test_what_lies_behind_a_sequence_is_not_seen():
    """NaN and infinities in the slots behind the last position and on the spare pages."""
    c = Paged([5, 37, 128], 4, 2, 64, 32, False, seed=5)
    used = torch.zeros(c.K.shape[0], c.page, dtype=torch.bool)
    for b, n in enumerate(c.lens):
        for i in range(n):
            p, s = R.position(c.table, b, i, c.page, c.K.shape[0])
            used[p, s] = True
    for name, v in (("K", float("nan")), ("V", float("inf"))):
        x = getattr(c, name)
        x.copy_(torch.where(used[:, None, :, None], x, torch.tensor(v, dtype=F)))
        c.dev[name].copy_(x)
    c.run()
    got = c.O.clone()
    assert bool(got.isfinite().all())
    for name in "KV":                                                     # (the reference multiplies everything)
        x = getattr(c, name)
        x.copy_(torch.where(used[:, None, :, None], x, torch.tensor(0.0, dtype=F)))
        c.dev[name].copy_(x)
    c.check()


@pytest.mark.parametrize("sigma", [0.0, 40.0])
def test_even_and_peaked_rows(sigma):
    c = Paged([300, 1, 77], 8, 2, 64, 16, False, sigma=sigma, seed=8)
    c.run()
    c.check()


@pytest.mark.parametrize("fp8,weights", [(False, True), (True, False)])
def test_the_same_bits_again_on_another_stream_and_in_a_graph(fp8, weights):
    """A graph's replays take the lengths that are there then."""
    c = Paged([900, 33, 2000], 8, 2, 64, 32, fp8, weights, seed=3)
    lens = c.lens

    def once(run, what):
        c.dev["W"].copy_(c.W.to(DEV)), c.O.fill_(7.0), c.ws.fill_(0xEE)
        torch.cuda.synchronize()
        run()
        torch.cuda.synchronize()
        return c.O.clone(), c.dev["W"].clone()
    first = once(c.run, "eager")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        for run in (c.run, lambda: c.run(side.cuda_stream), graph.replay):
            got = once(run, "again")
            assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1])
    c.len.copy_(torch.tensor([17, 2000, 0]).clamp_max(torch.tensor([900, 33, 2000])))
    c.lens = [17, 33, 0]
    once(graph.replay, "shorter")
    c.check("shorter ")
    assert lens == [900, 33, 2000]


def test_offsets_beyond_32_bits():
    """A pool of 6 GB whose used pages lie at its end; table entries, rows and weights far behind."""
    kv, page, dh, pages = 8, 128, 128, 23000
    g = torch.Generator().manual_seed(2)
    K, V = (torch.zeros(pages, kv, page, dh, dtype=F, device=DEV) for _ in range(2))
    W = torch.zeros(pages, kv, page, device=DEV)
    table = torch.tensor([[pages - 1, pages - 3, 0], [pages - 2, 1, pages - 7]], dtype=torch.int32)
    lens = [300, 290]
    new = torch.randn(2, 2, kv, 300, dh, generator=g).half()
    nd, td, ld = new.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    cd = torch.tensor(lens, dtype=torch.int32, device=DEV)
    us.cache_store(ptr(nd), ptr(nd[1]), None, ptr(K), ptr(V), us.F16, pages, page, ptr(td), 3, ptr(ld), ptr(cd), 2, kv, 300, dh, stream())
    Q = torch.randn(2, kv * dh, generator=g).half()
    qd, O = Q.to(DEV), torch.empty(2, kv * dh, dtype=F, device=DEV)
    wsb = us.attention_paged_workspace_bytes(2, kv, kv, dh, 300, True)
    ws = torch.empty(wsb, dtype=torch.uint8, device=DEV)
    us.attention_paged(ptr(qd), kv * dh, ptr(K), ptr(V), us.F16, pages, page, ptr(td), 3, ptr(ld), ptr(W), ptr(O), kv * dh, 2, kv, kv, dh, 300, 0.0, ptr(ws), wsb, stream())
    for b in range(2):
        for h in range(kv):
            o, e, p, _, ep = R.rows_forward(Q[b, h * dh: (h + 1) * dh].view(1, dh).double(), new[0, b, h, : lens[b]].double(), new[1, b, h, : lens[b]].double(), lens[b], 0.0)
            R.close(O[b, h * dh: (h + 1) * dh].view(1, dh), (o, e), "O")
            w = torch.cat([W[int(x), h] for x in table[b]])[: lens[b]]
            R.close(w.view(1, -1), (p, (ep + 16 * R.V) * p + 2.0 ** -126), "weights")
    # one sequence of those pages, evicted there
    kept, new_len = torch.empty(2, kv, 100, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV)
    before, w = K.clone(), W.cpu()
    us.cache_evict(ptr(K), ptr(V), ptr(W), us.F16, pages, page, ptr(td), 3, ptr(td), 3, ptr(ld), ptr(new_len), ptr(kept), 2, kv, dh, 300, 100, 10, stream())
    want = R.evict(w, table, lens, page, 300, 100, 10)
    assert kept.cpu().tolist() == want and new_len.tolist() == [100, 100]
    for b in range(2):
        for h in (0, kv - 1):
            src = torch.stack([before[R.position(table, b, i, page, pages)[0], h, i % page] for i in want[b][h]])
            assert torch.equal(K[int(table[b, 0]), h, :100], src)


# ---- eviction ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,kv,dh,page,keep,recent,ties", [([40], 1, 16, 16, 20, 0, False), ([100, 20, 0, 1, 21], 2, 64, 16, 20, 5, False), ([300, 299, 64], 3, 80, 32, 64, 64, False),
                                                            ([500, 33], 1, 128, 64, 100, 1, True), ([3000, 1025], 2, 32, 128, 1024, 100, True), ([70, 65], 2, 256, 16, 64, 0, True),
                                                            ([2500, 40], 1, 96, 16, 2400, 300, False), ([50, 9], 2, 48, 16, 1, 0, False), ([30, 9], 2, 48, 16, 1, 1, True)], ids=str)
def test_evict(lens, kv, dh, page, keep, recent, ties, fp8, in_place):
    g = torch.Generator().manual_seed(len(lens) + keep)
    n = len(lens)
    into = [] if in_place else [min(x, keep) for x in lens]
    both, pages = tables(lens + into, page, g)
    table, to = both[:n].contiguous(), (both[:n] if in_place else both[n:]).contiguous()
    K, V = pool(pages, kv, page, dh, fp8, g), pool(pages, kv, page, dh, fp8, g)
    W = torch.rand(pages, kv, page, generator=g) * 3 - 1
    if ties:
        W = (W * 4).round() / 4                          # few different values, zeros of both signs among them
        W.view(-1)[::7] *= -1.0
        W.view(-1)[5::50] = float("nan")
        W.view(-1)[6::70] = -math.inf
        W.view(-1)[8::90] = math.inf
    dev = {m: x.to(DEV) for m, x in (("K", K), ("V", V), ("W", W), ("table", table))}
    td = dev["table"] if in_place else to.to(DEV)
    ld = torch.tensor(lens, dtype=torch.int32, device=DEV)
    new, kept = torch.full((n,), -9, dtype=torch.int32, device=DEV), torch.full((n, kv, keep), -9, dtype=torch.int32, device=DEV)
    us.cache_evict(ptr(dev["K"]), ptr(dev["V"]), ptr(dev["W"]), dt(fp8), pages, page, ptr(dev["table"]), table.shape[1], ptr(td), to.shape[1], ptr(ld), ptr(new), ptr(kept), n, kv,
                   dh, max(lens), keep, recent, stream())
    want = R.evict(W, table, lens, page, max(lens), keep, recent)
    assert kept.cpu().tolist() == [[h + [-1] * (keep - len(h)) for h in s] for s in want]
    assert new.tolist() == [min(x, keep) for x in lens]
    for name, x in (("K", bits(K)), ("V", bits(V)), ("W", W)):
        y = x.clone()
        for b in range(n):
            for h in range(kv):
                for i, j in enumerate(want[b][h]):
                    p, s = R.position(to, b, i, page, pages)
                    q, t = R.position(table, b, j, page, pages)
                    y[p, h, s] = x[q, h, t]
        got = bits(dev[name]).cpu()
        assert torch.equal(got.view(torch.int32) if name == "W" else got, y.view(torch.int32) if name == "W" else y), name


def test_evict_cuts_off_and_leaves_out():
    """len itself as new_len; sequences beyond max_len; pages that there are not rank below everything and are neither read nor written; nothing kept at all."""
    g = torch.Generator().manual_seed(7)
    kv, dh, page = 2, 32, 16
    table, pages = tables([200, 200, 90], page, g)
    table[1, 3], table[1, 0], table[2, 5] = -1, pages, 2 ** 31 - 1
    K, V, W = pool(pages, kv, page, dh, False, g), pool(pages, kv, page, dh, False, g), torch.rand(pages, kv, page, generator=g) - 0.5
    dev = {m: x.to(DEV) for m, x in (("K", K), ("V", V), ("W", W), ("table", table))}
    ld, kept = torch.tensor([200, 200, 90], dtype=torch.int32, device=DEV), torch.empty(3, kv, 60, dtype=torch.int32, device=DEV)
    go = lambda keep, recent: us.cache_evict(ptr(dev["K"]), ptr(dev["V"]), ptr(dev["W"]), us.F16, pages, page, ptr(dev["table"]), table.shape[1], ptr(dev["table"]),      # noqa: E731
                                             table.shape[1], ptr(ld), ptr(ld), ptr(kept), 3, kv, dh, 150, keep, recent, stream())
    go(60, 12)
    want = R.evict(W, table, [200, 200, 90], page, 150, 60, 12)
    assert kept.cpu().tolist() == want and ld.tolist() == [60, 60, 60]
    y = K.clone()
    for b in range(3):
        for h in range(kv):
            for i, j in enumerate(want[b][h]):
                to, at = R.position(table, b, i, page, pages), R.position(table, b, j, page, pages)
                if to and at:
                    y[to[0], h, to[1]] = K[at[0], h, at[1]]
    assert torch.equal(dev["K"].cpu(), y)
    go(0, 0)
    assert ld.tolist() == [0, 0, 0]
    assert torch.equal(dev["K"].cpu(), y)


def test_evict_in_a_graph():
    g = torch.Generator().manual_seed(17)
    kv, dh, page, lens = 2, 64, 32, [700, 300]
    table, pages = tables(lens, page, g)
    K, V, W = (x.to(DEV) for x in (pool(pages, kv, page, dh, False, g), pool(pages, kv, page, dh, False, g), torch.rand(pages, kv, page, generator=g)))
    td, ld, new, kept = table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), torch.empty(2, dtype=torch.int32, device=DEV), torch.empty(2, kv, 256, dtype=torch.int32, device=DEV)
    work = [x.clone() for x in (K, V, W)]

    def go():
        for x, y in zip(work, (K, V, W)):
            x.copy_(y)
        us.cache_evict(*(ptr(x) for x in work), us.F16, pages, page, ptr(td), table.shape[1], ptr(td), table.shape[1], ptr(ld), ptr(new), ptr(kept), 2, kv, dh, 700, 256, 32,
                       torch.cuda.current_stream().cuda_stream)
    go()
    torch.cuda.synchronize()
    first = [x.clone() for x in (*work, new, kept)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for _ in range(3):
        for x in (*work, new, kept):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(first, (*work, new, kept)))


# ---- together ------------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True])
def test_generation(fp8):
    """Tokens of a decoder layer, one by one: norms and rotation -> the cache -> attention over it with its weights -> eviction when a sequence outgrows its budget, and
    attention over an encoder's states.  The same in 64 bits, from the heads that the library's norms and rotation leave and the positions that it keeps (their
    choice hangs on sums of nearly equal weights; each choice is checked against the accumulated weights, within their error)."""
    batch, h, kv, dh, page, steps, prompt, keep, recent, sk = 2, 4, 2, 32, 16, 30, 25, 40, 8, 50
    rep, cols, wide = h // kv, (h + 2 * kv) * dh, 8
    g = torch.Generator().manual_seed(23)
    pages = batch * wide + 1
    table = torch.randperm(pages, generator=g)[: batch * wide].int().view(batch, wide).contiguous()
    freq = (10000.0 ** (-torch.arange(dh // 2, dtype=torch.float64) / (dh // 2))).to(DEV)
    E = torch.randn(batch, sk, 2, kv, dh, generator=g).half()
    klen = [50, 31]
    new = lambda *s, d=F: torch.zeros(s, dtype=d, device=DEV)      # noqa: E731
    kc, vc, W = new(pages, kv, page, dh, d=F8 if fp8 else F), new(pages, kv, page, dh, d=F8 if fp8 else F), new(pages, kv, page, d=torch.float32)
    td, ed, kl = table.to(DEV), E.to(DEV), torch.tensor(klen, dtype=torch.int32, device=DEV)
    length = torch.zeros(batch, dtype=torch.int32, device=DEV)
    st, d8 = stream(), dt(fp8)
    keys = [[[] for _ in range(kv)] for _ in range(batch)]          # the reference's cache: rows by position
    values = [[[] for _ in range(kv)] for _ in range(batch)]
    weight = [[torch.zeros(0, dtype=torch.float64) for _ in range(kv)] for _ in range(batch)]
    kept = new(batch, kv, keep, d=torch.int32)
    most = keep + max(steps, prompt)
    wsb = max(us.attention_paged_workspace_bytes(batch, h, kv, dh, most, True), us.attention_cross_workspace_bytes(batch, h, kv, 1, sk, dh), 16)
    ws = new(wsb, d=torch.uint8)
    evictions = 0
    for step in range(1 + steps):
        s = prompt if step == 0 else 1
        first = 0 if step == 0 else prompt + step - 1
        qkv = torch.randn(batch * s, cols, generator=g).half().to(DEV)
        pos = torch.arange(first, first + s, dtype=torch.int32).repeat(batch).to(DEV)
        Q, K, V = (new(batch * h, s, dh) for _ in range(3))
        us.qk_norm_rope_fwd(ptr(qkv), cols, None, None, ptr(pos), ptr(freq), ptr(Q), ptr(K), ptr(V), batch, s, h, kv, dh, dh, us.ROPE_HALVES, 1e-6, st)
        length += s
        us.cache_store(ptr(K), ptr(V), us.HeadsLayout(h * s * dh, rep * s * dh, dh), ptr(kc), ptr(vc), d8, pages, page, ptr(td), wide, ptr(length), None, batch, kv, s, dh, st)
        for b in range(batch):
            for k in range(kv):
                for src, dst in ((K, keys), (V, values)):
                    x = src.view(batch, h, s, dh)[b, k * rep].cpu()
                    dst[b][k] += list((x.float().clamp(-448, 448).to(F8) if fp8 else x).double())
                weight[b][k] = torch.cat([weight[b][k], torch.zeros(s, dtype=torch.float64)])
        if step == 0:
            continue
        O, X = new(batch, h * dh), new(batch, h * dh)
        us.attention_paged(ptr(Q), h * dh, ptr(kc), ptr(vc), d8, pages, page, ptr(td), wide, ptr(length), ptr(W), ptr(O), h * dh, batch, h, kv, dh, most, 0.0, ptr(ws), wsb, st)
        lay = us.HeadsLayout(sk * 2 * kv * dh, dh, 2 * kv * dh)
        us.attention_cross_fwd(ptr(Q), ptr(ed), ptr(ed) + 2 * kv * dh, ptr(kl), ptr(X), None, batch, h, kv, 1, sk, dh, 0.0, None, lay, None, ptr(ws), wsb, st)
        q = Q.view(batch, h, dh).cpu().double()
        enc = R.cross(Q.view(batch, h, 1, dh).cpu(), E[:, :, 0].transpose(1, 2), E[:, :, 1].transpose(1, 2), klen)
        R.close(X.view(batch, h, 1, dh), enc["O"], f"step {step}: encoder")
        for b in range(batch):
            for k in range(kv):
                kk, vv = torch.stack(keys[b][k]), torch.stack(values[b][k])
                o, e, p, _, _ = R.rows_forward(q[b, k * rep: (k + 1) * rep], kk, vv, len(kk), 0.0)
                R.close(O[b].view(h, dh)[k * rep: (k + 1) * rep], (o, e), f"step {step}: cache")
                weight[b][k] += p.sum(0)
        n = len(keys[0][0])
        if n > keep and step % 5 == 0:
            us.cache_evict(ptr(kc), ptr(vc), ptr(W), d8, pages, page, ptr(td), wide, ptr(td), wide, ptr(length), ptr(length), ptr(kept), batch, kv, dh, most, keep, recent, st)
            evictions += 1
            for b in range(batch):
                for k in range(kv):
                    chosen = kept[b, k].cpu().tolist()
                    assert chosen == sorted(set(chosen)) and chosen[-recent:] == list(range(n - recent, n))
                    rest = [i for i in range(n - recent) if i not in set(chosen)]
                    # sums of up to 30 FP32 additions of weights below 2, each within 1e-5
                    assert float(weight[b][k][chosen[: keep - recent]].min()) >= float(weight[b][k][rest].max()) - 1e-3
                    keys[b][k], values[b][k], weight[b][k] = [keys[b][k][i] for i in chosen], [values[b][k][i] for i in chosen], weight[b][k][chosen]
            # a position that comes anew starts without weight: the slots behind the kept ones
            for b in range(batch):
                for i in range(keep, wide * page):
                    p_, s_ = R.position(table, b, i, page, pages)
                    W[p_, :, s_] = 0
    assert evictions >= 2 and length.tolist() == [len(keys[0][0])] * batch
