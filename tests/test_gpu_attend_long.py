"""Lengths and batches at which the operators of tests/test_gpu_cache.py and tests/test_gpu_attention_cross.py take another way: eviction that reads the weights again each
round, joins of more parts than are looked at together, more items than one launch of the store holds.  Small heads, so that a case takes little memory; each test
computes from the workspace's size, or from the sizes themselves, that its case goes that way (parts of the queries' test: a multiple of 256 keys, less a few, is cut into parts of 256)."""
import math

import pytest
import torch

import attend_ref as R
import paper_2303_11257_amd as us
from gpu_util import DEV, ptr, stream
from test_gpu_attention_cross import Call
from test_gpu_cache import F8, Paged, bits, dt, pool, tables

pytestmark = pytest.mark.gpu


# ---- eviction: 4 to 16 weights a thread in registers, and more ------------------------------------------------------------------

@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("lens,kv,page,keep,recent,fp8", [([5000, 4097, 4096, 3, 0], 1, 64, 700, 0, False), ([16384, 9001], 2, 256, 4000, 130, True), ([20011, 16385, 400], 1, 128, 701, 0, False),
                                                          ([40000, 16400], 1, 1024, 17000, 33, True), ([17000], 3, 16, 1, 0, False), ([24000], 1, 512, 23999, 4001, False)], ids=str)
def test_evict_long(lens, kv, page, keep, recent, fp8, ties, in_place):
    """Few different weights (ties), zeros of both signs, NaN and infinities; pages that there are not at the start, in the middle and at the end."""
    g = torch.Generator().manual_seed(len(lens) * keep)
    n, dh, most = len(lens), 16, max(lens)
    assert most - recent > 4096
    into = [] if in_place else [min(x, keep) for x in lens]
    both, pages = tables(lens + into, page, g)
    table, to = both[:n].contiguous(), (both[:n] if in_place else both[n:]).contiguous()
    for i in (0, lens[0] // page // 2, lens[0] // page - 3):
        table[0, i] = (-1, pages, 2 ** 31 - 1)[i % 3]
        if in_place:
            to[0, i] = table[0, i]
    K, V = pool(pages, kv, page, dh, fp8, g), pool(pages, kv, page, dh, fp8, g)
    W = torch.rand(pages, kv, page, generator=g) * 3 - 1
    if ties:
        W = (W * 4).round() / 4
        W.view(-1)[::7] *= -1.0
        W.view(-1)[5::5000] = float("nan")
        W.view(-1)[6::7000] = -math.inf
        W.view(-1)[8::9000] = math.inf
    dev = {m: x.to(DEV) for m, x in (("K", K), ("V", V), ("W", W), ("table", table))}
    td = dev["table"] if in_place else to.to(DEV)
    ld = torch.tensor(lens, dtype=torch.int32, device=DEV)
    new, kept = torch.full((n,), -9, dtype=torch.int32, device=DEV), torch.full((n, kv, keep), -9, dtype=torch.int32, device=DEV)
    us.cache_evict(ptr(dev["K"]), ptr(dev["V"]), ptr(dev["W"]), dt(fp8), pages, page, ptr(dev["table"]), table.shape[1], ptr(td), to.shape[1], ptr(ld), ptr(new), ptr(kept), n, kv,
                   dh, most, keep, recent, stream())
    want = R.evict(W, table, lens, page, most, keep, recent)
    assert kept.cpu().tolist() == [[h + [-1] * (keep - len(h)) for h in s] for s in want]
    assert new.tolist() == [min(x, keep) for x in lens]

    def rows_of(tab, b, positions):      # (page, slot) of positions, and which of them there are
        i = torch.tensor(positions, dtype=torch.long)
        p = tab[b].long()[i // page] if len(positions) else i
        return p, i % page, (p >= 0) & (p < pages)
    for name, x in (("K", bits(K)), ("V", bits(V)), ("W", W)):
        y = x.clone()
        for b in range(n):
            for h in range(kv):
                q, t, from_ok = rows_of(table, b, want[b][h])
                p, s, to_ok = rows_of(to, b, list(range(len(want[b][h]))))
                ok = from_ok & to_ok
                y[p[ok], h, s[ok]] = x[q[ok], h, t[ok]]
        got = bits(dev[name]).cpu()
        assert torch.equal(got.view(torch.int32) if name == "W" else got, y.view(torch.int32) if name == "W" else y), name


# ---- attention of one token: more than 256 parts of a row, the join's second statistics of a thread ------------------------------

@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,heads,dh", [([40001], 1, 16), ([33500], 5, 32), ([100003], 2, 16)], ids=str)
@pytest.mark.parametrize("weights", [False, True])
def test_attention_of_long_sequences(lens, heads, dh, weights, fp8):
    """One key head.  Keys grow along the sequence, so that the largest score lies in the last parts."""
    plain = us.attention_paged_workspace_bytes(1, heads, 1, dh, max(lens), False)
    assert plain >= 257 * heads * (8 + 4 * dh)
    c = Paged(lens, heads, 1, dh, 64, fp8, weights, seed=heads)
    grow = torch.zeros(c.K.shape[0])
    for i in range(-(-lens[0] // 64)):
        grow[int(c.table[0, i])] = 0.5 + 2.0 * i * 64 / lens[0]
    K = c.K.float() * grow[:, None, None, None]
    c.K = K.clamp(-448, 448).to(F8) if fp8 else K.half()
    c.dev["K"].copy_(c.K)
    c.run()
    c.check()


# ---- attention over another sequence ----------------------------------------------------------------------------------------------

def grown(dims, klen=None, seed=0):
    """Keys that grow along the sequence."""
    c = Call(*dims, klen=klen, seed=seed, fill=float("nan"))
    c.K.copy_((c.K.float() * torch.linspace(0.5, 2.5, dims[4])[:, None]).half())
    c.t["K"].copy_(c.K)
    return c


@pytest.mark.parametrize("dims", [(1, 1, 1, 40001, 16), (1, 4, 1, 36000, 32), (1, 1, 1, 70000, 80)], ids=str)
def test_one_query_in_more_than_256_parts(dims):
    batch, heads, kv, sk, dh = dims
    c = grown((batch, heads, kv, 1, sk, dh), seed=dh)
    assert c.wsb >= 257 * heads * (8 + 4 * dh)
    c.fwd()
    c.check(back=False)


@pytest.mark.parametrize("dims,klen", [((1, 1, 1, 20, 20479, 16), None), ((1, 2, 1, 30, 24575, 96), [24570]), ((2, 1, 1, 40, 18431, 64), [18431, 17000]), ((1, 1, 1, 33, 33001, 160), None)], ids=str)
def test_queries_in_more_than_64_parts(dims, klen):
    """The join takes 64 parts at a time; its maximum moves with the second 64."""
    c = grown(dims, klen, seed=dims[5])
    batch, heads, kv, sq, sk, dh = dims
    rows = batch * heads * sq
    assert c.wsb >= 65 * rows * (8 + 4 * dh)
    c.fwd()
    c.bwd()
    c.check()


# ---- store: more items than a launch holds ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("batch", [32767, 32768, 65535])
def test_store_of_many_sequences(batch, fp8):
    g = torch.Generator().manual_seed(batch)
    kv, s, dh, page = 1, 2, 16, 16
    table = torch.randperm(batch, generator=g).int().view(batch, 1)
    count = torch.randint(0, 3, (batch,), generator=g).int()
    lens = count + torch.randint(0, 15, (batch,), generator=g).int()
    lens = torch.minimum(lens, torch.tensor(page, dtype=torch.int32))
    x = torch.randn(2, batch, kv, s, dh, generator=g).half()
    cache = [torch.zeros(batch, kv, page, dh, dtype=torch.uint8 if fp8 else torch.float16, device=DEV) for _ in range(2)]
    xd, td, ld, cd = x.to(DEV), table.to(DEV), lens.to(DEV), count.to(DEV)
    us.cache_store(ptr(xd[0]), ptr(xd[1]), None, ptr(cache[0]), ptr(cache[1]), dt(fp8), batch, page, ptr(td), 1, ptr(ld), ptr(cd), batch, kv, s, dh, stream())
    for i in range(2):
        rows = x[i].float().clamp(-448, 448).to(F8).view(torch.uint8) if fp8 else x[i]
        want = torch.zeros(batch, kv, page, dh, dtype=rows.dtype)
        for t in range(s):
            b = (t < count).nonzero().view(-1)
            want[table[b, 0].long(), :, (lens - count)[b].long() + t] = rows[b, :, t]
        assert torch.equal(cache[i].cpu(), want)
