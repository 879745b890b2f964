"""Chunks of new tokens over the paged cache: page tables and slot maps against the oracle's
entry-by-entry form, packed writes, and the attention of packed queries against fp64, at the
sizes, lengths and masks where they can go wrong. Tolerances are the bounds on the kernels'
roundings that test_gpu_sequence derives (logits, probabilities and output; one rounding of the
probabilities in bf16)."""
import math
import random

import numpy as np
import pytest

from oracle import seq
from tests.test_gpu_sequence import DT, _bounds, _ca, _close, _gen, _np, _pages, _rand, _torch, _u

pytestmark = pytest.mark.gpu


def _i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- pages and slots ---------------------------------------------------------------------------

class _Both:
    """The same pool and table on the GPU and in the oracle."""

    def __init__(self, B, width, page, pages, seed=0):
        import torch
        self.page, self.pages = page, pages
        order = torch.randperm(pages, generator=_gen(seed)).tolist()
        self.free, self.rows = list(order), [[-1] * width for _ in range(B)]
        self.pool = _ca().PagePool(page, _i32(order), _i32([pages, 7, 7]))
        self.wide = torch.full((B, width + 3), 99, dtype=torch.int32, device="cuda")
        self.table = self.wide[:, :width]  # rows further apart than they are long
        self.table.fill_(-1)

    def grow(self, lens, new, tokens, **kw):
        got = _ca().cache_grow(self.pool, self.table, _i32(lens), _i32(new), tokens, **kw)
        state, starts, slots, positions = seq.cache_grow(self.rows, self.free, lens, new, self.page, self.pages, tokens)
        assert got.starts.tolist() == starts
        assert got.slots.tolist() == slots and got.positions[0].tolist() == positions
        assert self.pool.state.tolist() == state
        self.same()
        return got

    def release(self, lens, left=-1, sinks=0):
        _ca().cache_release(self.pool, self.table, _i32(lens), left=left, sinks=sinks)
        seq.cache_release(self.rows, self.free, lens, self.page, self.pages, left, sinks)
        self.same()

    def same(self):
        assert self.table.tolist() == self.rows
        n = int(self.pool.state[0])
        assert n == len(self.free) and self.pool.free[:n].tolist() == self.free
        assert bool((self.wide[:, self.table.shape[1]:] == 99).all())


@pytest.mark.parametrize("page", [1, 5, 16, 100, 256])
@pytest.mark.parametrize("B", [1, 3, 64, 1025])
def test_pages_through_many_steps(page, B):
    """Sequences that grow by nothing, a token or many, are cut back, finish, and give back what lies
    behind a window; a pool that runs short now and then."""
    r = random.Random(page + B)
    width = max(3, 700 // page // (1 + B // 100) + 2)
    both = _Both(B, width, page, max(2, B * width * 2 // 3), seed=page)
    lens = [0] * B
    for step in range(7):
        new = [r.choice((0, 1, 1, r.randrange(1, 2 * page + 40))) for _ in range(B)]
        lens = [min(a + n, width * page) for a, n in zip(lens, new)]
        tokens = max(1, sum(min(a, n) for a, n in zip(lens, new)) + r.choice((0, 0, 5)))
        both.grow(lens, new, tokens)
        if r.random() < 0.4:
            lens = [max(0, a - r.randrange(3)) for a in lens]
            both.release(lens)
        if r.random() < 0.4:
            both.release(lens, left=r.choice((0, 1, page, 3 * page + 2)), sinks=r.choice((0, 1, page + 1)))
        if r.random() < 0.6:
            lens[r.randrange(B)] = 0
            both.release(lens)
    both.release([0] * B)
    assert int(both.pool.state[0]) == both.pages


@pytest.mark.parametrize("B,cached,new,page", [(1, 0, 30000, 1), (2, 5, 20000, 16), (64, 1000, 500, 32), (3000, 7, 9, 2),
                                               (1, 0, 1, 16), (5, 0, 0, 16)])
def test_pages_of_prompts(B, cached, new, page):
    """Many new pages at once, and back: the free list ends as it was."""
    width = (cached + new) // page + 2
    both = _Both(B, width, page, B * width)
    if cached:
        both.grow([cached] * B, [cached] * B, B * cached)
    before, n = both.pool.free.clone(), int(both.pool.state[0])
    lens = [cached + (new if b % 3 != 1 else 0) for b in range(B)]
    grown = [a - cached for a in lens]
    one = both.grow(lens, grown, sum(grown) + 10)
    both.grow(lens, grown, sum(grown) + 10, out=one)  # changes nothing
    both.release([cached] * B)
    assert (both.pool.free == before).all() and int(both.pool.state[0]) == n


def test_pages_that_lack_and_come_later():
    """A pool that runs short: later entries stay, say so, and get theirs when pages come back."""
    both = _Both(3, 6, 4, 5)
    both.grow([4, 12, 9], [4, 12, 9], 25)
    assert both.pool.state.tolist() == [0, 2, 0]
    both.release([0, 12, 9])
    both.grow([0, 12, 9], [0, 12, 9], 20)  # fewer rows than tokens
    assert both.pool.state.tolist() == [0, 1, 1]


def test_pages_lengths_that_make_no_sense():
    """Lengths below 0 and beyond the table, more new tokens than tokens, entries outside the pool."""
    both = _Both(4, 5, 8, 30)
    both.table[2, 1], both.rows[2][1] = 2 ** 31 - 1, 2 ** 31 - 1
    both.table[3, 0], both.rows[3][0] = 30, 30
    both.grow([-3, 10 ** 9, 20, 5], [4, 7, 10 ** 9, -1], 40)
    both.release([2 ** 31 - 1, -2 ** 31, 12, 3], left=3, sinks=2 ** 31 - 1)
    both.release([2 ** 31 - 1, -2 ** 31, 12, 3], left=2 ** 31 - 1, sinks=0)
    both.release([40, 0, 12, 3], left=2)


def test_pages_of_a_state_that_makes_no_sense():
    """Counts outside the stack are cut to it: nothing is read or written outside."""
    ca = _ca()
    for n in (-5, 10 ** 9):
        pool = ca.PagePool(4, _i32([0, 1, 2]), _i32([n, 0, 0]))
        table = _i32([[-1] * 5, [0, 1, 2, 0, 1]])
        ca.cache_grow(pool, table, _i32([20, 20]), _i32([20, 0]), 20)
        assert pool.state[0] == 0 and pool.state[1] == (5 if n < 0 else 2)
        ca.cache_release(pool, table, _i32([0, 0]))
        assert pool.state[0] == 3 and bool((table == -1).all()) and bool(((pool.free >= 0) & (pool.free < 3)).all())


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("page,Hk,d", [(16, 2, 64), (7, 3, 128), (1, 1, 64), (64, 5, 64)])
def test_write(dt, page, Hk, d):
    """Rows with a slot are written, nothing else; slots outside the pools are left out."""
    import torch
    ca = _ca()
    g = _gen(page)
    pages, T = 40, 23
    kp, vp = (_rand(g, (pages, page, Hk, d), dt).cuda() for _ in range(2))
    k, v = (_rand(g, (T, Hk, d), dt).cuda() for _ in range(2))
    slots = torch.randperm(pages * page, generator=g)[:T] if pages * page >= T else None
    slots[3], slots[8], slots[9], slots[10] = -1, pages * page, -2 ** 62, 2 ** 62
    wk, wv = kp.clone(), vp.clone()
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < pages * page:
            wk[s // page, s % page], wv[s // page, s % page] = k[t], v[t]
    heads_first = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kp, vp)]  # other strides
    both = torch.stack((kp, vp), 2)
    fused = torch.stack((k, v), 1)  # rows of a fused projection
    ca.cache_write(k, v, kp, vp, slots.cuda())
    ca.cache_write(fused[:, 0], fused[:, 1], *heads_first, slots.cuda())
    ca.cache_write(k, v, *both.unbind(2), slots.cuda())
    for a, b in ((kp, vp), heads_first, both.unbind(2)):
        assert torch.equal(a, wk) and torch.equal(b, wv)
    one = k[:1].expand(T, Hk, d)  # a stride of 0 repeats an input
    ca.cache_write(one, one, kp, vp, slots.cuda())
    at = [s for s in slots.tolist() if 0 <= s < pages * page]
    assert all(torch.equal(kp[s // page, s % page], k[0]) for s in at)


@pytest.mark.parametrize("d", [4, 20, 100])
def test_write_f32_head_dims(d):
    import torch
    g = _gen(d)
    kp, vp = (torch.zeros(3, 5, 2, d, device="cuda") for _ in range(2))
    k, v = (_rand(g, (4, 2, d), "f32").cuda() for _ in range(2))
    _ca().cache_write(k, v, kp, vp, torch.tensor([14, 0, 6, -1], device="cuda"))
    assert torch.equal(kp.flatten(0, 1)[[14, 0, 6]], k[:3]) and torch.equal(vp.flatten(0, 1)[[14, 0, 6]], v[:3])
    assert int(kp.any(-1).any(-1).sum()) == 3


# ---- attention ---------------------------------------------------------------------------------

def _chunk_check(dt, tokens, H, Hk, d, page, seed=0, scale=None, spare=3, size=1.0, q=None, heads_first=False, pages=None,
                 layout="thd", ws=None, change=None, **kw):
    """tokens: (all, new) of each sequence. `change(k_pages, v_pages, table, rows, lens)` may alter what
    is hidden. Rows behind the last sequence keep what they held."""
    import torch
    ca = _ca()
    g = _gen(seed)
    lens, new = [a for a, _ in tokens], [n for _, n in tokens]
    kp, vp, table, rows = pages or _pages(g, dt, lens, page, Hk, d, heads_first=heads_first)
    if change:
        change(kp, vp, table, rows, lens)
    starts = np.cumsum([0] + new).tolist()
    T = starts[-1] + spare
    q = _rand(g, (T, H, d), dt, size) if q is None else q
    qc = q.cuda()
    if layout == "htd":
        qc = qc.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.full_like(qc, 7.0)
    lse = torch.full((T, H), 7.0, device="cuda")
    w = ca.Window(**kw)
    o, z = ca.paged_chunk_attn(w, qc, kp, vp, table, _i32(lens), _i32(starts), scale=scale, out=out, lse=lse, ws=ws)
    assert o is out and z is lse
    assert bool((out[starts[-1]:] == 7).all()) and bool((lse[starts[-1]:] == 7).all())
    for b, (a, n) in enumerate(tokens):
        see = seq.visible(n, a, kw.get("left", -1), kw.get("right", -1), kw.get("sinks", 0), kw.get("causal", False))
        for h in range(H):
            hk, at = h // (H // Hk), slice(starts[b], starts[b + 1])
            want = _bounds(_np(q)[at, h], rows[b][0][:, hk], rows[b][1][:, hk], None, see, scale or 1.0 / math.sqrt(d), dt)
            _close(_np(out)[at, h], *want["out"], f"sequence {b} head {h}")
            _close(_np(lse)[at, h], *want["lse"], f"lse of sequence {b} head {h}")
    return out, lse


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("page", [1, 7, 16, 48, 64, 100, 128])
@pytest.mark.parametrize("kw", [dict(causal=True), dict(), dict(left=0, right=0), dict(left=90, sinks=5, causal=True),
                                dict(left=33, right=10, sinks=200), dict(left=70, right=40, sinks=3, causal=True)])
def test_chunk_lengths(dt, page, kw):
    """Sequences without tokens, without new ones, with nothing but new ones, of one token, lengths at and
    beside the edges of tiles."""
    tokens = [(0, 0), (1, 1), (5, 0), (64, 64), (65, 3), (63, 1), (129, 40), (300, 1), (200, 131), (32, 16), (31, 31)]
    _chunk_check(dt, tokens, 2, 2, 64, page, seed=page, **kw)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("H,Hk", [(1, 1), (5, 1), (16, 1), (17, 1), (40, 1), (24, 8), (66, 2), (3, 3), (6, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_heads(dt, H, Hk, d):
    _chunk_check(dt, [(200, 9), (31, 31), (70, 1)], H, Hk, d, 16, seed=H, scale=0.2, heads_first=H % 2 == 0,
                 layout="htd" if H % 3 else "thd", causal=True)


@pytest.mark.parametrize("d", [4, 20, 32, 36, 100])
def test_chunk_f32_head_dims(d):
    _chunk_check("f32", [(150, 20), (17, 17), (90, 2)], 4, 2, d, 8, seed=d, left=60, sinks=3, causal=True)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [dict(causal=True), dict(), dict(left=700, sinks=70, causal=True), dict(left=400, right=150)])
def test_chunk_longer(dt, d, kw):
    """Prompts of several blocks beside sequences that go on by a token, some cut into parts."""
    _chunk_check(dt, [(900, 300), (5000, 1), (260, 260), (3000, 5), (1, 1), (2500, 129)], 4, 2, d, 32, seed=d, **kw)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("H,Hk,n", [(1, 1, 1), (2, 1, 16), (8, 2, 40), (40, 1, 3)])
def test_chunk_few_queries_on_a_long_cache(dt, H, Hk, n):
    """The split over the cache; a table wider than needed gives the same."""
    import torch
    ca = _ca()
    d, lens = 64, [20003]
    pages = _pages(_gen(5), dt, lens, 32, Hk, d)
    a = _chunk_check(dt, [(lens[0], n)], H, Hk, d, 32, size=4.0, pages=pages, causal=True)
    kp, vp, table, rows = pages
    wide = torch.full((1, 9000), -1, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    _chunk_check(dt, [(lens[0], n)], H, Hk, d, 32, size=4.0, pages=(kp, vp, wide, rows), causal=True)
    b = _chunk_check(dt, [(lens[0], n)], H, Hk, d, 32, size=4.0, pages=pages, causal=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))  # same bits twice


@pytest.mark.parametrize("dt", DT)
def test_chunk_more_new_tokens_than_tokens(dt):
    """Lengths cut to the table and below the new tokens: queries before the first key see nothing (causal)
    or what lies to their right."""
    import torch
    ca = _ca()
    g = _gen(6)
    lens = [20, 0, 48]
    kp, vp, table, rows = _pages(g, dt, lens, 16, 2, 64)
    q = _rand(g, (130, 4, 64), dt)
    starts = [0, 50, 60, 130]
    for kw in (dict(causal=True), dict(left=5, right=12), dict(), dict(sinks=4, causal=True, left=2)):
        out, lse = ca.paged_chunk_attn(ca.Window(**kw), q.cuda(), kp, vp, table, _i32([20, -7, 48]), _i32(starts), want_lse=True)
        for b, a in enumerate(lens):
            at = slice(starts[b], starts[b + 1])
            see = seq.visible(starts[b + 1] - starts[b], a, kw.get("left", -1), kw.get("right", -1), kw.get("sinks", 0),
                              kw.get("causal", False))
            for h in range(4):
                want = _bounds(_np(q)[at, h], rows[b][0][:, h // 2], rows[b][1][:, h // 2], None, see, 0.125, dt)
                _close(_np(out)[at, h], *want["out"], f"{kw} {b} {h}")
                _close(_np(lse)[at, h], *want["lse"], f"{kw} lse {b} {h}")


@pytest.mark.parametrize("dt", DT)
def test_chunk_bad_entries_hold_no_tokens(dt):
    """Entries outside the pool inside what is seen: their keys are not there. Lengths beyond the table are
    cut to it; starts are cut to the rows."""
    import torch
    ca = _ca()
    g = _gen(7)
    for page in (16, 10, 64):
        lens = [6 * page + 5, 6 * page, 20]
        kp, vp, table, rows = _pages(g, dt, lens, page, 1, 64)
        table = table[:, :6].contiguous()
        table[0, 2], table[1, 5], table[1, 0] = 10 ** 6, -7, 2 ** 31 - 1
        q = _rand(g, (60, 2, 64), dt)
        out, lse = ca.paged_chunk_attn(ca.Window(causal=True), q.cuda(), kp, vp, table, _i32([10 ** 9, 6 * page, -3]),
                                       _i32([0, 25, 60, 10 ** 9]), want_lse=True)
        for b, gone in ((0, (2,)), (1, (0, 5))):
            n, at = (25, 35)[b], slice(0, 25) if b == 0 else slice(25, 60)
            see = seq.visible(n, 6 * page, causal=True)
            for e in gone:
                see[:, e * page:(e + 1) * page] = False
            for h in range(2):
                want = _bounds(_np(q)[at, h], rows[b][0][:6 * page, 0], rows[b][1][:6 * page, 0], None, see, 0.125, dt)
                _close(_np(out)[at, h], *want["out"], f"{page} {b}")
                _close(_np(lse)[at, h], *want["lse"], f"{page} {b} lse")


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("page", [16, 24])
def test_chunk_hidden_pages_are_not_read(dt, page):
    """Pages that no new token sees may be gone: their entries lie outside the pool. A common beginning is
    read by both sequences."""
    import torch
    lens, left = [40 * page, 40 * page], 10 * page

    def change(kp, vp, table, rows, lens):
        table[1, :2] = table[0, :2]
        for i in range(2):
            rows[1][i][:2 * page] = rows[0][i][:2 * page]
        bad = torch.tensor([-1, -5, 10 ** 6, 2 ** 31 - 1], dtype=torch.int32).repeat(7).cuda()
        table[:, 2:28] = bad[:26]

    _chunk_check(dt, [(n, 2 * page) for n in lens], 4, 2, 64, page, left=left, sinks=2 * page, causal=True, change=change)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [dict(causal=True), dict(left=30, causal=True, sinks=3), dict(left=20, right=10)])
@pytest.mark.parametrize("where,value", [("v", float("nan")), ("v", float("inf")), ("k", float("nan")), ("k", float("inf"))])
def test_chunk_hidden_values_may_be_anything(dt, d, kw, where, value):
    """One token's key or value is not finite: the queries that do not see it are what they were, those that see
    such a value are not finite."""
    import torch
    ca = _ca()
    g = _gen(8)
    lens, new, at = [300, 90], [140, 90], 200
    kp, vp, table, rows = _pages(g, dt, lens, 16, 1, d)
    starts = _i32([0, 140, 230])
    q = _rand(g, (230, 2, d), dt).cuda()
    w, n = ca.Window(**kw), _i32(lens)
    a, la = ca.paged_chunk_attn(w, q, kp, vp, table, n, starts, want_lse=True)
    pool = vp if where == "v" else kp
    pool[int(table[0, at // 16]), at % 16] = value
    b, lb = ca.paged_chunk_attn(w, q, kp, vp, table, n, starts, want_lse=True)
    see = seq.visible(140, 300, kw.get("left", -1), kw.get("right", -1), kw.get("sinks", 0), kw.get("causal", False))
    sees = torch.from_numpy(np.concatenate((see[:, at], np.zeros(90, bool)))).cuda()
    tol = 4 * _u(dt) * float(vp.float().nan_to_num(posinf=0.0).abs().max())  # each within 2 u of the exact result
    assert (a[~sees].float() - b[~sees].float()).abs().max() <= tol and (la[~sees] - lb[~sees]).abs().max() <= 1e-4
    if where == "v":
        assert not bool(torch.isfinite(b[sees]).any()) and (la - lb).abs().max() <= 1e-4


def _steep(dt, d, bits, v, n, page, **kw):
    """Every query's logit of key j is bits[j] in log2 units, exactly before the scale."""
    import torch
    g = _gen(9)
    k = _rand(g, (len(bits), 1, d), dt)
    k[:, 0, 0] = torch.from_numpy(np.asarray(bits) / 2.0).to(_torch(dt))
    v = v.to(_torch(dt))[:, None]
    count = -(-len(bits) // page)
    kp, vp = (torch.zeros(count * page, 1, d, dtype=_torch(dt)) for _ in range(2))
    kp[:len(bits)], vp[:len(bits)] = k, v
    q = torch.zeros(n + 1, 1, d, dtype=_torch(dt))
    q[..., 0] = 2.0
    pages = (kp.reshape(count, page, 1, d).cuda(), vp.reshape(count, page, 1, d).cuda(),
             torch.arange(count, dtype=torch.int32, device="cuda")[None], [(_np(k), _np(v))])
    _chunk_check(dt, [(len(bits), n)], 1, 1, d, page, scale=math.log(2.0), q=q, spare=1, pages=pages, **kw)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("slope", [0.90, 0.97, 1.0])
@pytest.mark.parametrize("kw", [dict(causal=True), dict(left=190, right=0), dict(left=10, right=0, sinks=200)])
def test_chunk_rising_ramps(dt, d, slope, kw):
    """Logits that rise to just below the range of fp32 over the first ones; the values change sign at a tile's edge."""
    import torch
    n = 256
    bits = torch.tensor([slope * j - 100 for j in range(n)]).to(torch.bfloat16).double().numpy()
    v = torch.randn(n, d, generator=_gen(40))
    v[:, ::2] = torch.where(torch.arange(n) < 192, 1.0, -1.0)[:, None]
    _steep(dt, d, bits, v, n, 16, **kw)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mid,top", [(117.0, 125.0), (118.0, 128.0), (110.0, 127.0), (118.0, 250.0), (-20.0, 130.0)])
def test_chunk_last_tile_far_above(dt, d, mid, top):
    import torch
    n = 320
    for last in (0, 8, 63):
        bits = np.where(np.arange(n) < 64, 0.0, mid)
        bits[256:] = -60.0
        bits[256 + last] = top
        _steep(dt, d, bits, torch.randn(n, d, generator=_gen(42)), 64, 32, left=310, right=0)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tops,firsts", [((117, 0, 117, 117, 60, 117, 0, 116), 0), ((117,) * 8, 127), ((0, 117) * 4, 240)])
def test_chunk_parts_far_apart(dt, d, tops, firsts):
    """Few queries on keys in parts: each lies far above or below its first tile and the other parts."""
    import torch
    nk = 512 * len(tops)
    bits = np.zeros(nk)
    for i, t in enumerate(tops):
        bits[512 * i + 64:512 * (i + 1)] = t
        if i % 2:
            bits[512 * i + 5] = firsts
    _steep(dt, d, bits, torch.randn(nk, d, generator=_gen(43)), 9, 64)


@pytest.mark.parametrize("dt", DT)
def test_chunk_large_logits(dt):
    _chunk_check(dt, [(300, 100), (700, 3)], 2, 1, 64, 16, size=30.0, causal=True)


@pytest.mark.parametrize("dt", DT)
def test_chunk_of_one_is_paged_attn(dt):
    """With a token each, the results of paged_attn: both within their bounds of the exact ones."""
    ca = _ca()
    lens = [1, 700, 64, 333]
    kp, vp, table, _ = _pages(_gen(10), dt, lens, 16, 2, 64)
    q = _rand(_gen(11), (4, 6, 64), dt).cuda()
    for kw in (dict(), dict(left=100, sinks=9)):
        a, la = ca.paged_attn(q, kp, vp, table, _i32(lens), want_lse=True, **kw)
        b, lb = ca.paged_chunk_attn(ca.Window(causal=True, **kw), q, kp, vp, table, _i32(lens), _i32(range(5)), want_lse=True)
        tol = 4 * (_u(dt) + 2.0 ** -20) * float(vp.float().nan_to_num().abs().max())
        assert (a.float() - b.float()).abs().max() <= tol and (la - lb).abs().max() <= 1e-4


# ---- strides, places, streams, graphs ------------------------------------------------------------

@pytest.mark.parametrize("dt", DT)
def test_chunk_pools_that_lie_in_one_tensor(dt):
    """Keys and values of a page, a token or a head side by side; a query repeated; an output inside a larger one."""
    import torch
    ca = _ca()
    lens, w = [37, 100], _ca().Window(causal=True)
    kp, vp, table, _ = _pages(_gen(12), dt, lens, 16, 2, 64)
    q = _rand(_gen(13), (1, 4, 64), dt).cuda().expand(50, 4, 64)
    n, starts = _i32(lens), _i32([0, 20, 50])
    want = ca.paged_chunk_attn(w, q.contiguous(), kp, vp, table, n, starts, want_lse=True)
    for dim in (1, 2, 3):
        big = torch.zeros(50, 8, 128, dtype=_torch(dt), device="cuda")
        a, b = torch.stack((kp, vp), dim).unbind(dim)
        _, z = ca.paged_chunk_attn(w, q, a, b, table, n, starts, out=big[:, ::2, 64:], want_lse=True)
        assert torch.equal(big[:, ::2, 64:], want[0]) and torch.equal(z, want[1])
        assert not big[:, 1::2].any() and not big[..., :64].any()


def test_chunk_offsets_past_32_bits():
    """Pages, rows and heads whose elements lie past 2^32; slots past 2^31."""
    import torch
    ca = _ca()
    g = _gen(14)
    far = 2 ** 32 + 2 ** 20
    pool = torch.empty(far + 2 ** 20, dtype=torch.bfloat16, device="cuda")
    kp, vp = (pool.as_strided((2, 64, 2, 64), (far, 128, 64, 1), 8192 * (40 + i)) for i in range(2))
    k, v = (_rand(g, (100, 2, 64), "bf16").cuda() for _ in range(2))
    slots = torch.cat((torch.arange(64, 128), torch.arange(36))).cuda()
    ca.cache_write(k, v, kp, vp, slots)
    assert torch.equal(kp[1], k[:64]) and torch.equal(vp[0, :36], v[64:])
    table, lens, starts = _i32([[1, 0]]), _i32([100]), _i32([0, 30])
    near = _rand(g, (30, 2, 64), "bf16").cuda()
    q, out = (pool.as_strided((30, 2, 64), (64, far, 1), 32768 * i) for i in (1, 2))
    q.copy_(near)
    w = ca.Window(causal=True, left=80)
    a, la = ca.paged_chunk_attn(w, q, kp, vp, table, lens, starts, want_lse=True, out=out)
    b, lb = ca.paged_chunk_attn(w, near, kp.clone(), vp.clone(), table, lens, starts, want_lse=True)
    assert torch.equal(a, b) and torch.equal(la, lb)
    del pool, kp, vp, q, out, a
    # 2^31 places and some: rows of 16 bytes
    page, pages = 2 ** 20, 2 ** 11 + 3
    kp = torch.empty(pages, page, 1, 4, device="cuda")
    k = _rand(g, (3, 1, 4), "f32").cuda()
    slots = torch.tensor([2 ** 31 + 5, 2 ** 31 + 2 ** 21 + 1, 0], device="cuda")
    ca.cache_write(k, k, kp, kp.as_strided(kp.shape, kp.stride()), slots)
    assert torch.equal(kp.flatten(0, 1)[slots], k)
    # the last pages of a pool beyond 2^31 places, from the free list
    p = ca.PagePool(page, _i32([pages - 1, pages - 2]), _i32([2, 0, 0]))
    p = ca.PagePool(page, torch.cat((p.free, torch.zeros(pages - 2, dtype=torch.int32, device="cuda"))), p.state)
    got = ca.cache_grow(p, _i32([[-1, -1]]), _i32([page + 1]), _i32([2]), 2)
    assert got.slots.tolist() == [(pages - 2) * page + page - 1, (pages - 1) * page]


def test_chunk_places_near_2_to_the_30():
    """A sequence of almost 2^30 tokens whose window leaves a few pages to see."""
    import torch
    ca = _ca()
    g = _gen(15)
    page = 1 << 14
    width = (1 << 16) - 1
    n = width * page
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, -1], table[0, 0] = 1, 0
    for dt in DT:
        kp, vp = (_rand(g, (2, page, 1, 64), dt).cuda() for _ in range(2))
        q = _rand(g, (20, 2, 64), dt)
        for kw in (dict(left=500, sinks=30, causal=True), dict(left=500, right=2 ** 31 - 1), dict(left=400, sinks=3, right=5)):
            out, lse = ca.paged_chunk_attn(ca.Window(**kw), q.cuda(), kp, vp, table, _i32([n]), _i32([0, 20]), want_lse=True)
            sinks = kw.get("sinks", 0)
            keep = 600
            see = seq.visible(20, keep, kw["left"], min(kw.get("right", -1), 10 ** 6), 0, kw.get("causal", False))
            see = np.concatenate((np.ones((20, sinks), bool), see), 1)
            k, v = (np.concatenate((_np(x)[0, :sinks, 0], _np(x)[1, page - keep:, 0])) for x in (kp, vp))
            for h in range(2):
                want = _bounds(_np(q)[:, h], k, v, None, see, 0.125, dt)
                _close(_np(out)[:, h], *want["out"], f"{dt} {kw}")
                _close(_np(lse)[:, h], *want["lse"], f"{dt} {kw} lse")


def _step(ca, s, ws=None):
    """A serving step on the tensors of s: pages, rotary, write, attention, pages back."""
    plan = ca.cache_grow(s["pool"], s["table"], s["lens"], s["new"], s["q"].shape[0])
    q, k = ca.rope(s["rope"], s["q"][None], s["k"][None], positions=plan.positions, layout="bnhd")
    ca.cache_write(k[0], s["v"], s["kp"], s["vp"], plan.slots)
    out, lse = ca.paged_chunk_attn(s["w"], q[0], s["kp"], s["vp"], s["table"], s["lens"], plan.starts, want_lse=True, ws=ws)
    ca.cache_release(s["pool"], s["table"], s["lens"], left=s["w"].left, sinks=s["w"].sinks)
    return out, lse, plan


def _serving(dt, w, page, pages, B, width, T, H=4, Hk=2, d=64):
    import torch
    ca = _ca()
    z = lambda *n: torch.zeros(*n, dtype=_torch(dt), device="cuda")  # noqa: E731
    return dict(w=w, rope=ca.rope_axes((d,), pairing="halves"), pool=ca.page_pool(pages, page),
                table=torch.full((B, width), -1, dtype=torch.int32, device="cuda"), lens=_i32([0] * B), new=_i32([0] * B),
                kp=z(pages, page, Hk, d), vp=z(pages, page, Hk, d), q=z(T, H, d), k=z(T, Hk, d), v=z(T, Hk, d))


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("kw", [dict(causal=True), dict(left=37, sinks=5, causal=True)])
def test_steps_of_any_size_equal_one_pass(dt, kw):
    """Three sequences served in steps of nothing, one, a few or many tokens, pages behind the window given back and
    taken by others, against one causal pass each."""
    import torch
    ca = _ca()
    g, r = _gen(16), random.Random(3)
    B, n, H, Hk, d, page = 3, [190, 75, 140], 4, 2, 64, 8
    w = ca.Window(**kw)
    s = _serving(dt, w, page, 60, B, 32, 200)
    xs = [[_rand(g, (m, h, d), dt).cuda() for h in (H, Hk, Hk)] for m in n]
    whole = []
    for (q, k, v), m in zip(xs, n):
        qr, kr = ca.rope(s["rope"], q[None], k[None], grid=(m,), layout="bnhd")
        whole.append(ca.window_attn(w, qr, kr, v[None], layout="bnhd", want_lse=True))
    at = [0] * B
    while at != n:
        new = [min(r.choice((0, 1, 1, 4, 33, 70)), m - a) for a, m in zip(at, n)]
        rows = 0
        for b in range(B):
            for x, name in zip(xs[b], ("q", "k", "v")):
                s[name][rows:rows + new[b]] = x[at[b]:at[b] + new[b]]
            rows += new[b]
        at = [a + m for a, m in zip(at, new)]
        s["lens"].copy_(_i32(at))
        s["new"].copy_(_i32(new))
        out, lse, plan = _step(ca, s)
        assert s["pool"].state[1:].tolist() == [0, 0]
        for b in range(B):
            i0 = int(plan.starts[b])
            got, lg = out[i0:i0 + new[b]].float(), lse[i0:i0 + new[b]]
            want, lw = whole[b][0][0, at[b] - new[b]:at[b]].float(), whole[b][1][0, :, at[b] - new[b]:at[b]].T
            if new[b]:
                assert (got - want).abs().max() <= 4 * (_u(dt) + 2.0 ** -20) * xs[b][2].float().abs().max()
                assert (lg - lw).abs().max() <= 1e-4
    if kw.get("left"):  # no more pages than the windows and sinks need
        assert 60 - int(s["pool"].state[0]) <= B * (37 // page + 2 + 1)


@pytest.mark.parametrize("dt", DT)
def test_steps_captured_and_replayed(dt):
    """A whole step captured once, replayed for steps of other lengths, with eager work and
    synchronizations between; two captured steps share one workspace."""
    import torch
    ca = _ca()
    w = ca.Window(causal=True)
    sets = [_serving(dt, w, 16, 400, 3, 100, 60) for _ in range(4)]  # two captured, two eager
    ws = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")

    def fill(s, seed, lens, new):
        g = _gen(seed)
        for x in ("q", "k", "v"):
            s[x].copy_(_rand(g, s[x].shape, dt))
        s["lens"].copy_(_i32(lens))
        s["new"].copy_(_i32(new))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(ca, sets[0], ws)
    torch.cuda.synchronize()
    graphs, held = [], []
    for s in sets[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            held.append(_step(ca, s, ws))
        torch.cuda.synchronize()
    lens = [0, 0, 0]
    for i, new in enumerate(([20, 0, 40], [1, 1, 1], [1, 50, 1], [30, 3, 0], [0, 0, 0], [1, 1, 58])):
        lens = [a + n for a, n in zip(lens, new)]
        for x in range(2):
            fill(sets[x], 10 * i + x, lens, new)
            fill(sets[2 + x], 10 * i + x, lens, new)
        for x in ((0, 1), (1, 0))[i % 2]:
            graphs[x].replay()
        want = [_step(ca, sets[2 + x]) for x in range(2)]
        torch.cuda.synchronize()
        m = sum(new)
        for x in range(2):
            out, lse, plan = held[x]
            assert torch.equal(out[:m], want[x][0][:m]) and torch.equal(lse[:m], want[x][1][:m])
            assert all(torch.equal(a, b) for a, b in zip(plan, want[x][2]))
            for name in ("table", "kp", "vp"):
                assert torch.equal(sets[x][name], sets[2 + x][name])
            assert torch.equal(sets[x]["pool"].state, sets[2 + x]["pool"].state)


@pytest.mark.parametrize("dt", DT)
def test_chunk_two_streams_at_once(dt):
    import torch
    ca = _ca()
    w = ca.Window(left=600, sinks=20, causal=True)
    args = []
    for i in range(2):
        lens = [3000 + 500 * i, 40, 900]
        kp, vp, table, _ = _pages(_gen(20 + i), dt, lens, 16, 2, 64)
        args.append((w, _rand(_gen(30 + i), (150, 4, 64), dt).cuda(), kp, vp, table, _i32(lens), _i32([0, 9, 49, 150])))
    want = [ca.paged_chunk_attn(*a, want_lse=True) for a in args]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(3):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = ca.paged_chunk_attn(*args[i], want_lse=True)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for x, y in zip(want, got) for a, b in zip(x, y))


@pytest.mark.parametrize("dt", DT)
def test_chunk_workspaces_and_refusals(dt):
    """A workspace of the caller's, one that is too small, and arguments that do not fit."""
    import torch
    ca = _ca()
    lens = [9000, 30]
    kp, vp, table, _ = _pages(_gen(50), dt, lens, 16, 2, 64)
    q, n, starts = _rand(_gen(51), (40, 4, 64), dt).cuda(), _i32(lens), _i32([0, 10, 40])
    w = ca.Window(causal=True)
    a = ca.paged_chunk_attn(w, q, kp, vp, table, n, starts, want_lse=True)
    ws = torch.full((256 << 20,), 255, dtype=torch.uint8, device="cuda")  # NaN all over
    b = ca.paged_chunk_attn(w, q, kp, vp, table, n, starts, want_lse=True, ws=ws)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    with pytest.raises(ca.CAError, match="workspace"):
        ca.paged_chunk_attn(w, q, kp, vp, table, n, starts, ws=ws[:256])
    call = lambda **kw: ca.paged_chunk_attn(w, **{**dict(q=q, k_pages=kp, v_pages=vp, page_table=table, lens=n,  # noqa: E731
                                                         starts=starts), **kw})
    other = torch.float32 if dt == "bf16" else torch.bfloat16
    for kw, word in ((dict(q=q.to(other)), "q: expected"), (dict(q=q[0]), r"\[T, H, d\]"), (dict(lens=n.long()), "lens"),
                     (dict(starts=starts[:2]), "starts"), (dict(v_pages=vp[:, :8]), "v_pages"), (dict(page_table=table[0]), "page_table"),
                     (dict(q=q[..., :32]), "last dimension"), (dict(lse=torch.zeros(4, 40, device="cuda")), "lse"),
                     (dict(lens=n.cpu()), "on cuda"), (dict(page_table=table.t().contiguous().t()), "contiguous"),
                     (dict(out=q[:, :2]), "out")):
        with pytest.raises(ValueError, match=word):
            call(**kw)
    with pytest.raises(ca.CAError, match="multiple of heads_k"):
        call(q=q[:, :3])
    p = ca.page_pool(9, 16)
    for bad, word in ((lambda: ca.cache_grow(p, table, n.long(), n, 5), "lens"), (lambda: ca.cache_grow(p, table, n, n[:1], 5), "new"),
                      (lambda: ca.cache_grow(p, table[0], n, n, 5), "page_table"), (lambda: ca.cache_release(p, table.t(), n), "lens|contig"),
                      (lambda: ca.cache_write(q, q, kp, vp, torch.zeros(40, dtype=torch.int64, device="cuda")), "k: expected"),
                      (lambda: ca.cache_write(q[:, :2], q[:, :2], kp, vp, torch.zeros(40, dtype=torch.int32, device="cuda")), "slots")):
        with pytest.raises(ValueError, match=word):
            bad()
    with pytest.raises(ca.CAError, match="table_stride"):  # rows that overlap
        ca.cache_grow(p, table[:1].expand(2, table.shape[1]), n, n, 5)


@pytest.mark.parametrize("dt", DT)
def test_chunk_given_outputs_count_as_changed(dt):
    import torch
    ca = _ca()
    lens = [40]
    kp, vp, table, _ = _pages(_gen(52), dt, lens, 16, 2, 64)
    kp, vp = torch.nan_to_num(kp), torch.nan_to_num(vp)
    q, n, starts = _rand(_gen(53), (5, 4, 64), dt).cuda(), _i32(lens), _i32([0, 5])
    out, lse = torch.zeros_like(q), torch.zeros(5, 4, device="cuda")
    pool = ca.page_pool(4, 16)
    k = _rand(_gen(54), (5, 2, 64), dt).cuda()
    slots = torch.arange(5, device="cuda")
    for call, written in ((lambda: ca.paged_chunk_attn(ca.Window(), q, kp, vp, table, n, starts, out=out, lse=lse), (out, lse)),
                          (lambda: ca.cache_write(k, k, kp, vp, slots), (kp, vp)),
                          (lambda: ca.cache_grow(pool, table, n, n, 40), (table, pool.state)),
                          (lambda: ca.cache_release(pool, table, n), (table, pool.state, pool.free))):
        before = [t._version for t in written]
        call()
        assert all(t._version > v for t, v in zip(written, before))
    for x in (q.clone().requires_grad_(),):
        with pytest.warns(UserWarning, match="not recorded"):
            got, _ = ca.paged_chunk_attn(ca.Window(), x, kp, vp, table, n, starts)
        assert not got.requires_grad


def test_numbers_given_as_tensors_are_read_anew_by_chunks():
    import torch
    ca = _ca()
    lens = [90]
    kp, vp, table, _ = _pages(_gen(55), "bf16", lens, 16, 2, 64)
    q, n, starts = _rand(_gen(56), (30, 4, 64), "bf16").cuda(), _i32(lens), _i32([0, 30])
    scale, left, tokens = torch.tensor(0.25), torch.tensor(3), torch.tensor(20)
    for s, m, t in ((0.25, 3, 20), (0.5, 9, 33)):
        scale.fill_(s)
        left.fill_(m)
        tokens.fill_(t)
        a = ca.paged_chunk_attn(ca.Window(left=left), q, kp, vp, table, n, starts, scale=scale)[0]
        assert torch.equal(a, ca.paged_chunk_attn(ca.Window(left=m), q, kp, vp, table, n, starts, scale=s)[0])
        pool, rows = ca.page_pool(20, 16), torch.full((1, 6), -1, dtype=torch.int32, device="cuda")
        assert ca.cache_grow(pool, rows, n, _i32([20]), tokens).slots.shape[0] == t
        ca.cache_release(pool, rows, n, left=left)
        assert int((rows >= 0).sum()) == 1 + (m > 10)


# ---- how the work is divided -----------------------------------------------------------------------

def _divided(dt, tokens, H, Hk, d, page, pick, wide=0, scale=None, **kw):
    """A call of many blocks: the bounds of some sequences and heads (`pick`), checked on the GPU in 64 bits.
    tokens: (all, new) of each sequence; wide: tokens that the table has room for."""
    import torch
    ca = _ca()
    g = torch.Generator(device="cuda")
    g.manual_seed(len(tokens) + H)
    lens, new = [a for a, _ in tokens], [n for _, n in tokens]
    need = [-(-n // page) for n in lens]
    width = max(max(need), -(-wide // page))
    pool = sum(need) + 1
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = np.cumsum([0] + need)
    for b, n in enumerate(need):
        table[b, :n] = order[at[b]:at[b + 1]]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=_torch(dt))  # noqa: E731
    kp, vp = rnd(pool, page, Hk, d), rnd(pool, page, Hk, d)
    starts = np.cumsum([0] + new).tolist()
    q = rnd(starts[-1], H, d)
    args = ca.Window(**kw), q, kp, vp, table, _i32(lens), _i32(starts)
    out, lse = ca.paged_chunk_attn(*args, scale=scale, want_lse=True)
    # again, into tensors and a workspace of NaN: nothing is left out, nothing read that was not written
    again = torch.full_like(out, math.nan), torch.full_like(lse, math.nan)
    ca.paged_chunk_attn(*args, scale=scale, out=again[0], lse=again[1],
                        ws=torch.full((160 << 20,), 255, dtype=torch.uint8, device="cuda"))
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    assert bool(torch.isfinite(out).all())
    scale = scale or 1.0 / math.sqrt(d)
    u, r = _u(dt), 2.0 ** -8 if dt == "bf16" else 0.0
    for b, h in pick:
        n, a, hk = new[b], lens[b], h // (H // Hk)
        j = torch.arange(a, device="cuda")
        e = table[b, j // page].long()
        k, v = (x[e, j % page, hk].double() for x in (kp, vp))
        x = q[starts[b]:starts[b + 1], h].double()
        p = (torch.arange(n, device="cuda") + a - n)[:, None]
        see = torch.ones(n, a, dtype=torch.bool, device="cuda")
        if kw.get("left", -1) >= 0:
            see &= j >= p - kw["left"]
        if kw.get("right", -1) >= 0:
            see &= j <= p + kw["right"]
        see |= (j < kw.get("sinks", 0))[None]
        if kw.get("causal"):
            see &= j <= p
        s = torch.where(see, x @ k.T * scale, -math.inf)
        want_lse = torch.logsumexp(s, 1)
        P = torch.exp(s - want_lse[:, None])
        o, A = P @ v, P @ v.abs()
        w = 2 * (d + 8) * 2.0 ** -24 * scale * (x.abs() @ k.abs().T).max() + 2.0 ** -20
        got, gl = out[starts[b]:starts[b + 1], h].double(), lse[starts[b]:starts[b + 1], h].double()
        assert ((got - o).abs() <= u * o.abs() + (r + w) * A).all(), f"sequence {b} head {h}"
        assert ((gl - want_lse).abs() <= 2 * w + 2.0 ** -23 * want_lse.abs()).all(), f"lse of sequence {b} head {h}"


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("H,Hk", [(4, 1), (2, 2), (3, 3), (8, 4), (5, 5), (6, 6), (16, 8), (12, 12), (20, 20)])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_shares_over_every_number_of_heads(dt, H, Hk, d):
    """Key heads that the XCDs take alone, in twos, fours or together; blocks that are cut."""
    tokens = [(3000, 200), (2500, 1), (1700, 333), (1, 1), (4100, 77)]
    _divided(dt, tokens, H, Hk, d, 32, [(0, 0), (1, H - 1), (2, H // 2), (3, 0), (4, H - 1)], causal=True)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("kw", [dict(), dict(left=1500, sinks=300), dict(causal=True)])
def test_chunk_whole_rounds_and_shares(dt, kw):
    """A little more than one, two and three rounds of blocks: whole ones first, the rest in shares."""
    for H, n in ((40, 700 if dt == "f32" else 1560), (40, 2 * 1560), (16, 900)):
        _divided(dt, [(2000 + n, n)], H, H, 128, 32, [(0, 0), (0, H // 2 + 1), (0, H - 1)], **kw)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("d,held", [(128, 64), (64, 96)])
@pytest.mark.parametrize("rounds,extra", [(1, 1), (1, 2), (1, 9), (2, 1), (2, 3), (3, 5)])
def test_chunk_whole_rounds_and_a_few_blocks(dt, d, held, rounds, extra):
    """`held` blocks of a key head run at a time: some rounds of them, and a few blocks more, of one length and of two."""
    n, rows = rounds * held + extra, 128 if dt == "bf16" else 64
    for lens, kw in (([2000] * n, dict()), ([2000 + 100 * (b % 2) for b in range(n)], dict(causal=True))):
        _divided(dt, [(a, rows) for a in lens], 8, 8, d, 32, [(0, 0), (n - 1, 7), (n - 2, 3), (held - 1, 1), (held, 2), (n // 2, 4)],
                 **kw)


@pytest.mark.parametrize("dt", DT)
def test_chunk_many_sequences(dt):
    """More sequences than the planning workgroup takes at a time, with and without new tokens; more than a call
    without a plan has, and as many."""
    r = random.Random(5)
    for B, wide in ((700, 0), (256, 0), (257, 0), (300, 5000)):
        tokens = [(a, min(a, r.choice((0, 1, 1, 2, 40)))) for a in (r.randrange(0, 300) for _ in range(B))]
        tokens[3] = (2000, 17) if wide else tokens[3]
        tokens[-1] = (250, 60)
        _divided(dt, tokens, 4, 2, 64, 16, [(3, 1), (B - 1, 3)] + [(b, 0) for b in range(0, B, 61) if tokens[b][1]],
                 wide=wide, causal=True)


@pytest.mark.parametrize("dt", DT)
def test_chunk_more_blocks_than_the_index(dt):
    """Thousands of blocks, of which some are cut."""
    tokens = [(1100, 1000)] * 34 + [(9000, 3)]
    _divided(dt, tokens, 8, 1, 64, 64, [(0, 0), (17, 3), (33, 7), (34, 5)], wide=9500, causal=True)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("page", [8, 16, 24, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_pages_that_end_inside_tiles(dt, page, d):
    _divided(dt, [(1000, 150), (777, 3), (2049, 65)], 4, 2, d, page, [(0, 0), (1, 3), (2, 2)], left=600, sinks=70, causal=True)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("kind", ["tokens the same", "tokens overlapping", "heads the same", "pages the same", "tokens far apart",
                                  "pages far apart"])
def test_chunk_pools_of_any_strides(dt, kind):
    """Strides of 0, strides below a row's length, and offsets past 2^32 bytes on every way to address
    a row give the bits that a dense copy gives; an output may lie where the queries do."""
    import torch
    ca = _ca()
    g, D, P, page, Hk = _gen(60), 64, 5, 16, 2
    shape, unit = (P, page, Hk, D), 128 // torch.finfo(_torch(dt)).bits  # elements of 16 bytes
    strides = {"tokens the same": (Hk * D, 0, D, 1), "tokens overlapping": (page * Hk * D, unit, 4 * D, 1),
               "heads the same": (page * D, D, 0, 1), "pages the same": (0, Hk * D, D, 1),
               "tokens far apart": (Hk * D, (1 << 23) - unit, D, 1), "pages far apart": ((1 << 30) - unit, Hk * D, D, 1)}[kind]
    size = sum((n - 1) * s for n, s in zip(shape, strides)) + 1
    pools = []
    for i in range(2):
        if size > 1 << 24:
            x = torch.empty(size, dtype=_torch(dt), device="cuda").as_strided(shape, strides)
            x.copy_(_rand(g, shape, dt))
        else:
            x = _rand(g, (size,), dt).cuda().as_strided(shape, strides)
        pools.append(x)
    for lens, new in (([70, 33], [40, 2]), ([9, 80], [9, 80])):
        table = _i32([[4, 1, 3, 0, 2], [0, 2, 4, 1, 3]])
        starts = _i32(np.cumsum([0] + new).tolist())
        q = _rand(g, (sum(new), 4, D), dt).cuda()
        for w in (ca.Window(causal=True), ca.Window(left=20, right=5, sinks=3)):
            a, la = ca.paged_chunk_attn(w, q, *pools, table, _i32(lens), starts, want_lse=True)
            b, lb = ca.paged_chunk_attn(w, q, *(x.contiguous() for x in pools), table, _i32(lens), starts, want_lse=True)
            assert torch.equal(a, b) and torch.equal(la, lb)
            c = q.clone()
            ca.paged_chunk_attn(w, c, *pools, table, _i32(lens), starts, out=c)
            assert torch.equal(c, a)


@pytest.mark.parametrize("dt", DT)
def test_chunk_cut_blocks_may_be_written_over_their_queries(dt):
    import torch
    ca = _ca()
    lens, w = [9000, 30, 4000], ca.Window(causal=True)
    kp, vp, table, _ = _pages(_gen(61), dt, lens, 16, 2, 64)
    q = _rand(_gen(62), (240, 4, 64), dt).cuda()
    n, starts = _i32(lens), _i32([0, 10, 40, 240])
    a, _ = ca.paged_chunk_attn(w, q, kp, vp, table, n, starts)
    ca.paged_chunk_attn(w, q, kp, vp, table, n, starts, out=q)
    assert torch.equal(q, a)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("H,Hk", [(200, 1), (300, 2), (257, 1)])
def test_chunk_more_heads_than_a_block_has_rows(dt, H, Hk):
    """A token's query heads fill a block and go on in the next one; alone, and cut into parts."""
    _chunk_check(dt, [(40, 3), (7, 7), (300, 1)], H, Hk, 64, 16, seed=H, causal=True)
    _divided(dt, [(4000, 2), (700, 9)], H, Hk, 64, 16, [(0, 0), (0, 127), (0, H - 1), (1, 64)], causal=True)


@pytest.mark.parametrize("dt", DT)
def test_chunk_sinks_without_end(dt):
    """Windows beside sinks that reach beyond the last key."""
    for sinks in (2 ** 31 - 1, 5000):
        _chunk_check(dt, [(3000, 3), (90, 90), (1, 1)], 2, 1, 64, 16, left=5, sinks=sinks, causal=True)
        _chunk_check(dt, [(300, 3), (90, 90)], 2, 1, 64, 16, left=5, right=2, sinks=sinks)
