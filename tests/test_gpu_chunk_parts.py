"""Attention of chunks where blocks are cut into parts: head dimensions, pages of any size, parts without keys, values and
keys that are not finite, rows before the first sequence, two streams, captured steps. Every call is shown to be cut by
what its plan left in the workspace.

Against 64 bits on the GPU. Tolerances: those of test_gpu_chunk's _divided (logits, probabilities and output rounded), and
for the joining 2^-22 a part: what was added up before is scaled by an exponential (one unit, 2^-23) and a product
(2^-24) for each part that comes, its sum and its results alike."""
import math

import numpy as np
import pytest

from tests.test_gpu_chunk import _i32, _serving, _step
from tests.test_gpu_sequence import DT, _ca, _gen, _rand, _torch, _u

pytestmark = pytest.mark.gpu


class _Call:
    """tokens: (all, new) of each sequence, whose rows begin at row `first`."""

    def __init__(self, dt, tokens, H, Hk, d, page, seed=0, first=0, spare=3):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.dt, self.tokens, self.H, self.Hk, self.d, self.page, self.first = dt, tokens, H, Hk, d, page, first
        need = [-(-a // page) for a, _ in tokens]
        self.pages = sum(need) + 1
        order = torch.randperm(self.pages, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(tokens), max(need)), -1, dtype=torch.int32, device="cuda")
        at = np.cumsum([0] + need)
        for b, n in enumerate(need):
            self.table[b, :n] = order[at[b]:at[b + 1]]
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=_torch(dt))  # noqa: E731
        self.kp, self.vp = rnd(self.pages, page, Hk, d), rnd(self.pages, page, Hk, d)
        self.kp[order[-1]] = self.vp[order[-1]] = math.nan  # nobody's page
        self.starts = np.cumsum([first] + [n for _, n in tokens]).tolist()
        self.q = rnd(self.starts[-1] + spare, H, d)
        self.ws = torch.full((160 << 20,), 255, dtype=torch.uint8, device="cuda")

    def place(self, b, j):
        return int(self.table[b, j // self.page]), j % self.page

    def __call__(self, cut=True, **kw):
        """(out, lse); cut: some block is, checked."""
        import torch
        out = torch.full_like(self.q, 7.0)
        lse = torch.full(self.q.shape[:2], 7.0, device="cuda")
        self.ws.fill_(255)
        args = (_ca().Window(**kw), self.q, self.kp, self.vp, self.table, _i32([a for a, _ in self.tokens]), _i32(self.starts))
        _ca().paged_chunk_attn(*args, out=out, lse=lse, ws=self.ws)
        blocks, _, cuts, whole = self.ws[:16].view(torch.int32).tolist()
        assert not cut or (blocks > 0 and cuts > 0 and whole == 0)
        for x in (out, lse):
            assert bool((x[:self.first] == 7).all()) and bool((x[self.starts[-1]:] == 7).all())
        again = _ca().paged_chunk_attn(*args, want_lse=True)  # same bits, a workspace of its own
        at = slice(self.first, self.starts[-1])
        for x, y in zip((out, lse), again):
            assert torch.equal(x[at].nan_to_num(nan=9e9), y[at].nan_to_num(nan=9e9))
        return out, lse

    def see(self, b, left=-1, right=-1, sinks=0, causal=False):
        """[new, all]: whom the new tokens of sequence b see, and which of the keys are there."""
        import torch
        a, n = self.tokens[b]
        j, p = torch.arange(a, device="cuda"), (torch.arange(n, device="cuda") + a - n)[:, None]
        m = torch.ones(n, a, dtype=torch.bool, device="cuda")
        if left >= 0:
            m &= j >= p - left
        if right >= 0:
            m &= j <= p + right
        m |= (j < sinks)[None]
        if causal:
            m &= j <= p
        e = self.table[b, j // self.page]
        return m & ((e >= 0) & (e < self.pages))[None]

    def check(self, got, b, h, rows=None, **kw):
        """Rows (a mask, all by default) of head h of sequence b against 64 bits."""
        import torch
        out, lse = (x[self.starts[b]:self.starts[b + 1], h].double() for x in got)
        a, n = self.tokens[b]
        j = torch.arange(a, device="cuda")
        e = self.table[b, j // self.page].long()
        e = torch.where((e >= 0) & (e < self.pages), e, 0)
        k, v = (x[e, j % self.page, h // (self.H // self.Hk)].double() for x in (self.kp, self.vp))
        rows = torch.ones(n, dtype=torch.bool, device="cuda") if rows is None else rows
        see = self.see(b, **kw)[rows]
        seen = see.any(0)[:, None]
        k, v = (torch.where(seen, x, 0.0) for x in (k, v))  # (what nobody sees may be NaN)
        x, scale = self.q[self.starts[b]:self.starts[b + 1], h].double()[rows], 1.0 / math.sqrt(self.d)
        s = torch.where(see, x @ k.T * scale, -math.inf)
        want = torch.logsumexp(s, 1)
        P = torch.exp(s - torch.where(want == -math.inf, 0.0, want)[:, None])
        o, A = P @ v, P @ v.abs()
        parts = (a / 64 / 2 + 2) * 2.0 ** -22
        w = 2 * (self.d + 8) * 2.0 ** -24 * scale * (x.abs() @ k.abs().T).max() + 2.0 ** -20 + parts
        r = 2.0 ** -8 if self.dt == "bf16" else 0.0
        assert ((out[rows] - o).abs() <= _u(self.dt) * o.abs() + (r + w) * A).all(), f"sequence {b} head {h}"
        none = want == -math.inf
        assert torch.equal(lse[rows][none], want[none]), f"lse of sequence {b} head {h}"
        assert ((lse[rows] - want)[~none].abs() <= 2 * w + 2.0 ** -23 * want[~none].abs()).all(), f"lse of sequence {b} head {h}"

    def check_all(self, got, **kw):
        for b, (_, n) in enumerate(self.tokens):
            for h in sorted({0, self.H // 2, self.H - 1}):
                if n:
                    self.check(got, b, h, **kw)


# one block in 7 parts and in about 25; blocks of prompts beside single tokens
_CUT = ([(1600, 2)], [(6000, 3)], [(3000, 200), (2500, 1), (1700, 333)])


@pytest.mark.parametrize("tokens", _CUT)
@pytest.mark.parametrize("d", [4, 20, 32, 36, 96, 100, 128])
def test_parts_f32_head_dims(d, tokens):
    c = _Call("f32", tokens, 4, 2, d, 16, seed=d)
    for kw in (dict(causal=True), dict(left=1550, sinks=70, causal=True)):
        c.check_all(c(**kw), **kw)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("page", [1, 3, 7, 8, 24, 40, 100])
@pytest.mark.parametrize("d", [64, 128])
def test_parts_pages_of_any_size(dt, page, d):
    """Tiles whose rows lie on many pages, walked from somewhere inside the cache."""
    for tokens in _CUT:
        c = _Call(dt, tokens, 2, 1, d, page, seed=page, first=5)
        c.check_all(c(causal=True), causal=True)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("page", [7, 16, 24, 64, 100])
@pytest.mark.parametrize("gone", [(0, 3000), (1500, 4500), (3000, 6000), (64, 5990), (0, 6000)])
def test_parts_without_keys(dt, page, gone):
    """Entries outside the pool over several parts: at the beginning, inside, at the end, all but a few, all."""
    import torch
    c = _Call(dt, [(6000, 3), (4000, 40)], 2, 1, 64, page, seed=1)
    bad = torch.tensor([-1, c.pages, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    i = torch.arange(-(-gone[0] // page), -(-gone[1] // page), device="cuda")
    c.table[0, i] = bad[i % 4]
    for kw in (dict(causal=True), dict(), dict(left=5000, sinks=200, causal=True)):
        got = c(**kw)
        c.check_all(got, **kw)
        if gone == (0, 6000):
            assert not got[0][:3].any() and bool((got[1][:3] == -math.inf).all())


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("page", [7, 16, 24])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", ["v", "k"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_parts_values_that_are_not_finite(dt, page, d, where, value):
    """A key or a value in one part, seen by all rows, by some, by none: rows that do not see it are what they are without
    it, those that do are not finite."""
    import torch
    for at, kw in ((100, dict(causal=True)), (4950, dict(causal=True)), (3200, dict(left=1700, sinks=5, causal=True)),
                   (2000, dict(left=2900, right=20)), (1000, dict(left=2000, sinks=300))):
        c = _Call(dt, [(5000, 130), (4000, 1)], 2, 1, d, page, seed=at)
        pool = c.vp if where == "v" else c.kp
        e, i = c.place(0, at)
        pool[e, i] = value
        got = c(**kw)
        sees = c.see(0, **kw)[:, at]
        if at in (4950, 3200):
            assert bool(sees.any()) and not bool(sees.all())
        for h in range(2):
            if not bool(sees.all()):
                c.check(got, 0, h, rows=~sees, **kw)
            c.check(got, 1, h, **kw)
            out, lse = (x[c.starts[0]:c.starts[1], h][sees] for x in got)
            assert not bool(torch.isfinite(out).any())
            assert bool(torch.isfinite(lse).all()) if where == "v" else not bool(torch.isfinite(lse).any())


@pytest.mark.parametrize("dt", DT)
def test_parts_and_rows_that_see_nothing(dt):
    """More new tokens than tokens, and sequences without either, in a call that is cut."""
    c = _Call(dt, [(20, 50), (5000, 3), (0, 0), (0, 9), (130, 1)], 4, 2, 64, 16, first=2)
    for kw in (dict(causal=True), dict(left=3, right=4), dict(sinks=2, left=1, causal=True)):
        got = c(cut=kw.get("left", -1) < 0, **kw)
        assert not got[0][c.starts[3]:c.starts[4]].any() and bool((got[1][c.starts[3]:c.starts[4]] == -math.inf).all())
        for b in (0, 1, 4):
            for h in (0, 3):
                c.check(got, b, h, **kw)


@pytest.mark.parametrize("dt", DT)
@pytest.mark.parametrize("tokens,cut", [([(100, 9), (40, 40)], False), ([(70, 1)] * 300, False), ([(4000, 2), (300, 300)], True)])
def test_rows_before_the_first_sequence(dt, tokens, cut):
    """Without a plan, with whole blocks, with blocks that are cut."""
    for first in (1, 64, 1000):
        c = _Call(dt, tokens, 2, 2, 64, 16, seed=first, first=first)
        got = c(cut=cut, causal=True)
        for b in {0, len(tokens) // 2, len(tokens) - 1}:
            c.check(got, b, 1, causal=True)


@pytest.mark.parametrize("dt", DT)
def test_parts_on_two_streams_at_once(dt):
    import torch
    ca, calls = _ca(), [_Call(dt, [(9000 + 700 * i, 5), (40, 4), (5000, 90 + i)], 4, 2, 64, 16, seed=i) for i in range(2)]
    args, want = [], []
    for c in calls:
        out, lse = c(causal=True)
        want.append((out[:c.starts[-1]], lse[:c.starts[-1]]))
        args.append((ca.Window(causal=True), c.q, c.kp, c.vp, c.table, _i32([a for a, _ in c.tokens]), _i32(c.starts)))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(ca.paged_chunk_attn(*args[i], want_lse=True))
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i]:
            assert all(torch.equal(a, b[:len(a)]) for a, b in zip(want[i], x))


@pytest.mark.parametrize("dt", DT)
def test_parts_in_captured_steps(dt):
    """Steps on long caches, captured and replayed for other lengths, with eager work and synchronizations between; two
    graphs share one workspace, and each replay leaves a plan of cut blocks."""
    import torch
    ca, w, page, width, T = _ca(), _ca().Window(causal=True), 16, 400, 60
    sets = [_serving(dt, w, page, 1200, 3, width, T) for _ in range(4)]  # two captured, two eager
    ws = torch.full((160 << 20,), 255, dtype=torch.uint8, device="cuda")
    for i, s in enumerate(sets):  # caches of some thousand tokens
        g = torch.Generator(device="cuda")
        g.manual_seed(i % 2)
        for x in (s["kp"], s["vp"]):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        s["lens"].copy_(_i32([5000, 0, 3100]))
        s["new"].copy_(s["lens"])
        ca.cache_grow(s["pool"], s["table"], s["lens"], s["new"], 8100)
        s["new"].zero_()

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
    lens = [5000, 0, 3100]
    for i, new in enumerate(([1, 20, 39], [1, 1, 1], [50, 1, 1], [3, 0, 7], [1, 58, 1])):
        lens = [a + n for a, n in zip(lens, new)]
        for x in range(2):
            fill(sets[x], 10 * i + x, lens, new)
            fill(sets[2 + x], 10 * i + x, lens, new)
        ws.fill_(255)
        for x in ((0, 1), (1, 0))[i % 2]:
            graphs[x].replay()
        want = [_step(ca, sets[2 + x]) for x in range(2)]
        torch.cuda.synchronize()
        blocks, _, cuts, whole = ws[:16].view(torch.int32).tolist()
        assert blocks > 0 and cuts > 0 and whole == 0
        m = sum(new)
        for x in range(2):
            out, lse, plan = held[x]
            assert torch.equal(out[:m], want[x][0][:m]) and torch.equal(lse[:m], want[x][1][:m])
            assert all(torch.equal(a, b) for a, b in zip(plan, want[x][2]))
            for name in ("table", "kp", "vp"):
                assert torch.equal(sets[x][name], sets[2 + x][name])
