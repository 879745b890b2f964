"""The operators of a paged cache that takes chunks of new tokens, as cases that can be timed and compared: the page table
and the slot map built on the GPU from the sequences' lengths, new keys and values written by that map, the attention of
the chunks over the cache, and a serving step that runs them together.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges, ``prepare(case, seed)`` makes what a user's
program has in hand, ``run(state)`` is one pass: the framework's calls where ``own`` is true, else the same operators in
plain torch. ``work(case)`` is what a pass cannot do without, ``exact(case, seed)`` its result in 64 bits.

The new tokens of all sequences lie packed, one sequence after the other: those of sequence b are rows starts[b] ..
starts[b + 1] - 1. lens[b] counts a sequence's tokens, the new ones (its last) included.

Kinds of cases ("kind"):

* ``pages``  ``cache_grow`` (pages for the new tokens, starts, slots, positions), then ``cache_release`` back to the
             lengths before, so that a pass ends where it began.
* ``write``  ``cache_write`` of packed keys and values to their slots.
* ``chunk``  ``paged_chunk_attn``: every sequence's new tokens against its pages.
* ``step``   ``cache_grow``, ``rope`` of the packed queries and keys, ``cache_write``, ``paged_chunk_attn``.

Lengths come from the case alone ("spread"): ``even`` (all sequences alike), ``ragged`` (over the logarithm of the range,
one in four without a cache), ``mixed`` (three of four sequences have one new token and a cache, the others are prompts).
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BASE = dict(kind="chunk", dtype="bf16", batch=1, heads=8, heads_k=8, d=64, page=16, cached=1024, new=16, spread="even",
             lens_seed=0, left=-1, right=-1, sinks=0, causal=True, spare=0)


def _case(name, **kw):
    c = dict(_BASE, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # One new token each of 256 sequences in tables for 32,768 tokens: the smallest call, once a step.
        _case("pages_decode", kind="pages", batch=256, cached=32767, new=1, spread="ragged", lens_seed=1),
        # 64 requests, some continued, some fresh, with up to 4,096 new tokens each.
        _case("pages_prompts", kind="pages", batch=64, cached=8192, new=4096, page=32, spread="ragged", lens_seed=2),
        # The new tokens of 64 sequences, two heads of 64: latency.
        _case("write_decode", kind="write", batch=64, heads_k=2, cached=4000, new=1),
        # The keys and values of a 480p video layer's 32,760 tokens, written in one go. All memory traffic.
        _case("write_video", kind="write", batch=1, heads_k=40, d=128, cached=0, new=32760, page=64),
        # A streamed video model's new frame of 1,560 tokens, all of which see each other, three frames before them and
        # the first one; two streams.
        _case("chunk_frame", batch=2, heads=40, heads_k=40, d=128, page=32, cached=9360, new=1560, left=4679, sinks=1560,
              causal=False),
        # A long prompt's second part: 8,192 new tokens on 24,576 cached ones, four query heads to a key head.
        _case("chunk_prompt", heads=32, heads_k=8, d=128, page=64, cached=24576, new=8192),
        # Eighteen sequences that go on by a token each, beside six prompts of up to 2,000; five query heads to a key head.
        _case("chunk_mixed", batch=24, heads=40, heads_k=8, d=128, cached=32768, new=2000, spread="mixed", lens_seed=3),
        # Five drafted tokens of eight sequences, to be checked against up to 16,000 cached ones.
        _case("chunk_draft", batch=8, heads=16, heads_k=4, cached=16000, new=5, spread="ragged", lens_seed=4),
        # Sixteen new rows against a cached table of 262,144 rows that they see whole, 16 heads: the split over the cache.
        _case("chunk_table", heads=16, heads_k=16, page=64, cached=262128, new=16, causal=False),
        # fp32, four ragged sequences, windows and sinks, odd page size.
        _case("chunk_f32", dtype="f32", batch=4, heads=8, heads_k=4, page=48, cached=4099, new=701, spread="ragged",
              lens_seed=5, left=1500, sinks=4),
        # The smallest step: four sequences, three of them by one token, a short prompt, in arrays with room for more.
        _case("step_small", kind="step", batch=4, heads_k=2, cached=500, new=33, spread="mixed", lens_seed=6, spare=28),
        # A step of 32 sequences, prompts of up to 1,024 among them, shared key heads, a window and sinks.
        _case("step_mixed", kind="step", batch=32, heads=24, heads_k=8, d=128, page=32, cached=6000, new=1024,
              spread="mixed", lens_seed=7, left=4095, sinks=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the logarithm of the listed range, odd ones among them, never over the largest."""
    kind = rng.choice(("pages", "pages", "write", "chunk", "chunk", "chunk", "chunk", "step"))
    spread = rng.choice(("even", "ragged", "mixed"))
    page = rng.choice((1, 7, 16, 16, 32, 48, 64, 100, 128, 256))
    seed = rng.randrange(1000)
    if kind == "pages":
        batch, cached, new = _log(rng, 1, 512), _log(rng, 1, 32768), _log(rng, 1, 4096)
        while batch * (cached + new) // page > 1 << 18 or batch * new > 1 << 18:
            batch, cached = max(1, batch * 2 // 3), max(1, cached * 2 // 3)
            new = max(1, new * 2 // 3)
        left = rng.choice((-1, -1, _log(rng, 1, 8192)))
        return _case(None, kind=kind, batch=batch, cached=cached, new=new, page=page, spread=spread, lens_seed=seed,
                     left=left, sinks=rng.choice((0, 4, 100)) if left >= 0 else 0, spare=rng.choice((0, 0, 1, 300)))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    heads_k = rng.choice((1, 2, 3, 4, 8))
    heads = heads_k * rng.choice((1, 1, 2, 3, 4, 5, 8))
    d = rng.choice((64, 128)) if dtype == "bf16" else rng.choice((20, 32, 64, 96, 128))
    if kind == "write":
        batch, new = rng.choice((1, 2, 7, 32, 64)), _log(rng, 1, 32768)
        while batch * new * heads_k * d > 32760 * 40 * 128:
            new = max(1, new // 2)
        return _case(None, kind=kind, dtype=dtype, batch=batch, heads_k=heads_k, d=d, page=page, new=new,
                     cached=_log(rng, 1, 4096), spread=spread, lens_seed=seed, spare=rng.choice((0, 0, 5, 100)))
    batch, cached, new = rng.choice((1, 2, 4, 7, 24, 32)), _log(rng, 1, 65536), _log(rng, 1, 8192)
    left = rng.choice((-1, -1, _log(rng, 1, 8192)))
    causal = kind == "step" or rng.random() < 0.7
    right = -1 if causal else rng.choice((-1, _log(rng, 1, 4096)))
    c = _case(None, kind=kind, dtype=dtype, batch=batch, heads=heads, heads_k=heads_k, d=d, page=page, cached=cached,
              new=new, spread=spread, lens_seed=seed, left=left, right=right, causal=causal,
              sinks=rng.choice((0, 0, 4, 100, 1560)) if left >= 0 else 0, spare=rng.choice((0, 0, 0, 17)))
    cap = 1e11 if dtype == "f32" else 2e12 if kind == "chunk" else 2e11
    while work(c)["flops"] > cap or batch * (c["cached"] + c["new"]) * heads_k * d > 1 << 28:
        c["cached"], c["new"] = max(1, c["cached"] * 2 // 3), max(1, c["new"] * 2 // 3)
    return c


def _tokens(c):
    """(cached, new) of each sequence, from the case alone."""
    if c["spread"] == "even":
        return [(c["cached"], c["new"])] * c["batch"]
    r = random.Random(1000 * c["lens_seed"] + c["batch"])
    some = lambda n: _log(r, max(1, n // 64), n) if n else 0  # noqa: E731
    if c["spread"] == "mixed":
        got = [(0, max(1, _log(r, max(1, c["new"] // 8), c["new"]))) if b % 4 == 3 else (some(c["cached"]), 1)
               for b in range(c["batch"])]
    else:
        got = [(0 if r.random() < 0.25 and c["new"] > 1 else some(c["cached"]), _log(r, 1, c["new"]))
               for _ in range(c["batch"])]
    got[0] = (c["cached"], 1 if c["spread"] == "mixed" else c["new"])
    return got


def _seen(c, cached, new):
    """(visible pairs of a query and a key, keys that some query sees) of one sequence and head. Query i sits at
    p = cached + i and sees key j where j < sinks or p - left <= j <= p + right, and j <= p in causal attention."""
    nk = cached + new
    p = torch.arange(new, dtype=torch.int64) + cached
    hi = torch.full_like(p, nk - 1) if c["right"] < 0 else (p + c["right"]).clamp(max=nk - 1)
    lo = torch.zeros_like(p) if c["left"] < 0 else (p - c["left"]).clamp(min=0)
    top = torch.full_like(p, nk - 1)
    if c["causal"]:
        hi, top = torch.minimum(hi, p), p
    sink = torch.minimum(top + 1, torch.tensor(c["sinks"]))
    pairs = int((sink + (hi + 1 - torch.maximum(lo, sink)).clamp(min=0)).sum())
    most = int(sink[-1])
    return pairs, most + max(0, int(hi[-1]) + 1 - max(int(lo[0]), most))


def _touched(c):
    """Pages that the new tokens lie on, over all sequences."""
    return sum(-(-(a + n) // c["page"]) - a // c["page"] for a, n in _tokens(c))


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    tokens = _tokens(c)
    T = sum(n for _, n in tokens)
    if c["kind"] == "pages":
        # lengths, starts, a slot of eight bytes and a position of four for each token and spare place; a page that
        # comes and goes is read from the free list and written to the table, and back again
        return {"bytes": 16 * c["batch"] + 12 * (T + c["spare"]) + 16 * _touched(c), "flops": 0}
    new = T * c["heads_k"] * c["d"]
    if c["kind"] == "write":
        return {"bytes": 4 * new * e + 8 * (T + c["spare"]), "flops": 0}
    pairs, keys = map(sum, zip(*(_seen(c, a, n) for a, n in tokens)))
    q = T * c["heads"] * c["d"]
    w = {"bytes": (2 * q + 2 * keys * c["heads_k"] * c["d"]) * e, "flops": 4 * pairs * c["heads"] * c["d"]}
    if c["kind"] == "step":  # queries and keys turned, keys and values written
        w["bytes"] += (2 * q + 6 * new) * e + 12 * T
    else:
        w["bytes"] += 4 * T * c["heads"]
    return w


# ---- inputs ----------------------------------------------------------------------------------------------------

class _State:
    """What a user's program has in hand before the call."""


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _mixture(g, centres, *shape):
    at = torch.randint(0, centres.shape[0], shape, generator=g, device="cuda")
    return centres[at].add_(torch.randn(*shape, centres.shape[1], generator=g, device="cuda"), alpha=0.6)


def _int32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _kept_pages(c, n):
    """Which pages a sequence of n tokens holds: those with a token that its next one sees."""
    i = torch.arange(-(-n // c["page"]))
    if c["left"] < 0:
        return i
    return i[(i * c["page"] < c["sinks"]) | (((i + 1) * c["page"]).clamp(max=n) - 1 >= n - c["left"])]


def prepare(case, seed):
    c, s = case, _State()
    s.case = c
    g = _gen(seed)
    dt = _DT[c["dtype"]]
    B, page = c["batch"], c["page"]
    tokens = _tokens(c)
    s.host_lens, s.host_new = [a + n for a, n in tokens], [n for _, n in tokens]
    s.host_starts = [sum(s.host_new[:b]) for b in range(B + 1)]
    s.lens, s.new, s.starts = _int32(s.host_lens), _int32(s.host_new), _int32(s.host_starts)
    s.T = s.host_starts[-1] + c["spare"]
    s.left, s.right, s.sinks, s.causal, s.page = c["left"], c["right"], c["sinks"], c["causal"], page

    # the table: pages of the pool in random order, those of the cached tokens ("pages", "step") or of all
    need = [-(-n // page) for n in s.host_lens]
    s.pages = sum(need) + 3
    order = torch.randperm(s.pages, generator=g, device="cuda").to(torch.int32)
    grows = c["kind"] in ("pages", "step")
    host = torch.full((B, max(need) + 3), -1, dtype=torch.int64)
    at = 0
    for b in range(B):
        hold = _kept_pages(c, tokens[b][0]) if grows else torch.arange(need[b])
        host[b, hold] = torch.arange(at, at + len(hold))
        at += len(hold)
    host = host.cuda()
    s.table = torch.where(host >= 0, order[host.clamp(min=0)], -1).to(torch.int32)
    if grows:
        s.before = _int32([a for a, _ in tokens])
        s.free = torch.zeros(s.pages, dtype=torch.int32, device="cuda")
        s.free[:s.pages - at] = order[at:]
        s.state = _int32([s.pages - at, 0, 0])
        if own:
            import paper_2608_26965_amd as ca
            s.pool = ca.PagePool(page=page, free=s.free, state=s.state)
    if c["kind"] == "pages":
        return s

    H, Hk, d, T = c["heads"], c["heads_k"], c["d"], s.T
    centres = torch.randn(64, d, generator=g, device="cuda").mul_(0.8)
    s.k_pages = torch.empty(s.pages, page, Hk, d, dtype=dt, device="cuda")
    for lo in range(0, s.pages, max(1, (1 << 26) // (page * Hk * d))):  # drawn in fp32, some pages at a time
        part = s.k_pages[lo:lo + max(1, (1 << 26) // (page * Hk * d))]
        part.copy_(_mixture(g, centres, *part.shape[:3]))
    s.v_pages = torch.randn(s.pages, page, Hk, d, generator=g, device="cuda", dtype=dt)
    if c["kind"] in ("write", "step"):
        s.k, s.v = (torch.randn(T, Hk, d, generator=g, device="cuda", dtype=dt) for _ in range(2))
    if c["kind"] == "write":
        parts = [torch.arange(n - m, n) for n, m in zip(s.host_lens, s.host_new)]
        pos, seq = torch.cat(parts).cuda(), torch.repeat_interleave(torch.arange(B), torch.tensor(s.host_new)).cuda()
        s.slots = torch.full((T,), -1, dtype=torch.int64, device="cuda")
        s.slots[:len(pos)] = s.table[seq, pos // page].long() * page + pos % page
        return s
    s.q = _mixture(g, centres, T, H).to(dt)
    s.out, s.lse = torch.zeros_like(s.q), torch.full((T, H), -math.inf, device="cuda")
    if own:
        import paper_2608_26965_amd as ca
        s.window = ca.Window(left=s.left, right=s.right, sinks=s.sinks, causal=s.causal)
    if c["kind"] == "step":
        s.freqs = [10000.0 ** (-2.0 * i / d) for i in range(d // 2 // 8 * 8)]
        if own:
            s.rope = ca.Rope(sections=(len(s.freqs),), freqs=tuple(s.freqs), pairing="halves")
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------

def _plain_grow(s):
    """Pages of the free list's end to the entries that the new tokens need and that hold none, by row and column."""
    lens, new, n = s.lens.long(), s.new.long(), s.state[0].long()
    col = torch.arange(s.table.shape[1], device="cuda")
    first, end = (lens - new) // s.page, (lens + s.page - 1) // s.page
    lack = (col >= first[:, None]) & (col < end[:, None]) & (new > 0)[:, None] & ((s.table < 0) | (s.table >= s.pages))
    rank = lack.flatten().cumsum(0)
    at = n - rank.reshape(lack.shape)
    s.table.copy_(torch.where(lack & (at >= 0), s.free[at.clamp(min=0)], s.table))
    total = new.sum()
    starts = torch.cat((torch.zeros_like(lens[:1]), new.cumsum(0)))
    s.state.copy_(torch.stack(((n - rank[-1]).clamp(min=0), (rank[-1] - n).clamp(min=0), (total - s.T).clamp(min=0))))
    t = torch.arange(s.T, device="cuda")
    seq = torch.searchsorted(starts[1:], t, right=True).clamp(max=len(lens) - 1)
    pos = torch.where(t < total, lens[seq] - new[seq] + t - starts[seq], 0)
    entry = s.table[seq, pos // s.page].long()
    there = (t < total) & (entry >= 0) & (entry < s.pages)
    slots = torch.where(there, entry * s.page + pos % s.page, -1)
    return starts.clamp(max=s.T).to(torch.int32), slots, pos.to(torch.int32)


def _plain_release(s, lens):
    """Pages without a token that the next one sees go to the free list's end, the first on top."""
    n, left = lens.long()[:, None], s.left
    first = torch.arange(s.table.shape[1], device="cuda") * s.page
    last = torch.minimum(first + s.page, n) - 1
    keep = first < n
    if left >= 0:
        keep &= (first < s.sinks) | (last >= n - left)
    gone = (~keep & (s.table >= 0) & (s.table < s.pages)).flatten()
    rank = gone.cumsum(0)
    at = torch.where(gone, s.state[0] + rank[-1] - rank, s.pages)
    room = torch.cat((s.free, s.free[:1])).scatter(0, at, s.table.flatten())
    s.free.copy_(room[:-1])
    s.table.masked_fill_(gone.reshape(s.table.shape), -1)
    s.state[0] += rank[-1]


def _plain_write(s, k, slots):
    n = s.host_starts[-1]  # the spare places have no slots
    s.k_pages.flatten(0, 1)[slots[:n]] = k[:n]
    s.v_pages.flatten(0, 1)[slots[:n]] = s.v[:n]


def _plain_rope(s, x, positions):
    angle = positions.double()[:, None] * torch.tensor(s.freqs, dtype=torch.float64, device="cuda")
    cos, sin, m = angle.cos().float()[:, None], angle.sin().float()[:, None], len(s.freqs)
    f = x.float()
    a, b = f[..., :m], f[..., m:2 * m]
    return torch.cat((a * cos - b * sin, a * sin + b * cos, f[..., 2 * m:]), -1).to(x.dtype)


def _visible(s, p, j, lens):
    """Which keys j [m] the positions p [B, n] see, [B, n, m]."""
    j, p, lens = j[None, None], p[..., None], lens[:, None, None]
    see = torch.ones_like(p + j, dtype=torch.bool)
    if s.left >= 0:
        see &= j >= p - s.left
    if s.right >= 0:
        see &= j <= p + s.right
    see |= j < s.sinks
    if s.causal:
        see &= j <= p
    return see & (j < lens)


def _some(s, q, seqs, most_new, most_len):
    """Attention of the sequences `seqs` in one padded batch of most_new queries and most_len keys. A block of queries'
    logits are all that is held of the large matrix."""
    H, d = q.shape[1:]
    Hk, G, B = s.k_pages.shape[2], H // s.k_pages.shape[2], len(seqs)
    lens, new, start = (x[seqs].long() for x in (s.lens, s.new, s.starts))
    entries = s.table[seqs, :-(-most_len // s.page)].clamp(min=0).long()
    k, v = (x[entries].flatten(1, 2)[:, :most_len].float().transpose(1, 2) for x in (s.k_pages, s.v_pages))
    j = torch.arange(most_len, device="cuda")
    rows = max(16, min(most_new, int(1.5e9 / (B * H * most_len))))
    for i0 in range(0, most_new, rows):
        i = torch.arange(i0, min(most_new, i0 + rows), device="cuda")
        n = len(i)
        real = i < new[:, None]
        at = torch.where(real, start[:, None] + i, start[:, None])
        x = q[at].float().reshape(B, n, Hk, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hk, G * n, d)
        logit = torch.matmul(x, k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
        see = _visible(s, lens[:, None] - new[:, None] + i, j, lens)
        logit = logit.reshape(B, Hk, G, n, most_len).masked_fill_(~see[:, None, None], -math.inf)
        top = logit.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        prob = logit.sub_(top).exp_()
        total = prob.sum(-1, keepdim=True)
        o = torch.matmul(prob.reshape(B, Hk, G * n, most_len), v).reshape(B, Hk, G, n, d)
        o = (o / torch.where(total > 0, total, torch.ones_like(total))).permute(0, 3, 1, 2, 4).reshape(B, n, H, d)
        lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(B, n, H)
        if B > 1:  # without the rows that fill up the batch
            at, o, lse = at[real], o[real], lse[real]
        s.out[at] = o.to(q.dtype)
        s.lse[at] = lse


def _plain_chunk(s, q):
    """All sequences in one padded batch where that is not much larger, else one after the other."""
    most_new, most_len, B = max(s.host_new), max(s.host_lens), len(s.host_lens)
    each = sum(n * k for n, k in zip(s.host_new, s.host_lens))
    if B * most_new * most_len <= 3 * each and B * most_len * s.k_pages[0, 0].numel() < 1 << 29:
        _some(s, q, torch.arange(B, device="cuda"), most_new, most_len)
    else:
        for b in range(B):
            _some(s, q, torch.arange(b, b + 1, device="cuda"), s.host_new[b], s.host_lens[b])
    return {"out": s.out, "lse": s.lse}


# ---- one pass --------------------------------------------------------------------------------------------------

def run(s):
    kind = s.case["kind"]
    if not own:
        if kind == "pages":
            starts, slots, positions = _plain_grow(s)
            _plain_release(s, s.before)
            return {"starts": starts, "slots": slots, "positions": positions, "table": s.table, "free": s.free, "state": s.state}
        if kind == "write":
            _plain_write(s, s.k, s.slots)
            return {"k_pages": s.k_pages, "v_pages": s.v_pages}
        if kind == "chunk":
            return _plain_chunk(s, s.q)
        starts, slots, positions = _plain_grow(s)
        q, k = _plain_rope(s, s.q, positions), _plain_rope(s, s.k, positions)
        _plain_write(s, k, slots)
        return {"out": _plain_chunk(s, q)["out"], "slots": slots, "table": s.table, "k_pages": s.k_pages, "v_pages": s.v_pages}
    import paper_2608_26965_amd as ca
    if kind == "pages":
        plan = ca.cache_grow(s.pool, s.table, s.lens, s.new, s.T)
        ca.cache_release(s.pool, s.table, s.before, left=s.left, sinks=s.sinks)
        return {"starts": plan.starts, "slots": plan.slots, "positions": plan.positions[0], "table": s.table, "free": s.free,
                "state": s.state}
    if kind == "write":
        ca.cache_write(s.k, s.v, s.k_pages, s.v_pages, s.slots)
        return {"k_pages": s.k_pages, "v_pages": s.v_pages}
    if kind == "chunk":
        # (with spare rows, which the call leaves alone, the outputs are the program's own)
        given = dict(out=s.out, lse=s.lse) if s.case["spare"] else dict(want_lse=True)
        out, lse = ca.paged_chunk_attn(s.window, s.q, s.k_pages, s.v_pages, s.table, s.lens, s.starts, **given)
        return {"out": out, "lse": lse}
    plan = ca.cache_grow(s.pool, s.table, s.lens, s.new, s.T)
    q, k = ca.rope(s.rope, s.q[None], s.k[None], positions=plan.positions, layout="bnhd")
    ca.cache_write(k[0], s.v, s.k_pages, s.v_pages, plan.slots)
    out, _ = ca.paged_chunk_attn(s.window, q[0], s.k_pages, s.v_pages, s.table, s.lens, plan.starts, out=s.out)
    return {"out": out, "slots": plan.slots, "table": s.table, "k_pages": s.k_pages, "v_pages": s.v_pages}


# ---- the same in 64 bits, from the definitions -----------------------------------------------------------------

def _exact_grow(c, s):
    """(table, free pages, slots, positions) after the growth, entry by entry on the host."""
    table, pages, page = s.table.tolist(), s.free.tolist(), c["page"]
    free = pages[:int(s.state[0])]
    slots, positions = [], []
    for b, (a, n) in enumerate(_tokens(c)):
        for j in range(a, a + n):
            if not 0 <= table[b][j // page] < s.pages:
                table[b][j // page] = free.pop()
            slots.append(table[b][j // page] * page + j % page)
            positions.append(j)
    spare = c["spare"]
    return table, free, slots + [-1] * spare, positions + [0] * spare


def _exact_chunk(c, s, q, k_rows, v_rows, table):
    """q [T, H, d] in 64 bits; k_rows, v_rows: a sequence's keys and values [n, Hk, d] from its pages."""
    T, H, d = q.shape
    G = H // c["heads_k"]
    out, lse = torch.zeros(T, H, d, dtype=torch.float64, device="cuda"), torch.full((T, H), -math.inf, dtype=torch.float64, device="cuda")
    for b, (a, n) in enumerate(_tokens(c)):
        j = torch.arange(a + n, device="cuda")
        entry = table[b][j // c["page"]]
        there = entry >= 0
        rows = entry.clamp(min=0) * c["page"] + j % c["page"]
        for lo in range(0, n, max(1, int(3e8) // (a + n))):
            i = torch.arange(lo, min(n, lo + max(1, int(3e8) // (a + n))), device="cuda")
            p = (i + a)[:, None]
            near = (p - j <= c["left"]) if c["left"] >= 0 else torch.ones(len(i), a + n, dtype=torch.bool, device="cuda")
            if c["right"] >= 0:
                near &= j - p <= c["right"]
            near |= (j < c["sinks"])[None]
            if c["causal"]:
                near &= j <= p
            near &= there[None]
            t0 = s.host_starts[b] + lo
            for h in range(H):
                y, z = k_rows[rows, h // G].double(), v_rows[rows, h // G].double()
                t = torch.where(near, q[t0:t0 + len(i), h] @ y.T / math.sqrt(d), -math.inf)
                e = torch.logsumexp(t, 1)
                out[t0:t0 + len(i), h], lse[t0:t0 + len(i), h] = torch.exp(t - e[:, None]) @ z, e
    return out, lse


def _exact_rope(s, x, positions):
    """Each pair as a complex number, times the unit number of its angle."""
    x, m = x.double().clone(), len(s.freqs)
    angle = positions.double()[:, None] * torch.tensor(s.freqs, dtype=torch.float64, device="cuda")
    z = torch.complex(x[..., :m], x[..., m:2 * m]) * torch.polar(torch.ones_like(angle), angle)[:, None]
    x[..., :m], x[..., m:2 * m] = z.real, z.imag
    return x


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    c, kind = case, case["kind"]
    if kind == "pages":
        _, _, slots, positions = _exact_grow(c, s)
        # (the table and the free list end as they were)
        return {"starts": s.starts, "slots": torch.tensor(slots), "positions": torch.tensor(positions, dtype=torch.int32),
                "table": s.table, "free": s.free, "state": s.state}
    if kind == "chunk":
        out, lse = _exact_chunk(c, s, s.q.double(), s.k_pages.flatten(0, 1), s.v_pages.flatten(0, 1), s.table.long())
        return {"out": out, "lse": lse}
    kp, vp = (x.flatten(0, 1).double() for x in (s.k_pages, s.v_pages))
    if kind == "write":
        real = s.slots >= 0
        kp[s.slots[real]], vp[s.slots[real]] = s.k[real].double(), s.v[real].double()
        return {"k_pages": kp.reshape(s.k_pages.shape), "v_pages": vp.reshape(s.v_pages.shape)}
    table, _, slots, positions = _exact_grow(c, s)
    n = s.host_starts[-1]
    positions, at = torch.tensor(positions, device="cuda"), torch.tensor(slots[:n], device="cuda")
    q, k = _exact_rope(s, s.q, positions), _exact_rope(s, s.k, positions)
    kp[at], vp[at] = k[:n], s.v[:n].double()
    table = torch.tensor(table, device="cuda")
    out, _ = _exact_chunk(c, s, q, kp, vp, table)
    return {"out": out, "slots": torch.tensor(slots), "table": table.to(torch.int32), "k_pages": kp.reshape(s.k_pages.shape),
            "v_pages": vp.reshape(s.v_pages.shape)}
