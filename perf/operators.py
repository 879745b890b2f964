"""The sequence operators as cases that can be timed and compared: rotary positions of several axes, attention with a
sliding window and sinks (forward, and with its gradients), one-token attention over a paged cache, and a serving step
that runs them together with the append to the cache.

``listed()`` names the cases, ``draw(rng)`` gives more of the same ranges, ``prepare(case, seed)`` makes what a user's
program has in hand, ``run(state)`` is one pass: the framework's calls where ``own`` is true, else the same operators in
plain torch. ``work(case)`` is what a pass cannot do without, ``exact(case, seed)`` its result in 64 bits.

Kinds of cases ("kind"):

* ``rope``    ``rope`` of queries and keys, by a grid of positions or by positions given per token, and its transpose
              (``inverse``: the gradients' rotation).
* ``window``  ``window_attn``: output and log-sum-exp.
* ``train``   ``window_attn`` and ``window_attn_backward``: output, log-sum-exp and the three gradients.
* ``paged``   ``paged_attn``: one new token of each sequence against its pages.
* ``step``    ``rope`` of the new token's query and key, ``cache_append``, ``paged_attn``: output and the cache.

Queries and keys come from one Gaussian mixture with independent labels (so that attention has something to find),
values and gradients from a normal distribution. Lengths of ragged batches come from the case alone.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_BASE = dict(kind="window", dtype="bf16", batch=1, heads=8, heads_k=8, nq=1024, nk=1024, d=64, left=-1, right=-1,
             sinks=0, causal=False, layout="bhnd", ragged=False, lens_seed=0)
_ROPE = dict(kind="rope", dtype="bf16", batch=1, heads=8, heads_k=8, n=1024, d=64, axes="64", pairing="interleaved",
             shared=False, base=10000.0, grid="", far=0, inverse=False, layout="bhnd")
_PAGED = dict(kind="paged", dtype="bf16", batch=1, heads=8, heads_k=8, d=64, page=64, max_len=1024, left=-1, sinks=0,
              ragged=False, lens_seed=0)


def _case(start, name, **kw):
    c = dict(start, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Queries and keys of a 480p video layer (21 latent frames of 30 x 52), time, height and width in one head of
        # 128, read in a transformer's [B, N, H, d] layout. All memory traffic.
        _case(_ROPE, "rope_video_480p", heads=40, heads_k=40, n=32760, d=128, axes="44,42,42", grid="21,30,52",
              layout="bnhd"),
        # The gradients' rotation of two fp32 images of 45 x 80 patches, pairs taken from the two halves of the head.
        _case(_ROPE, "rope_image_f32_grad", dtype="f32", batch=2, n=3600, axes="32,32", pairing="halves", grid="45,80",
              inverse=True),
        # One new token of each of 64 streams at far positions, shared key heads: the smallest call.
        _case(_ROPE, "rope_token", batch=64, heads_k=2, n=1, axes="16,24,24", pairing="halves", shared=True,
              far=1 << 20),
        # Causal attention of a 480p video layer over the last three frames, the first frame kept as sinks.
        _case(_BASE, "window_video_480p", heads=40, heads_k=40, nq=32760, nk=32760, d=128, left=4679, sinks=1560,
              causal=True, layout="bnhd"),
        # A long table in sorted order, each row against 1,024 rows to both sides and 16 summary rows; odd length.
        _case(_BASE, "window_tab_65k", nq=65521, nk=65521, left=1024, right=1024, sinks=16, layout="fused"),
        # The smallest training call: one fp32 head of 1,024 tokens.
        _case(_BASE, "train_f32_1k", kind="train", dtype="f32", heads=1, heads_k=1, left=128, right=128, sinks=4),
        # Training of a sequence of 8,192, four query heads to a key head, causal, four sinks.
        _case(_BASE, "train_gqa_8k", kind="train", heads_k=2, nq=8192, nk=8192, left=1023, sinks=4, causal=True),
        # Training of a padded batch: three sequences of different lengths, no window, no mask but the lengths.
        _case(_BASE, "train_ragged", kind="train", batch=3, heads=12, heads_k=12, nq=4099, nk=4099, d=128, ragged=True,
              lens_seed=1, layout="bnhd"),
        # One new row against a cached table of 262,144 rows, 16 heads: the split over the cache's length.
        _case(_PAGED, "paged_262k", heads=16, heads_k=16, max_len=262144),
        # 32 sequences of very different lengths, five query heads to a key head.
        _case(_PAGED, "paged_ragged", batch=32, heads=40, heads_k=8, d=128, page=16, max_len=32768, ragged=True,
              lens_seed=2),
        # A serving step of four short sequences: latency.
        _case(_PAGED, "step_small", kind="step", batch=4, heads_k=2, page=16, max_len=500, left=127, sinks=4,
              ragged=True, lens_seed=3),
        # A serving step of a streamed video model: four streams of 40 heads, three frames of window and one of sinks.
        _case(_PAGED, "step_video", kind="step", batch=4, heads=40, heads_k=40, d=128, page=32, max_len=9360,
              left=4679, sinks=1560),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the logarithm of the listed range, odd ones among them, never over the largest."""
    kind = rng.choice(("rope", "window", "window", "train", "train", "paged", "paged", "step"))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    heads_k = rng.choice((1, 2, 3, 4, 8))
    heads = heads_k * rng.choice((1, 1, 2, 3, 4, 5, 8))
    d = rng.choice((64, 128))
    if kind == "rope":
        d = rng.choice((40, 64, 96, 128))
        n, batch = _log(rng, 1, 60000), rng.choice((1, 1, 2, 3, 16))
        while batch * n * (heads + heads_k) * d > 2 * 32760 * 40 * 128:
            n = max(1, n // 2)
        pairing = rng.choice(("interleaved", "halves"))
        axes = rng.choice((1, 2, 3))
        unit = 16 if pairing == "halves" else 2
        rot = d // unit * unit
        parts = [max(2, rot // axes // 2 * 2)] * axes
        parts[0] += rot - sum(parts)
        grid = ""
        if rng.random() < 0.6:
            cut = [max(1, round(n ** (1 / axes))) for _ in range(axes - 1)]
            grid = ",".join(str(v) for v in [-(-n // math.prod(cut))] + cut)
        return _case(_ROPE, None, dtype=dtype, batch=batch, heads=heads, heads_k=heads_k, n=n, d=d,
                     axes=",".join(map(str, parts)), pairing=pairing, shared=rng.random() < 0.5,
                     base=rng.choice((100.0, 10000.0, 500000.0)), grid=grid, far=_log(rng, 16, 1 << 20),
                     inverse=rng.random() < 0.3, layout=rng.choice(("bhnd", "bnhd")))
    if kind in ("window", "train"):
        batch = rng.choice((1, 1, 2, 3))
        # (one visible key a row has zero gradients of q and k, which no relative measure compares: training from 8 on)
        least = 8 if kind == "train" else 1
        nq = _log(rng, least, 65536)
        cross = rng.random() < 0.3
        nk = _log(rng, least, 65536) if cross else nq
        left = rng.choice((-1, _log(rng, 1, 4096), _log(rng, 1, 4096)))
        causal = rng.random() < 0.6
        right = 0 if causal else rng.choice((-1, _log(rng, 1, 4096)))
        sinks = rng.choice((0, 1, 4, 16, 300, 1560))
        c = _case(_BASE, None, kind=kind, dtype=dtype, batch=batch, heads=heads, heads_k=heads_k, nq=nq, nk=nk,
                  d=d, left=left, right=right, sinks=sinks, causal=causal,
                  layout=rng.choice(("bhnd", "bnhd", "fused" if heads == heads_k and not cross else "bhnd")),
                  ragged=batch > 1 and rng.random() < 0.6, lens_seed=rng.randrange(1000))
        cap = (2e10 if dtype == "f32" else 2e11) if kind == "train" else (4e10 if dtype == "f32" else 1e12)
        while work(c)["flops"] > cap:
            c["nq"], c["nk"] = max(least, c["nq"] * 2 // 3), max(least, c["nk"] * 2 // 3)
        return c
    max_len, batch = _log(rng, 1, 65536), rng.choice((1, 2, 4, 7, 32, 64))
    while batch * max_len * heads_k * d > 2 << 28 or (kind == "step" and batch * max_len * heads_k * d > 1 << 27):
        max_len = max(1, max_len // 2)
    return _case(_PAGED, None, kind=kind, dtype=dtype, batch=batch, heads=heads, heads_k=heads_k, d=d,
                 page=rng.choice((1, 7, 16, 32, 64, 128, 256)) if max_len < 20000 else rng.choice((16, 32, 64, 256)),
                 max_len=max_len, left=rng.choice((-1, -1, _log(rng, 1, 8192))), sinks=rng.choice((0, 0, 4, 100)),
                 ragged=batch > 1 and rng.random() < 0.7, lens_seed=rng.randrange(1000))


def _lens(c, n, salt):
    """Lengths of a ragged batch: the longest fills the tensor, the others fall over the range's logarithm."""
    if not c["ragged"]:
        return [n] * c["batch"]
    r = random.Random(1000 * c["lens_seed"] + salt)
    out = [max(1, _log(r, max(1, n // 64), n)) for _ in range(c["batch"])]
    out[r.randrange(len(out))] = n
    return out


def _lens_qk(c):
    lq = _lens(c, c["nq"], 1)
    return lq, lq if c["nq"] == c["nk"] else _lens(c, c["nk"], 2)


def _pairs(c):
    """Visible pairs (one head), queries and keys of all sequences. Key j of nk is visible to query i, which sits at
    p = i + nk - nq, where j < sinks or p - left <= j <= p + right, and j <= p in causal attention."""
    pairs = 0
    lens = _lens_qk(c)
    for nq, nk in zip(*lens):
        p = torch.arange(nq, dtype=torch.int64) + nk - nq
        hi = torch.full_like(p, nk - 1) if c["right"] < 0 else (p + c["right"]).clamp(max=nk - 1)
        lo = torch.zeros_like(p) if c["left"] < 0 else (p - c["left"]).clamp(min=0)
        top = torch.full_like(p, nk - 1)
        if c["causal"]:
            hi, top = torch.minimum(hi, p), torch.minimum(top, p)
        sink = torch.minimum(top + 1, torch.tensor(c["sinks"])).clamp(min=0)  # sinks visible: keys [0, sink)
        band = (hi + 1 - torch.maximum(lo, sink)).clamp(min=0)
        pairs += int((sink + band).sum())
    return pairs, sum(lens[0]), sum(lens[1])


def work(c):
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rope":
        x = c["batch"] * (c["heads"] + c["heads_k"]) * c["n"] * c["d"]
        return {"bytes": 2 * x * e, "flops": 3 * x}
    if c["kind"] in ("window", "train"):
        pairs, nq, nk = _pairs(c)
        q, kv = c["heads"] * nq * c["d"], 2 * c["heads_k"] * nk * c["d"]
        w = {"bytes": (2 * q + kv) * e + 4 * c["heads"] * nq, "flops": 4 * pairs * c["heads"] * c["d"]}
        if c["kind"] == "train":  # reads q, k, v, out, dout and the lse, writes three gradients; five products
            w["bytes"] += (4 * q + 2 * kv) * e + 4 * c["heads"] * nq
            w["flops"] += 10 * pairs * c["heads"] * c["d"]
        return w
    keys = 0
    for n in _lens(c, c["max_len"], 1):
        keys += n if c["left"] < 0 else min(n, c["left"] + 1 + min(c["sinks"], max(0, n - c["left"] - 1)))
    q = c["batch"] * c["heads"] * c["d"]
    w = {"bytes": (2 * q + 2 * keys * c["heads_k"] * c["d"]) * e + 4 * c["batch"] * c["heads"],
         "flops": 4 * keys * c["heads"] * c["d"]}
    if c["kind"] == "step":
        w["bytes"] += (2 * q + 6 * c["batch"] * c["heads_k"] * c["d"]) * e
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


def _freqs(c):
    """Radians per position of each pair, and the pairs of each axis."""
    dims = [int(x) for x in c["axes"].split(",")]
    if c["shared"]:
        f = [c["base"] ** (-2.0 * i / sum(dims)) for i in range(sum(dims) // 2)]
    else:
        f = [c["base"] ** (-2.0 * i / n) for n in dims for i in range(n // 2)]
    return f, [n // 2 for n in dims]


def _make_rope(s, c):
    s.freqs, s.sections = _freqs(c)
    s.pairing, s.inverse, s.layout = c["pairing"], c["inverse"], c["layout"]
    if own:
        import paper_2608_26965_amd as ca
        s.rope = ca.Rope(sections=tuple(s.sections), freqs=tuple(s.freqs), pairing=s.pairing)


def prepare(case, seed):
    c, s = case, _State()
    s.case = c
    g = _gen(seed)
    dt = _DT[c["dtype"]]
    centres = torch.randn(64, c["d"], generator=g, device="cuda").mul_(0.8)
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda").to(dt)  # noqa: E731
    if c["kind"] == "rope":
        ax = len(c["axes"].split(","))
        shape = (lambda h: (c["batch"], h, c["n"])) if c["layout"] == "bhnd" else (lambda h: (c["batch"], c["n"], h))
        s.q, s.k = rnd(*shape(c["heads"]), c["d"]), rnd(*shape(c["heads_k"]), c["d"])
        s.grid = tuple(int(x) for x in c["grid"].split(",")) if c["grid"] else None
        s.positions = None
        if not s.grid:
            s.positions = torch.randint(0, c["far"], (c["batch"], ax, c["n"]), generator=g, device="cuda",
                                        dtype=torch.int32)
        _make_rope(s, c)
        return s
    s.left, s.sinks = c["left"], c["sinks"]
    if c["kind"] in ("window", "train"):
        B, H, Hk, nq, nk, d = (c[x] for x in ("batch", "heads", "heads_k", "nq", "nk", "d"))
        s.right, s.causal = c["right"], c["causal"]
        s.layout = "strided" if c["layout"] == "fused" else c["layout"]
        if c["layout"] == "fused":
            qkv = torch.empty(B, nq, 3, H, d, dtype=dt, device="cuda")
            qkv[:, :, 0], qkv[:, :, 1] = _mixture(g, centres, B, nq, H), _mixture(g, centres, B, nq, H)
            qkv[:, :, 2] = rnd(B, nq, H, d)
            s.q, s.k, s.v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
            s.dout = rnd(B, H, nq, d)
        else:
            shape = (lambda h, n: (B, h, n)) if c["layout"] == "bhnd" else (lambda h, n: (B, n, h))
            s.q, s.k = (_mixture(g, centres, *shape(h, n)).to(dt) for h, n in ((H, nq), (Hk, nk)))
            s.v, s.dout = rnd(*shape(Hk, nk), d), rnd(*shape(H, nq), d)
        s.lens_q, s.lens_k = _lens_qk(c)
        s.len_q = s.len_k = None
        if c["ragged"]:
            s.len_q, s.len_k = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (s.lens_q, s.lens_k))
        if own:
            import paper_2608_26965_amd as ca
            s.window = ca.Window(left=s.left, right=s.right, sinks=s.sinks, causal=s.causal)
        return s
    B, H, Hk, d, page = (c[x] for x in ("batch", "heads", "heads_k", "d", "page"))
    s.host_lens = _lens(c, c["max_len"], 1)
    s.lens = torch.tensor(s.host_lens, dtype=torch.int32, device="cuda")
    width = -(-c["max_len"] // page)
    need = [-(-n // page) for n in s.host_lens]
    pool = sum(need) + 3
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    s.table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        s.table[b, :n] = order[at:at + n]
        at += n
    s.k_pages = torch.empty(pool, page, Hk, d, dtype=dt, device="cuda")
    for lo in range(0, pool, max(1, (1 << 26) // (page * Hk * d))):  # drawn in fp32, some pages at a time
        part = s.k_pages[lo:lo + max(1, (1 << 26) // (page * Hk * d))]
        part.copy_(_mixture(g, centres, *part.shape[:3]))
    s.v_pages = torch.randn(pool, page, Hk, d, generator=g, device="cuda", dtype=dt)
    if c["kind"] == "paged":
        s.q = _mixture(g, centres, B, H).to(dt)
        return s
    s.q, s.k = _mixture(g, centres, B, 1, H).to(dt), _mixture(g, centres, B, 1, Hk).to(dt)
    s.v = rnd(B, 1, Hk, d)
    # the new token's place in a grid of 30 x 52 patches a frame
    i = s.lens.to(torch.int64) - 1
    s.positions = torch.stack((i // 1560, i // 52 % 30, i % 52), 1).to(torch.int32)[:, :, None].contiguous()
    r = d // 3 // 2 * 2
    _make_rope(s, dict(_ROPE, axes="%d,%d,%d" % (d - 2 * r, r, r), layout="bnhd"))
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------

def _by_axis(s, n):
    """Positions [batch or 1, pairs, n] of each pair's axis, 64-bit."""
    if s.positions is not None:
        p = s.positions.double()
    else:
        i, parts = torch.arange(n, device="cuda"), []
        for size in reversed(s.grid):
            parts.insert(0, i % size)
            i = i // size
        p = torch.stack(parts)[None].double()
    return p.repeat_interleave(torch.tensor(s.sections, device="cuda"), 1)


def _plain_rope(s, x):
    t = x if s.layout == "bhnd" else x.transpose(1, 2)
    angle = _by_axis(s, t.shape[2]) * torch.tensor(s.freqs, dtype=torch.float64, device="cuda")[None, :, None]
    cos, sin = angle.cos().float().transpose(1, 2)[:, None], angle.sin().float().transpose(1, 2)[:, None]
    if s.inverse:
        sin = -sin
    m = len(s.freqs)
    f = t.float()
    if s.pairing == "halves":
        a, b = f[..., :m], f[..., m:2 * m]
        rot = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = f[..., 0:2 * m:2], f[..., 1:2 * m:2]
        rot = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    y = torch.cat((rot, f[..., 2 * m:]), -1).to(x.dtype)
    return (y if s.layout == "bhnd" else y.transpose(1, 2)).contiguous()


def _visible(s, i, j, lq, lk):
    """Which keys j [m] the queries i [n] see, [B, 1, 1, n, m] (lq, lk: [B] lengths)."""
    i, j = i[None, :, None], j[None, None, :]
    lq, lk = lq[:, None, None], lk[:, None, None]
    p = i + lk - lq
    see = torch.ones_like(p + j, dtype=torch.bool)
    if s.left >= 0:
        see &= j >= p - s.left
    if s.right >= 0:
        see &= j <= p + s.right
    see |= j < s.sinks
    if s.causal:
        see &= j <= p
    return (see & (j < lk) & (i < lq))[:, None, None]


def _plain_window(s, grads):
    """Softmax attention over blocks of queries against the keys that any of the block can see. A block's logits are
    all that is held of the large matrix, so a long sequence takes several blocks."""
    q, k, v, do = ((x if s.layout != "bnhd" else x.transpose(1, 2)) for x in (s.q, s.k, s.v, s.dout))
    B, H, nq, d = q.shape
    Hk, nk = k.shape[1], k.shape[2]
    G, scale = H // Hk, 1.0 / math.sqrt(d)
    dev = q.device
    lq, lk = (torch.tensor(x, device=dev) for x in (s.lens_q, s.lens_k))
    kf, vf = k.float()[:, :, None], v.float()[:, :, None]  # [B, Hk, 1, nk, d]
    out = torch.empty(B, Hk, G, nq, d, device=dev)
    lse = torch.empty(B, Hk, G, nq, device=dev)
    if grads:
        dq, dk, dv = torch.empty_like(out), torch.zeros_like(kf), torch.zeros_like(vf)
    offs = [b - a for a, b in zip(s.lens_q, s.lens_k)]
    reach = (s.left if s.left >= 0 else nk) + (s.right if s.right >= 0 and not s.causal else 0 if s.causal else nk)
    rows = max(64, min(nq, max(1024, reach), int(2e9 / (B * H * min(nk, 2 * reach + s.sinks + 1024)))))
    for i0 in range(0, nq, rows):
        i1 = min(nq, i0 + rows)
        lo = max(0, i0 + min(offs) - s.left) if s.left >= 0 else 0
        hi = i1 + max(offs) if s.causal else i1 + max(offs) + s.right if s.right >= 0 else nk
        hi = max(0, min(nk, hi))
        lo = min(lo, hi)
        first = min(s.sinks, lo, nk if not s.causal else hi)
        if not s.causal and s.sinks > hi:
            lo, first, hi = 0, 0, nk
        j = torch.cat((torch.arange(first, device=dev), torch.arange(lo, hi, device=dev)))
        kb, vb = (torch.cat((x[..., :first, :], x[..., lo:hi, :]), -2) for x in (kf, vf))
        qb = q[:, :, i0:i1].float().reshape(B, Hk, G, i1 - i0, d)
        logit = torch.matmul(qb, kb.transpose(-1, -2)).mul_(scale)
        logit.masked_fill_(~_visible(s, torch.arange(i0, i1, device=dev), j, lq, lk), -math.inf)
        top = logit.amax(-1, keepdim=True) if j.numel() else torch.full_like(qb[..., :1], -math.inf)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        prob = logit.sub_(top).exp_()
        total = prob.sum(-1, keepdim=True)
        prob.div_(torch.where(total > 0, total, torch.ones_like(total)))
        out[..., i0:i1, :] = torch.matmul(prob, vb)
        lse[..., i0:i1] = (top + total.log())[..., 0]
        if grads:
            dob = do[:, :, i0:i1].float().reshape(B, Hk, G, i1 - i0, d)
            gv = torch.matmul(prob.transpose(-1, -2), dob).sum(2, keepdim=True)
            dp = torch.matmul(dob, vb.transpose(-1, -2))
            ds = dp.sub_((prob * dp).sum(-1, keepdim=True)).mul_(prob).mul_(scale)
            dq[..., i0:i1, :] = torch.matmul(ds, kb)
            gk = torch.matmul(ds.transpose(-1, -2), qb).sum(2, keepdim=True)
            for acc, x in ((dk, gk), (dv, gv)):
                acc[..., :first, :] += x[..., :first, :]
                acc[..., lo:hi, :] += x[..., first:, :]
    give = lambda x, n, h: _laid_out(s, x.reshape(B, h, n, d).to(q.dtype))  # noqa: E731
    r = {"out": give(out, nq, H), "lse": lse.reshape(B, H, nq)}
    if grads:
        r.update(dq=give(dq, nq, H), dk=give(dk, nk, Hk), dv=give(dv, nk, Hk))
    return r


def _laid_out(s, x):
    return x if s.layout != "bnhd" else x.transpose(1, 2).contiguous()


def _plain_paged(s, q):
    """q [B, H, d] against the keys of each sequence's pages."""
    B, H, d = q.shape
    page, Hk = s.k_pages.shape[1], s.k_pages.shape[2]
    at = s.table.clamp(min=0).long()
    k, v = (x[at].flatten(1, 2).float().transpose(1, 2) for x in (s.k_pages, s.v_pages))  # [B, Hk, L, d]
    j = torch.arange(k.shape[2], device=q.device)[None]
    n = s.lens[:, None]
    see = j < n
    if s.left >= 0:
        see &= (j >= n - 1 - s.left) | (j < s.sinks)
    logit = torch.matmul(q.float().reshape(B, Hk, H // Hk, d), k.transpose(-1, -2)) / math.sqrt(d)
    logit.masked_fill_(~see[:, None, None], -math.inf)
    top = logit.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    prob = (logit - top).exp()
    total = prob.sum(-1, keepdim=True)
    out = torch.matmul(prob, v) / torch.where(total > 0, total, torch.ones_like(total))
    return {"out": out.reshape(B, H, d).to(q.dtype), "lse": (top + total.log()).reshape(B, H)}


def _plain_append(s, k):
    i = s.lens.long() - 1
    page = s.k_pages.shape[1]
    at = s.table.gather(1, (i // page)[:, None])[:, 0].long()
    s.k_pages[at, i % page] = k[:, 0]
    s.v_pages[at, i % page] = s.v[:, 0]


# ---- one pass --------------------------------------------------------------------------------------------------

def run(s):
    kind = s.case["kind"]
    if not own:
        if kind == "rope":
            return {"q": _plain_rope(s, s.q), "k": _plain_rope(s, s.k)}
        if kind in ("window", "train"):
            return _plain_window(s, kind == "train")
        if kind == "paged":
            return _plain_paged(s, s.q)
        q, k = _plain_rope(s, s.q), _plain_rope(s, s.k)
        _plain_append(s, k)
        return {"out": _plain_paged(s, q[:, 0])["out"], "k_pages": s.k_pages, "v_pages": s.v_pages}
    import paper_2608_26965_amd as ca
    if kind == "rope":
        q, k = ca.rope(s.rope, s.q, s.k, grid=s.grid, positions=s.positions, inverse=s.inverse, layout=s.layout)
        return {"q": q, "k": k}
    if kind in ("window", "train"):
        kw = dict(len_q=s.len_q, len_k=s.len_k, layout=s.layout)
        out, lse = ca.window_attn(s.window, s.q, s.k, s.v, want_lse=True, **kw)
        r = {"out": out, "lse": lse}
        if kind == "train":
            r["dq"], r["dk"], r["dv"] = ca.window_attn_backward(s.window, s.dout, s.q, s.k, s.v, out, lse, **kw)
        return r
    if kind == "paged":
        out, lse = ca.paged_attn(s.q, s.k_pages, s.v_pages, s.table, s.lens, left=s.left, sinks=s.sinks, want_lse=True)
        return {"out": out, "lse": lse}
    q, k = ca.rope(s.rope, s.q, s.k, positions=s.positions, layout="bnhd")
    ca.cache_append(k, s.v, s.k_pages, s.v_pages, s.table, s.lens)
    out, _ = ca.paged_attn(q[:, 0], s.k_pages, s.v_pages, s.table, s.lens, left=s.left, sinks=s.sinks)
    return {"out": out, "k_pages": s.k_pages, "v_pages": s.v_pages}


# ---- the same in 64 bits, from the definitions -----------------------------------------------------------------

def _exact_rope(c, s, x):
    """Each pair as a complex number, times the unit number of its angle."""
    x = x.double() if s.layout == "bhnd" else x.double().transpose(1, 2)
    B, H, n, d = x.shape
    y = x.clone()
    first = 0
    m = sum(s.sections)
    for a, pairs in enumerate(s.sections):
        if s.positions is not None:
            pos = s.positions[:, a].double()
        else:
            inner = math.prod(s.grid[a + 1:])
            pos = (torch.arange(n, device="cuda") // inner).remainder(s.grid[a])[None].double()
        for p in range(first, first + pairs):
            one, two = (p, p + m) if s.pairing == "halves" else (2 * p, 2 * p + 1)
            z = torch.complex(x[..., one], x[..., two])
            turn = torch.polar(torch.ones_like(pos), pos * (-s.freqs[p] if s.inverse else s.freqs[p]))[:, None]
            z = z * turn
            y[..., one], y[..., two] = z.real, z.imag
        first += pairs
    return y if s.layout == "bhnd" else y.transpose(1, 2).contiguous()


def _exact_window(c, s, grads):
    q, k, v, do = ((x if s.layout != "bnhd" else x.transpose(1, 2)) for x in (s.q, s.k, s.v, s.dout))
    B, H, nq, d = q.shape
    Hk, nk = k.shape[1], k.shape[2]
    new = lambda h, n, *r: torch.zeros(B, h, n, *r, dtype=torch.float64, device="cuda")  # noqa: E731
    out, lse, dq, dk, dv = new(H, nq, d), new(H, nq) - math.inf, new(H, nq, d), new(Hk, nk, d), new(Hk, nk, d)
    rows = max(1, min(nq, int(4e8 / max(1, nk))))
    for b in range(B):
        lq, lk = s.lens_q[b], s.lens_k[b]
        j = torch.arange(lk, device="cuda")
        for i0 in range(0, lq, rows):
            i = torch.arange(i0, min(lq, i0 + rows), device="cuda")
            p = (i + (lk - lq))[:, None]
            near = torch.ones(len(i), lk, dtype=torch.bool, device="cuda")
            if c["left"] >= 0:
                near &= (p - j) <= c["left"]
            if c["right"] >= 0:
                near &= (j - p) <= c["right"]
            near |= (j < c["sinks"])[None]
            if c["causal"]:
                near &= (j - p) <= 0
            for h in range(H):
                x, y, z = q[b, h, i].double(), k[b, h * Hk // H, :lk].double(), v[b, h * Hk // H, :lk].double()
                t = torch.where(near, x @ y.T / math.sqrt(d), -math.inf)
                e = torch.logsumexp(t, 1)
                w = torch.where(near, torch.exp(t - torch.where(e > -math.inf, e, 0.0)[:, None]), 0.0)
                out[b, h, i], lse[b, h, i] = w @ z, e
                if grads:
                    g = do[b, h, i].double()
                    dv[b, h * Hk // H, :lk] += w.T @ g
                    u = g @ z.T
                    u = w * (u - (w * u).sum(1, keepdim=True)) / math.sqrt(d)
                    dq[b, h, i] = u @ y
                    dk[b, h * Hk // H, :lk] += u.T @ x
    r = {"out": _laid_out(s, out), "lse": lse}
    if grads:
        r.update(dq=_laid_out(s, dq), dk=_laid_out(s, dk), dv=_laid_out(s, dv))
    return r


def _exact_paged(c, s, q, new_k=None):
    B, H, d = q.shape
    page, Hk = s.k_pages.shape[1], s.k_pages.shape[2]
    out = torch.zeros(B, H, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s.host_lens):
        keep = [j for j in range(min(c["sinks"], n))] if c["left"] >= 0 else []
        start = max(len(keep), n - 1 - c["left"]) if c["left"] >= 0 else 0
        j = torch.cat((torch.tensor(keep, dtype=torch.int64, device="cuda"), torch.arange(start, n, device="cuda")))
        at = s.table[b].long()[j // page]
        for h in range(Hk):
            y, z = (x[at, j % page, h].double() for x in (s.k_pages, s.v_pages))
            if new_k is not None:
                y[-1] = new_k[b, 0, h]
                z[-1] = s.v[b, 0, h].double()
            G = H // Hk
            t = q[b, h * G:(h + 1) * G].double() @ y.T / math.sqrt(d)
            e = torch.logsumexp(t, 1)
            out[b, h * G:(h + 1) * G], lse[b, h * G:(h + 1) * G] = torch.exp(t - e[:, None]) @ z, e
    return {"out": out, "lse": lse}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind = case["kind"]
    if kind == "rope":
        return {"q": _exact_rope(case, s, s.q), "k": _exact_rope(case, s, s.k)}
    if kind in ("window", "train"):
        return _exact_window(case, s, kind == "train")
    if kind == "paged":
        return _exact_paged(case, s, s.q)
    q, k = _exact_rope(case, s, s.q), _exact_rope(case, s, s.k)
    out = _exact_paged(case, s, q[:, 0], k)["out"]
    kp, vp = s.k_pages.double(), s.v_pages.double()
    for b, n in enumerate(s.host_lens):
        at = int(s.table[b, (n - 1) // case["page"]])
        kp[at, (n - 1) % case["page"]], vp[at, (n - 1) % case["page"]] = k[b, 0], s.v[b, 0].double()
    return {"out": out, "k_pages": kp, "v_pages": vp}
