"""The sequence operators in plain fp64 NumPy, one head at a time: rotary
positions of several axes, attention with a sliding window and sinks with its
gradients. Test infrastructure only; written from the formulas in
include/clusterattn.h."""
import numpy as np


def rope(x, pos, sections, freqs, pairing="interleaved", inverse=False):
    """x [n, d] turned by pos [axes, n]: pair i by the angle pos[axis of i] * freqs[i]."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    m = sum(sections)
    axis = np.repeat(np.arange(len(sections)), sections)
    for i in range(m):
        t = np.asarray(pos[axis[i]], np.float64) * np.float64(freqs[i])
        if inverse:
            t = -t
        a, b = (i, i + m) if pairing == "halves" else (2 * i, 2 * i + 1)
        y[:, a] = x[:, a] * np.cos(t) - x[:, b] * np.sin(t)
        y[:, b] = x[:, a] * np.sin(t) + x[:, b] * np.cos(t)
    return y


def grid_positions(n, grid, start=None):
    """[axes, n] of the first n elements of a row-major grid."""
    p = np.stack(np.unravel_index(np.arange(n), grid))
    return p if start is None else p + np.asarray(start)[:, None]


def visible(nq, nk, left=-1, right=-1, sinks=0, causal=False):
    """[nq, nk]: which keys a query sees; the last query sits beside the last key."""
    p, j = (np.arange(nq) + nk - nq)[:, None], np.arange(nk)[None]
    see = np.ones((nq, nk), bool)
    if left >= 0:
        see &= j >= p - left
    if right >= 0:
        see &= j <= p + right
    see |= j < sinks
    if causal:
        see &= j <= p
    return see


def attend(q, k, v, see, scale):
    """(out, lse, P): softmax attention over the visible keys; nothing visible: 0, -inf, 0."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    s = np.where(see, scale * (q @ k.T), -np.inf)
    m = s.max(1, initial=-np.inf, keepdims=True)
    m = np.where(np.isfinite(m), m, 0.0)
    e = np.exp(s - m)
    l = e.sum(1, keepdims=True)
    P = np.divide(e, l, out=np.zeros_like(e), where=l > 0)
    with np.errstate(divide="ignore"):
        lse = (m + np.log(l))[:, 0]
    return P @ v, lse, P


def attend_backward(q, k, v, do, see, scale):
    """(dq, dk, dv) of sum(do * out)."""
    q, k, v, do = (np.asarray(x, np.float64) for x in (q, k, v, do))
    o, _, P = attend(q, k, v, see, scale)
    dP = do @ v.T
    dS = P * (dP - (do * o).sum(1, keepdims=True))
    return scale * (dS @ k), scale * (dS.T @ q), P.T @ do


# ---- pages of a cache, entry by entry -----------------------------------------------------------

def cache_grow(table, free, lens, new, page, pages, tokens):
    """table: rows of entries and free: a list, its end taken first, both changed. Returns
    (state, starts, slots, positions)."""
    lacked, starts, slots, positions = 0, [0], [], []
    for b, row in enumerate(table):
        n = min(max(int(lens[b]), 0), len(row) * page)
        m = min(max(int(new[b]), 0), n)
        for i in range((n - m) // page, -(-n // page) if m else 0):
            if not 0 <= row[i] < pages:
                if free:
                    row[i] = free.pop()
                else:
                    lacked += 1
        for j in range(n - m, n):
            e = int(row[j // page])
            slots.append(e * page + j % page if 0 <= e < pages else -1)
            positions.append(j)
        starts.append(starts[-1] + m)
    total = starts[-1]
    rest = max(0, tokens - total)
    return ([len(free), lacked, max(0, total - tokens)], [min(x, tokens) for x in starts],
            slots[:tokens] + [-1] * rest, positions[:tokens] + [0] * rest)


def lens_with_rows(lens, new, most, tokens):
    """lens (cut to [0, most]) less the new tokens that have no row: the rows go to the first `tokens` new
    tokens, by sequence and place."""
    seen, row = [], 0
    for n, m in zip(lens, new):
        n = min(max(int(n), 0), most)
        for j in range(n - min(max(int(m), 0), n), n):
            n -= row >= tokens
            row += 1
        seen.append(n)
    return seen


def cache_release(table, free, lens, page, pages, left=-1, sinks=0):
    """Pages without a token that the sequence's next one sees go to free's end, the first of
    them last; their entries become -1."""
    gone = []
    for b, row in enumerate(table):
        n = min(max(int(lens[b]), 0), len(row) * page)
        for i, e in enumerate(row):
            places = range(i * page, min((i + 1) * page, n))
            if not any(left < 0 or j < sinks or j >= n - left for j in places) and 0 <= e < pages:
                gone.append(int(e))
                row[i] = -1
    free.extend(reversed(gone))
