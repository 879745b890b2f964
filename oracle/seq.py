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
