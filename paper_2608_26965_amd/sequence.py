"""The sequence operators of libclusterattn: rotary positions of several axes,
attention with a sliding window and sinks and its gradients, and the paged
key-value cache with the attention of one new token (see
include/clusterattn.h for their definitions).

    rope                              turn queries and keys by their positions
    window_attn, window_attn_backward
    cache_append, paged_attn          serving: write new tokens, attend over the pages

As in the rest of the binding, every step runs in the HIP library: these
functions read shapes and strides, allocate outputs and workspaces with torch
and call on the current stream of the tensors' device. They are not recorded by
autograd: a training program calls window_attn_backward, and rope with
inverse=True, for the gradients.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass

import torch

from . import _lib
from ._lib import CA_BF16, CA_F32

__all__ = ["Rope", "rope_axes", "rope", "Window", "window_attn", "window_attn_backward",
           "cache_append", "paged_attn"]

_DT = {torch.float32: CA_F32, torch.bfloat16: CA_BF16}
_I64x3 = ctypes.c_int64 * 3
_I64x2 = ctypes.c_int64 * 2
_I32x4 = ctypes.c_int32 * 4


# ---- what every call checks -----------------------------------------------------

def _dtype(t):
    dt = _DT.get(t.dtype)
    if dt is None:
        raise ValueError(f"expected float32 or bfloat16, got {t.dtype}")
    if not t.is_cuda:
        raise ValueError("expected tensors on the GPU")
    return dt


def _same(t, like, name):
    if t.dtype != like.dtype or t.device != like.device:
        raise ValueError(f"{name}: expected {like.dtype} on {like.device}, got {t.dtype} on "
                         f"{t.device}")


def _rows(t, name, dims):
    if t.dim() != dims or (t.stride(-1) != 1 and t.size(-1) > 1):
        raise ValueError(f"{name}: expected {dims} dimensions, the last one contiguous")


def _sizes(t, layout, name):
    """(batch, heads, tokens, d) of a [B,H,N,d] or ("bnhd") [B,N,H,d] tensor."""
    _rows(t, name, 4)
    s = t.shape
    if layout == "bnhd":
        return s[0], s[2], s[1], s[3]
    if layout not in ("bhnd", "strided"):
        raise ValueError(layout)
    return tuple(s)


def _strides(t, layout):
    """(batch, head, token) element strides (0 where there is one: never used)."""
    a, b, c, _ = t.stride()
    x, y, z, _ = t.shape
    if layout == "bnhd":
        b, c, y, z = c, b, z, y
    return _I64x3(a if x > 1 else 0, b if y > 1 else 0, c if z > 1 else 0)


def _lead(t):
    """The strides of a tensor's first three (four dimensions) or two (three)."""
    if t.dim() == 4:
        return _strides(t, "bhnd")
    a, b, _ = t.stride()
    x, y, _ = t.shape
    return _I64x2(a if x > 1 else 0, b if y > 1 else 0)


def _new(t):
    """A dense tensor of t's shape."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


_MOST = 2 ** 31 - 1


def _int(x, name, least=-_MOST - 1, most=_MOST):
    """x as the C int32 that it has to fit in."""
    x = int(x)
    if not least <= x <= most:
        raise ValueError(f"{name} = {x} is out of range")
    return x


def _side(x):
    # a window wider than any sequence is no limit; so is a negative one
    return -1 if x < 0 or x > _MOST else int(x)


def _expect(t, shape, name):
    if t.shape != shape:  # (a torch.Size compares with a tuple)
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")


def _int32(t, shape, like, name):
    if t.dtype != torch.int32 or t.device != like.device:
        raise ValueError(f"{name}: expected int32 on {like.device}, got {t.dtype} on {t.device}")
    _expect(t, shape, name)
    if t.dim() and t.stride(-1) != 1 and t.size(-1) > 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")


def _call(name, device, *args):
    """The library's call on the current stream of `device`, made the current
    device for the launch."""
    f = getattr(_lib.load(), name)
    i = device.index
    if i == torch.cuda.current_device():
        # the handle alone: a torch.cuda.Stream object costs 2 us of a small call's 12
        st = f(*args, torch._C._cuda_getCurrentRawStream(i))
    else:
        with torch.cuda.device(i):
            st = f(*args, torch._C._cuda_getCurrentRawStream(i))
    if st:
        _lib.check(st, name)


def _workspace(size, *args, device, ws):
    """The caller's workspace, or a new one of the bytes that the library asks for."""
    if ws is not None:
        if ws.device != device or not ws.is_contiguous():
            raise ValueError(f"ws: expected a contiguous tensor on {device}")
        return ws
    n = ctypes.c_size_t(0)
    st = getattr(_lib.load(), size)(*args, n)
    if st:
        _lib.check(st, size)
    return torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None


def _ptr(t):
    return None if t is None else t.data_ptr()


# ---- rotary positions --------------------------------------------------------------

@dataclass(frozen=True)
class Rope:
    """Rotary positions: sections[a] pairs turn with axis a (at most 4 axes);
    freqs[i] is pair i's angle per position in radians, over all axes in
    order; pairing "interleaved" pairs dims (2i, 2i+1), "halves" pairs dims
    (i, i + npairs). Dims past the pairs do not turn."""
    sections: tuple
    freqs: tuple
    pairing: str = "interleaved"

    def __post_init__(self):
        if self.pairing not in ("interleaved", "halves"):
            raise ValueError(self.pairing)
        if not 1 <= len(self.sections) <= 4 or sum(self.sections) != len(self.freqs):
            raise ValueError("one to four sections, and a frequency for each of their pairs")
        if not 1 <= len(self.freqs) <= 64:
            raise ValueError("1 to 64 pairs")
        f = (ctypes.c_double * 64)(*self.freqs)
        s = _I32x4(*(_int(x, "sections", 0, 64) for x in self.sections))
        object.__setattr__(self, "_c", (len(self.sections), s, f))


def rope_axes(dims, base=10000.0, pairing="interleaved", shared=False) -> Rope:
    """A Rope from the dims of each axis (even): pair i of an axis of n dims
    turns by base^(-2i/n) per position, or with shared=True pair i of all
    pairs by base^(-2i/sum(dims)). For a video head of 128 for example
    rope_axes((44, 42, 42)): time, height, width."""
    dims = tuple(int(n) for n in dims)
    if not dims or any(n < 0 or n % 2 for n in dims):
        raise ValueError("dims must be even")
    if shared:
        total = sum(dims)
        f = tuple(base ** (-2.0 * i / total) for i in range(total // 2))
    else:
        f = tuple(base ** (-2.0 * i / n) for n in dims for i in range(n // 2))
    return Rope(tuple(n // 2 for n in dims), f, pairing)


def rope(r: Rope, q, k=None, *, grid=None, start=None, positions=None, inverse=False,
         layout="bhnd", q_out=None, k_out=None):
    """Turns q and k (optional) by their tokens' positions. q: [B,H,n,d]
    ("bhnd", "strided") or [B,n,H,d] ("bnhd"), any strides, k the same with its own head count.
    Positions: `positions` int32 [axes,n] or [B,axes,n], or `grid` (axis
    sizes; token i is element i in row-major order), shifted by `start`.
    inverse=True turns back (also: the gradients of the turned rows to those
    of the rows). q_out, k_out: outputs, by default new dense tensors of the same shape; passing q and k
    themselves turns them in place. Returns q_out, or (q_out, k_out) with k."""
    dt = _dtype(q)
    B, H, n, d = _sizes(q, layout, "q")
    axes, section, freq = r._c
    if q_out is None:
        q_out = _new(q)
    else:
        _same(q_out, q, "q_out")
        _rows(q_out, "q_out", 4)
        _expect(q_out, q.shape, "q_out")
    Hk, zero = 0, _I64x3()
    ks = kos = zero
    if k is not None:
        _same(k, q, "k")
        Bk, Hk, nk, dk = _sizes(k, layout, "k")
        if (Bk, nk, dk) != (B, n, d):
            raise ValueError("q and k must have the same batch, tokens and head dimension")
        if k_out is None:
            k_out = _new(k)
        else:
            _same(k_out, q, "k_out")
            _rows(k_out, "k_out", 4)
            _expect(k_out, k.shape, "k_out")
        ks, kos = _strides(k, layout), _strides(k_out, layout)
    if (grid is None) == (positions is None):
        raise ValueError("give either grid or positions")
    g, s, ps = _I32x4(), _I32x4(), zero
    if grid is not None:
        if len(grid) != axes or (start is not None and len(start) != axes):
            raise ValueError(f"grid and start need {axes} entries")
        g = _I32x4(*(_int(x, "grid") for x in grid))
        if start is not None:
            s = _I32x4(*(_int(x, "start") for x in start))
    else:
        if start is not None:
            raise ValueError("start goes with grid")
        if positions.dtype != torch.int32 or positions.device != q.device:
            raise ValueError(f"positions: expected int32 on {q.device}")
        z, t = tuple(positions.shape), positions.stride()
        if z == (axes, n):
            ps = _I64x3(0, t[0], t[1])
        elif z in ((B, axes, n), (1, axes, n)):
            ps = _I64x3(t[0] if z[0] > 1 else 0, t[1], t[2])
        else:
            raise ValueError(f"positions: expected [{axes}, {n}] or [{B}, {axes}, {n}], got "
                             f"{list(z)}")
    c = _lib.CaRope(B, H, Hk, n, d, dt, axes, section, int(r.pairing == "halves"), int(inverse),
                    g, s, ps, _strides(q, layout), ks, _strides(q_out, layout), kos, freq)
    _call("ca_rope", q.device, c, q.data_ptr(), _ptr(k), _ptr(positions), q_out.data_ptr(),
          _ptr(k_out) if k is not None else None)
    return q_out if k is None else (q_out, k_out)


# ---- window attention ----------------------------------------------------------------

@dataclass(frozen=True)
class Window:
    """Who sees whom: a query at position p sees key j where (j < sinks or
    p - left <= j <= p + right) and, if causal, j <= p. Negative left or
    right: no limit on that side."""
    left: int = -1
    right: int = -1
    sinks: int = 0
    causal: bool = False


def _window(w, q, k, v, out, scale, len_q, len_k, layout, grads=()):
    dt = _dtype(q)
    B, H, nq, d = _sizes(q, layout, "q")
    Bk, Hk, nk, dk = _sizes(k, layout, "k")
    _same(k, q, "k")
    _same(v, q, "v")
    _rows(v, "v", 4)
    _expect(v, k.shape, "v")
    if (Bk, dk) != (B, d):
        raise ValueError("q and k must have the same batch and head dimension")
    for t, name in ((len_q, "len_q"), (len_k, "len_k")):
        if t is not None:
            _int32(t, (B,), q, name)
    _same(out, q, "out")
    _rows(out, "out", 4)
    _expect(out, q.shape, "out")
    return _lib.CaWindow(B, H, Hk, nq, nk, d, dt, _side(w.left), _side(w.right),
                         min(w.sinks, _MOST), int(w.causal),
                         0.0 if scale is None else float(scale), _strides(q, layout),
                         _strides(k, layout), _strides(v, layout), _strides(out, layout),
                         *(_strides(t, layout) for t in grads))


def _lse(q, layout):
    z = q.shape
    H, n = (z[2], z[1]) if layout == "bnhd" else (z[1], z[2])
    return q.new_empty((z[0], H, n), dtype=torch.float32)


def window_attn(w: Window, q, k, v, *, scale=None, len_q=None, len_k=None, layout="bhnd",
                want_lse=False, out=None, ws=None):
    """Attention with a sliding window and sinks. q: [B,H,nq,d] ("bhnd",
    "strided") or [B,nq,H,d] ("bnhd"), any strides; k, v the same with nk
    tokens and heads_k heads (a divisor of H). len_q, len_k: int32 [B], the
    lengths in a padded batch. Returns (out, lse [B,H,nq] fp32 or None); rows
    that see no key, and rows past len_q, are 0 with lse -inf."""
    if out is None:
        out = _new(q)
    c = _window(w, q, k, v, out, scale, len_q, len_k, layout)
    lse = _lse(q, layout) if want_lse else None
    ws = _workspace("ca_window_workspace_size", c, 0, device=q.device, ws=ws)
    _call("ca_window_attn", q.device, c, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(len_q),
          _ptr(len_k), out.data_ptr(), _ptr(lse), _ptr(ws), 0 if ws is None else ws.nbytes)
    return out, lse


def window_attn_backward(w: Window, dout, q, k, v, out, lse, *, scale=None, len_q=None,
                         len_k=None, layout="bhnd", dq=None, dk=None, dv=None, ws=None):
    """The gradients (dq, dk, dv) of window_attn for the output's gradient
    dout, from out and lse as window_attn gave them for the same arguments.
    dq, dk, dv: outputs of the inputs' shapes (any strides, for example slices
    of a fused projection's gradient), new dense tensors by default."""
    dq, dk, dv = (_new(t) if g is None else g for t, g in ((q, dq), (k, dk), (v, dv)))
    for t, like, name in ((dout, q, "dout"), (dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv")):
        _same(t, q, name)
        _rows(t, name, 4)
        _expect(t, like.shape, name)
    c = _window(w, q, k, v, out, scale, len_q, len_k, layout, (dout, dq, dk, dv))
    if lse.dtype != torch.float32 or lse.device != q.device or not lse.is_contiguous():
        raise ValueError("lse: expected a contiguous fp32 tensor on the same device")
    _expect(lse, (c.batch, c.heads, c.nq), "lse")
    ws = _workspace("ca_window_workspace_size", c, 1, device=q.device, ws=ws)
    _call("ca_window_attn_backward", q.device, c, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          out.data_ptr(), lse.data_ptr(), dout.data_ptr(), _ptr(len_q), _ptr(len_k),
          dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(ws), 0 if ws is None else ws.nbytes)
    return dq, dk, dv


# ---- paged cache -----------------------------------------------------------------------

def _paged(q, heads, k_pages, v_pages, table, lens, left, sinks, scale, q_st=None, o_st=None,
           n_new=0, kn=None, vn=None):
    dt = _dtype(k_pages)
    _rows(k_pages, "k_pages", 4)
    _rows(v_pages, "v_pages", 4)
    _same(v_pages, k_pages, "v_pages")
    _expect(v_pages, k_pages.shape, "v_pages")
    _same(q, k_pages, "queries or new keys")
    P, page, Hk, d = k_pages.shape
    B = q.shape[0]
    if q.shape[-1] != d:
        raise ValueError(f"expected rows of {d}, got {q.shape[-1]}")
    if table.dim() != 2:
        raise ValueError("page_table: expected [B, max_pages]")
    _int32(table, (B, table.shape[1]), k_pages, "page_table")
    _int32(lens, (B,), k_pages, "lens")
    z3, z2 = _I64x3(), _I64x2()
    return _lib.CaPaged(B, heads, Hk, d, dt, page, P, table.shape[1], _side(left), min(sinks, _MOST),
                        0.0 if scale is None else float(scale),
                        table.stride(0) if B > 1 else 0, _lead(k_pages),
                        _lead(v_pages), q_st or z2, o_st or z2, n_new, kn or z3, vn or z3)


def cache_append(k, v, k_pages, v_pages, page_table, lens):
    """Writes the new keys and values k, v [B,n,Hk,d] of B sequences into their
    pages: the last n of the lens[b] tokens of sequence b (lens counts them
    already). k_pages, v_pages: [pages, page, Hk, d], any strides;
    page_table: int32 [B, max_pages]; lens: int32 [B]. Returns nothing."""
    _rows(k, "k", 4)
    _rows(v, "v", 4)
    _same(v, k, "v")
    _expect(v, k.shape, "v")
    if k_pages.dim() == 4 and k.shape[2] != k_pages.shape[2]:
        raise ValueError(f"expected {k_pages.shape[2]} key heads, got {k.shape[2]}")
    c = _paged(k, k.shape[2], k_pages, v_pages, page_table, lens, -1, 0, None, n_new=k.shape[1],
               kn=_lead(k), vn=_lead(v))
    _call("ca_cache_append", k.device, c, k.data_ptr(), v.data_ptr(), k_pages.data_ptr(),
          v_pages.data_ptr(), page_table.data_ptr(), lens.data_ptr())


def paged_attn(q, k_pages, v_pages, page_table, lens, *, left=-1, sinks=0, scale=None,
               want_lse=False, out=None, ws=None):
    """Attention of one new token of each sequence, its last one, over the
    sequence's cached keys: all of them, or with left >= 0 the last left + 1
    and the first `sinks`. q: [B,H,d]; k_pages, v_pages: [pages, page, Hk, d],
    any strides, Hk a divisor of H; page_table: int32 [B, max_pages]; lens:
    int32 [B], the new token included. Returns (out [B,H,d], lse [B,H] fp32 or
    None); a sequence of no tokens gives 0 and -inf."""
    _rows(q, "q", 3)
    if out is None:
        out = _new(q)
    else:
        _same(out, q, "out")
        _rows(out, "out", 3)
        _expect(out, q.shape, "out")
    B, H = q.shape[0], q.shape[1]
    c = _paged(q, H, k_pages, v_pages, page_table, lens, left, sinks, scale, _lead(q),
               _lead(out))
    lse = q.new_empty((B, H), dtype=torch.float32) if want_lse else None
    ws = _workspace("ca_paged_workspace_size", c, device=q.device, ws=ws)
    _call("ca_paged_attn", q.device, c, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
          page_table.data_ptr(), lens.data_ptr(), out.data_ptr(), _ptr(lse), _ptr(ws),
          0 if ws is None else ws.nbytes)
    return out, lse
