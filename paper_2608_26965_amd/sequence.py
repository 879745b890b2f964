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
inverse=True, for the gradients (lse has none). Where autograd records, inputs
that require gradients give a warning, and tensors that require them are
refused as outputs; outputs that the caller gave count as changed in place.
"""
from __future__ import annotations

import ctypes
import functools
import warnings
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
#
# A call's descriptor (sizes, strides, type, options) takes longer to make than the
# launch of a small kernel, and a program makes the same few calls again and again:
# descriptors are kept by what they are made from. They hold no address. Numbers are
# made Python's own before they become part of a key: a tensor of one element is equal to
# itself whatever it holds by now.
_kept = functools.lru_cache(maxsize=1024)


def _geo(t):
    """What a descriptor says of a tensor."""
    return t.shape, t.stride(), t.dtype


def _on(like, *tensors):
    """Of a type that the library has, and all on one GPU."""
    _dtype(like.dtype)
    if not like.is_cuda:
        raise ValueError("expected tensors on the GPU")
    i = like.get_device()  # (half the time of a torch.device; -1 off the GPU)
    for t in tensors:
        if t is not None and t.get_device() != i:
            raise ValueError(f"expected all tensors on {like.device}, got one on {t.device}")


def _unrecorded(read, written):
    """Where autograd records, tells what the call does not do."""
    for t in written:
        if t is not None and t.requires_grad:
            raise ValueError("the call would write a tensor that requires gradients, unrecorded by "
                             "autograd: give it detached, or call under torch.no_grad()")
    for t in read:
        if t is not None and t.requires_grad:
            warnings.warn("not recorded by autograd: no gradient reaches the inputs that require one "
                          "(window_attn_backward and rope with inverse=True form them)", stacklevel=3)
            return


def _wrote(*tensors):
    """Tensors of the caller's that a call wrote (some may be None): their versions tell
    autograd, which saw none of it."""
    # (torch.autograd.graph.increment_version is this and 0.4 us more, of a small call's 9)
    torch._C._increment_version([t for t in tensors if t is not None])


def _dtype(dtype):
    dt = _DT.get(dtype)
    if dt is None:
        raise ValueError(f"expected float32 or bfloat16, got {dtype}")
    return dt


def _rows(geo, name, dims, dtype, shape=None):
    """(shape, strides) of rows that are contiguous; a stride of a dimension of one
    element, which is never used, as 0."""
    size, stride, dt = geo
    if len(size) != dims or (stride[-1] != 1 and size[-1] > 1):
        raise ValueError(f"{name}: expected {dims} dimensions, the last one contiguous")
    if dt != dtype:
        raise ValueError(f"{name}: expected {dtype}, got {dt}")
    if shape is not None and tuple(size) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(size)}")
    return tuple(size), tuple(b if a > 1 else 0 for a, b in zip(size, stride))


def _heads(geo, layout, name, dtype, shape=None):
    """((batch, heads, tokens, d), {batch, head, token} strides) of a [B,H,N,d] or
    ("bnhd") [B,N,H,d] tensor."""
    (a, b, c, d), (x, y, z, _) = _rows(geo, name, 4, dtype, shape)
    if layout == "bnhd":
        return (a, c, b, d), _I64x3(x, z, y)
    if layout not in ("bhnd", "strided"):
        raise ValueError(layout)
    return (a, b, c, d), _I64x3(x, y, z)


def _int32(geo, name, *shapes):
    if geo[2] != torch.int32:
        raise ValueError(f"{name}: expected int32, got {geo[2]}")
    if tuple(geo[0]) not in shapes:
        raise ValueError(f"{name}: expected {' or '.join(map(str, map(list, shapes)))}, got "
                         f"{list(geo[0])}")


def _dense(geo):
    """The geometry of a dense tensor of the same shape."""
    size, stride, n = geo[0], [], 1
    for x in reversed(size):
        stride.insert(0, n)
        n *= max(1, x)
    return size, tuple(stride), geo[2]


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


def _ints(x):
    return None if x is None else tuple(int(i) for i in x)


def _scale(x):
    return None if x is None else float(x)


def _side(x):
    # a window wider than any sequence is no limit; so is a negative one
    return -1 if x < 0 or x > _MOST else int(x)


def _call(name, device, *args):
    """The library's call on the current stream of `device`, made the current
    device for the launch."""
    f = getattr(_lib.load(), name)
    i = device.index
    if i == torch.cuda.current_device():
        # the handle alone: a torch.cuda.Stream object costs 2 us of a small call's 9
        st = f(*args, torch._C._cuda_getCurrentRawStream(i))
    else:
        with torch.cuda.device(i):
            st = f(*args, torch._C._cuda_getCurrentRawStream(i))
    if st:
        _lib.check(st, name)


def _bytes(size, *args):
    """Bytes of workspace that the library asks for."""
    n = ctypes.c_size_t(0)
    _lib.check(getattr(_lib.load(), size)(*args, n), size)
    return n.value


def _workspace(nbytes, like, ws):
    """The caller's workspace, or a new one."""
    if ws is None:
        return like.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    if ws.device != like.device or not ws.is_contiguous():
        raise ValueError(f"ws: expected a contiguous tensor on {like.device}")
    return ws


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
        object.__setattr__(self, "sections", _ints(self.sections))
        object.__setattr__(self, "freqs", tuple(float(x) for x in self.freqs))
        if self.pairing not in ("interleaved", "halves"):
            raise ValueError(self.pairing)
        if not 1 <= len(self.sections) <= 4 or sum(self.sections) != len(self.freqs):
            raise ValueError("one to four sections, and a frequency for each of their pairs")
        if not 1 <= len(self.freqs) <= 64:
            raise ValueError("1 to 64 pairs")
        f = (ctypes.c_double * 64)(*self.freqs)
        s = _I32x4(*(_int(x, "sections", 0, 64) for x in self.sections))
        object.__setattr__(self, "_c", (len(self.sections), s, f))
        object.__setattr__(self, "_hash", hash((self.sections, self.freqs, self.pairing)))

    def __hash__(self):
        return self._hash


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


@_kept
def _rope(r, q, k, q_out, k_out, positions, grid, start, inverse, layout):
    dtype = q[2]
    dt = _dtype(dtype)
    (B, H, n, d), qs = _heads(q, layout, "q", dtype)
    qos = _heads(q_out or _dense(q), layout, "q_out", dtype, q[0])[1]
    Hk, ks, kos = 0, _I64x3(), _I64x3()
    if k is not None:
        (Bk, Hk, nk, dk), ks = _heads(k, layout, "k", dtype)
        if (Bk, nk, dk) != (B, n, d):
            raise ValueError("q and k must have the same batch, tokens and head dimension")
        kos = _heads(k_out or _dense(k), layout, "k_out", dtype, k[0])[1]
    axes, section, freq = r._c
    g, s, ps = _I32x4(), _I32x4(), _I64x3()
    if grid is not None:
        if len(grid) != axes or (start is not None and len(start) != axes):
            raise ValueError(f"grid and start need {axes} entries")
        g = _I32x4(*(_int(x, "grid") for x in grid))
        if start is not None:
            s = _I32x4(*(_int(x, "start") for x in start))
    else:
        if start is not None:
            raise ValueError("start goes with grid")
        _int32(positions, "positions", (axes, n), (B, axes, n), (1, axes, n))
        t = positions[1]
        ps = _I64x3(0 if len(t) == 2 or positions[0][0] == 1 else t[0], t[-2], t[-1])
    return _lib.CaRope(B, H, Hk, n, d, dt, axes, section, int(r.pairing == "halves"), int(inverse),
                       g, s, ps, qs, ks, qos, kos, freq)


def rope(r: Rope, q, k=None, *, grid=None, start=None, positions=None, inverse=False,
         layout="bhnd", q_out=None, k_out=None):
    """Turns q and k (optional) by their tokens' positions. q: [B,H,n,d]
    ("bhnd", "strided") or [B,n,H,d] ("bnhd"), any strides, k the same with its
    own head count. Positions: `positions` int32 [axes,n] or [B,axes,n], or
    `grid` (axis sizes; token i is element i in row-major order), shifted by
    `start`. inverse=True turns back (also: the gradients of the turned rows to
    those of the rows). q_out, k_out: outputs, by default new dense tensors of
    the same shape; passing q and k themselves turns them in place. Returns
    q_out, or (q_out, k_out) with k. Not recorded by autograd."""
    if (grid is None) == (positions is None):
        raise ValueError("give either grid or positions")
    if k is None and k_out is not None:
        raise ValueError("k_out goes with k")
    if torch.is_grad_enabled():
        _unrecorded((q, k), (q_out, k_out))
    _on(q, k, positions, q_out, k_out)
    c = _rope(r, _geo(q), None if k is None else _geo(k), None if q_out is None else _geo(q_out),
              None if k_out is None else _geo(k_out),
              None if positions is None else _geo(positions), _ints(grid), _ints(start),
              bool(inverse), layout)
    qo = _new(q) if q_out is None else q_out
    ko = None if k is None else _new(k) if k_out is None else k_out
    _call("ca_rope", q.device, c, q.data_ptr(), _ptr(k), _ptr(positions), qo.data_ptr(), _ptr(ko))
    if q_out is not None or k_out is not None:
        _wrote(q_out, k_out)
    return qo if k is None else (qo, ko)


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

    def __post_init__(self):
        for x in ("left", "right", "sinks"):
            object.__setattr__(self, x, int(getattr(self, x)))
        object.__setattr__(self, "causal", bool(self.causal))


@_kept
def _window(w, q, k, v, out, scale, len_q, len_k, layout, grads):
    """(descriptor, bytes of workspace); grads: of the backward pass, dout and the three
    gradients."""
    dtype = q[2]
    dt = _dtype(dtype)
    (B, H, nq, d), qs = _heads(q, layout, "q", dtype)
    (Bk, Hk, nk, dk), ks = _heads(k, layout, "k", dtype)
    if (Bk, dk) != (B, d):
        raise ValueError("q and k must have the same batch and head dimension")
    vs = _heads(v, layout, "v", dtype, k[0])[1]
    os = _heads(out or _dense(q), layout, "out", dtype, q[0])[1]
    for t, name in ((len_q, "len_q"), (len_k, "len_k")):
        if t is not None:
            _int32(t, name, (B,))
            if t[1][0] != 1 and B > 1:
                raise ValueError(f"{name} must be contiguous")
    gs = ()
    if grads is not None:
        like = (("dout", q), ("dq", q), ("dk", k), ("dv", v))
        gs = tuple(_heads(t or _dense(x), layout, name, dtype, x[0])[1]
                   for t, (name, x) in zip(grads, like))
    c = _lib.CaWindow(B, H, Hk, nq, nk, d, dt, _side(w.left), _side(w.right),
                      _int(min(w.sinks, _MOST), "sinks"), int(w.causal),
                      0.0 if scale is None else scale, qs, ks, vs, os, *gs)
    return c, _bytes("ca_window_workspace_size", c, int(grads is not None))


def _lse_shape(q, layout):
    z = q.shape
    return (z[0], z[2], z[1]) if layout == "bnhd" else (z[0], z[1], z[2])


def window_attn(w: Window, q, k, v, *, scale=None, len_q=None, len_k=None, layout="bhnd",
                want_lse=False, out=None, ws=None):
    """Attention with a sliding window and sinks. q: [B,H,nq,d] ("bhnd",
    "strided") or [B,nq,H,d] ("bnhd"), any strides; k, v the same with nk
    tokens and heads_k heads (a divisor of H). len_q, len_k: int32 [B], the
    lengths in a padded batch. Returns (out, lse [B,H,nq] fp32 or None); rows
    that see no key, and rows past len_q, are 0 with lse -inf. Not recorded by
    autograd; window_attn_backward forms the gradients of out (lse has none)."""
    if torch.is_grad_enabled():
        _unrecorded((q, k, v), (out,))
    _on(q, k, v, out, len_q, len_k)
    c, nbytes = _window(w, _geo(q), _geo(k), _geo(v), None if out is None else _geo(out), _scale(scale),
                        None if len_q is None else _geo(len_q),
                        None if len_k is None else _geo(len_k), layout, None)
    o = _new(q) if out is None else out
    lse = q.new_empty(_lse_shape(q, layout), dtype=torch.float32) if want_lse else None
    ws = _workspace(nbytes, q, ws)
    _call("ca_window_attn", q.device, c, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(len_q),
          _ptr(len_k), o.data_ptr(), _ptr(lse), _ptr(ws), 0 if ws is None else ws.nbytes)
    if out is not None:
        _wrote(out)
    return o, lse


def window_attn_backward(w: Window, dout, q, k, v, out, lse, *, scale=None, len_q=None,
                         len_k=None, layout="bhnd", dq=None, dk=None, dv=None, ws=None):
    """The gradients (dq, dk, dv) of window_attn for the output's gradient
    dout, from out and lse as window_attn gave them for the same arguments.
    dq, dk, dv: outputs of the inputs' shapes (any strides, for example slices
    of a fused projection's gradient), new dense tensors by default."""
    given = dq, dk, dv
    if torch.is_grad_enabled():
        _unrecorded((), given)
    _on(q, k, v, out, lse, dout, len_q, len_k, dq, dk, dv)
    c, nbytes = _window(w, _geo(q), _geo(k), _geo(v), _geo(out), _scale(scale),
                        None if len_q is None else _geo(len_q),
                        None if len_k is None else _geo(len_k), layout,
                        (_geo(dout), *(None if t is None else _geo(t) for t in (dq, dk, dv))))
    if lse.dtype != torch.float32 or not lse.is_contiguous() or \
            tuple(lse.shape) != _lse_shape(q, layout):
        raise ValueError("lse: expected a contiguous fp32 tensor of [B, H, nq]")
    dq, dk, dv = (_new(t) if g is None else g for t, g in ((q, dq), (k, dk), (v, dv)))
    ws = _workspace(nbytes, q, ws)
    _call("ca_window_attn_backward", q.device, c, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          out.data_ptr(), lse.data_ptr(), dout.data_ptr(), _ptr(len_q), _ptr(len_k),
          dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), _ptr(ws), 0 if ws is None else ws.nbytes)
    _wrote(*given)
    return dq, dk, dv


# ---- paged cache -----------------------------------------------------------------------

@_kept
def _paged(k_pages, v_pages, table, lens, batch, heads, left, sinks, scale, q, out, k, v):
    """(descriptor, bytes of workspace) of an append (k, v given) or an attention (q
    given)."""
    dtype = k_pages[2]
    dt = _dtype(dtype)
    (P, page, Hk, d), ks = _rows(k_pages, "k_pages", 4, dtype)
    vs = _rows(v_pages, "v_pages", 4, dtype, k_pages[0])[1]
    if len(table[0]) != 2:
        raise ValueError("page_table: expected [B, max_pages]")
    _int32(table, "page_table", (batch, table[0][1]))
    _int32(lens, "lens", (batch,))
    if (table[1][1] != 1 and table[0][1] > 1) or (lens[1][0] != 1 and batch > 1):
        raise ValueError("lens and the rows of page_table must be contiguous")
    z3, z2 = _I64x3(), _I64x2()
    qs, os, kn, vn, n = z2, z2, z3, z3, 0
    if q is not None:
        size, st = _rows(q, "q", 3, dtype, (batch, heads, d))
        qs, os = _I64x2(*st[:2]), _I64x2(*_rows(out or _dense(q), "out", 3, dtype, q[0])[1][:2])
    else:
        size, st = _rows(k, "k", 4, dtype, (batch, k[0][1], Hk, d))
        n, kn, vn = size[1], _I64x3(*st[:3]), _I64x3(*_rows(v, "v", 4, dtype, k[0])[1][:3])
    c = _lib.CaPaged(batch, heads, Hk, d, dt, page, P, table[0][1], _side(left),
                     _int(min(sinks, _MOST), "sinks"), 0.0 if scale is None else scale,
                     table[1][0] if batch > 1 else 0, _I64x3(*ks[:3]), _I64x3(*vs[:3]), qs, os,
                     n, kn, vn)
    return c, _bytes("ca_paged_workspace_size", c) if q is not None else 0


def cache_append(k, v, k_pages, v_pages, page_table, lens):
    """Writes the new keys and values k, v [B,n,Hk,d] of B sequences into their
    pages: the last n of the lens[b] tokens of sequence b (lens counts them
    already). k_pages, v_pages: [pages, page, Hk, d], any strides;
    page_table: int32 [B, max_pages]; lens: int32 [B]. Returns nothing. Not
    recorded by autograd."""
    if torch.is_grad_enabled():
        _unrecorded((k, v), (k_pages, v_pages))
    _on(k, v, k_pages, v_pages, page_table, lens)
    if k.dim() != 4:
        raise ValueError("k: expected [B, n, Hk, d]")
    c, _ = _paged(_geo(k_pages), _geo(v_pages), _geo(page_table), _geo(lens), k.shape[0],
                  k.shape[2], -1, 0, None, None, None, _geo(k), _geo(v))
    _call("ca_cache_append", k.device, c, k.data_ptr(), v.data_ptr(), k_pages.data_ptr(),
          v_pages.data_ptr(), page_table.data_ptr(), lens.data_ptr())
    _wrote(k_pages, v_pages)


def paged_attn(q, k_pages, v_pages, page_table, lens, *, left=-1, sinks=0, scale=None,
               want_lse=False, out=None, ws=None):
    """Attention of one new token of each sequence, its last one, over the
    sequence's cached keys: all of them, or with left >= 0 the last left + 1
    and the first `sinks`. q: [B,H,d]; k_pages, v_pages: [pages, page, Hk, d],
    any strides, Hk a divisor of H; page_table: int32 [B, max_pages]; lens:
    int32 [B], the new token included. Returns (out [B,H,d], lse [B,H] fp32 or
    None); a sequence of no tokens gives 0 and -inf. The workspace goes with
    the table's width, not the lengths. Not recorded by autograd, and without a
    backward pass."""
    if torch.is_grad_enabled():
        _unrecorded((q, k_pages, v_pages), (out,))
    _on(q, k_pages, v_pages, page_table, lens, out)
    if q.dim() != 3:
        raise ValueError("q: expected [B, H, d]")
    B, H, _ = q.shape
    c, nbytes = _paged(_geo(k_pages), _geo(v_pages), _geo(page_table), _geo(lens), B, H, int(left),
                       int(sinks), _scale(scale), _geo(q), None if out is None else _geo(out), None, None)
    o = _new(q) if out is None else out
    lse = q.new_empty((B, H), dtype=torch.float32) if want_lse else None
    ws = _workspace(nbytes, q, ws)
    _call("ca_paged_attn", q.device, c, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
          page_table.data_ptr(), lens.data_ptr(), o.data_ptr(), _ptr(lse), _ptr(ws),
          0 if ws is None else ws.nbytes)
    if out is not None:
        _wrote(out)
    return o, lse
