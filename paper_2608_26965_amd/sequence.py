"""The sequence operators of libclusterattn: rotary positions of several axes,
attention with a sliding window and sinks and its gradients, and the paged
key-value cache with the attention of one new token or of chunks of them (see
include/clusterattn.h for their definitions).

    rope                              turn queries and keys by their positions
    window_attn, window_attn_backward
    cache_append, paged_attn          serving: write new tokens, attend over the pages
    cache_grow, cache_release         pages for the new tokens of a step, and back
    cache_write, paged_chunk_attn     packed new tokens: write them by slots, attend

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
from typing import NamedTuple

import torch
from torch.autograd import forward_ad

from . import _lib
from ._lib import CA_BF16, CA_F32

__all__ = ["Rope", "rope_axes", "rope", "Window", "window_attn", "window_attn_backward",
           "cache_append", "paged_attn", "PagePool", "page_pool", "CacheStep", "cache_grow",
           "cache_release", "cache_write", "paged_chunk_attn"]

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


def _recording():
    """Whether autograd records, backwards or forwards."""
    return torch.is_grad_enabled() or forward_ad._current_level >= 0


def _tangent(t):
    return t is not None and forward_ad.unpack_dual(t).tangent is not None


def _unrecorded(read, written, gradients=()):
    """Where autograd records, tells what the call does not do. gradients: also read, by a call that
    is a backward pass itself."""
    if torch.is_grad_enabled():
        for t in written:
            if t is not None and t.requires_grad:
                raise ValueError("the call would write a tensor that requires gradients, unrecorded by "
                                 "autograd: give it detached, or call under torch.no_grad()")
        for t in read:
            if t is not None and t.requires_grad:
                warnings.warn("not recorded by autograd: no gradient reaches the inputs that require one "
                              "(window_attn_backward and rope with inverse=True form them)", stacklevel=3)
                break
    if forward_ad._current_level >= 0:
        if any(map(_tangent, written)):
            raise ValueError("the call would write a tensor that has a tangent, which it would leave as it "
                             "is: give the tensor's primal")
        if any(map(_tangent, (*read, *gradients))):
            warnings.warn("not recorded by autograd: the tangents of the inputs do not reach the results",
                          stacklevel=3)


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
    if _recording():
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
    if _recording():
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
    if _recording():
        _unrecorded((), given, (dout, q, k, v, out, lse))
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
    if _recording():
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
    if _recording():
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


# ---- chunks of new tokens over the paged cache -------------------------------------------

@dataclass(frozen=True)
class PagePool:
    """The pages of `page` tokens that no sequence holds: free, int32 [pages],
    of which the first state[0] are free pages (a stack, the next one to be taken
    last); state, int32 [3]: free pages, pages that the last cache_grow lacked, new
    tokens for which it had no rows. page_pool makes one of a whole pool."""
    page: int
    free: torch.Tensor
    state: torch.Tensor

    def __post_init__(self):
        object.__setattr__(self, "page", int(self.page))

    @property
    def pages(self):
        return self.free.shape[0]


def page_pool(pages, page, device="cuda") -> PagePool:
    """A PagePool of `pages` pages, all free; page 0 is taken first."""
    pages = _int(pages, "pages", 1)
    return PagePool(_int(page, "page", 1),
                    torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=device),
                    torch.tensor([pages, 0, 0], dtype=torch.int32, device=device))


class CacheStep(NamedTuple):
    """Where a step's new tokens lie, packed: sequence b's in rows starts[b] ..
    starts[b + 1] - 1. starts: int32 [B + 1]; slots: int64 [tokens], places in the
    pools (-1: none); positions: int32 [1, tokens], places in the sequences, as
    rope takes them."""
    starts: torch.Tensor
    slots: torch.Tensor
    positions: torch.Tensor


@_kept
def _pages(page, free, state, table, lens, new, tokens, left, sinks, out, seen=None):
    """(descriptor, bytes of workspace) of a cache_grow (new given) or a
    cache_release."""
    if len(free[0]) != 1 or free[1][0] != 1:
        raise ValueError("pool.free: expected a contiguous [pages]")
    _int32(free, "pool.free", free[0])
    _int32(state, "pool.state", (3,))
    if len(table[0]) != 2:
        raise ValueError("page_table: expected [B, max_pages]")
    batch, width = table[0]
    _int32(table, "page_table", (batch, width))
    _int32(lens, "lens", (batch,))
    if state[1][0] != 1 or (table[1][1] != 1 and width > 1) or (lens[1][0] != 1 and batch > 1):
        raise ValueError("pool.state, lens and the rows of page_table must be contiguous")
    if new is not None:
        _int32(new, "new", (batch,))
        if new[1][0] != 1 and batch > 1:
            raise ValueError("new must be contiguous")
        if seen is not None:
            _int32(seen, "seen", (batch,))
            if seen[1][0] != 1 and batch > 1:
                raise ValueError("seen must be contiguous")
        if out is not None:
            starts, slots, positions = out
            _int32(starts, "out.starts", (batch + 1,))
            _int32(positions, "out.positions", (1, tokens))
            if slots[2] != torch.int64 or tuple(slots[0]) != (tokens,):
                raise ValueError(f"out.slots: expected int64 [{tokens}]")
            if starts[1][0] != 1 or (tokens > 1 and (slots[1][0] != 1 or positions[1][1] != 1)):
                raise ValueError("out: expected contiguous tensors")
    c = _lib.CaPages(batch, _int(page, "page"), free[0][0], width, tokens, _side(left),
                     _int(min(sinks, _MOST), "sinks"), table[1][0] if batch > 1 else 0)
    return c, _bytes("ca_cache_release_workspace_size", c) if new is None else 0


def cache_grow(pool: PagePool, page_table, lens, new, tokens, *, seen=None, out=None) -> CacheStep:
    """Pages for the new tokens of a step, and where they go. page_table: int32
    [B, max_pages], changed in place; lens: int32 [B], the sequences' tokens, the
    new ones, the last new[b] of them (int32 [B]), included; tokens: rows of the
    packed arrays, at least the sum of `new` (the program knows it, or a bound for
    arrays of a fixed size). Entries that a new token lies on and that hold no page
    (-1, or any value outside the pool) get one; entries that hold one stay, so pages
    that rows share (a common beginning) have to be full: sequences that go on inside
    one would write over each other. Where the pool runs short the entries stay, their
    tokens have slot -1, and pool.state[1] says how many pages lacked; those tokens are
    not there for the step's attention, and a later step has to bring them again.
    Repeating the call changes nothing. Returns CacheStep, in `out` (one of an earlier call of the
    same sizes) if given; rows behind the last sequence have slot -1 and position 0.

    Where the sum of `new` may pass `tokens` (pool.state[2] says by how much), the last
    sequences have rows for the first of their new tokens only, or none, and lens
    counts tokens that this step does not write. seen (int32 [B], written if given)
    then holds lens as far as the rows go: give it to paged_chunk_attn and cache_release
    in the place of lens (with lens itself the attention would take the rows of the
    sequence that is cut for its last tokens), and go on from it in the next step."""
    tokens = _int(tokens, "tokens", 1)
    if seen is not None and seen.data_ptr() in (lens.data_ptr(), new.data_ptr()):
        raise ValueError("seen: expected a tensor of its own (lens and new are read after it is written)")
    _on_ints(pool.free, pool.state, page_table, lens, new, *(out or ()), *(() if seen is None else (seen,)))
    c, _ = _pages(pool.page, _geo(pool.free), _geo(pool.state), _geo(page_table), _geo(lens), _geo(new),
                  tokens, -1, 0, None if out is None else tuple(_geo(t) for t in out),
                  None if seen is None else _geo(seen))
    if out is None:
        out = CacheStep(lens.new_empty(lens.shape[0] + 1), lens.new_empty(tokens, dtype=torch.int64),
                        lens.new_empty((1, tokens)))
    starts, slots, positions = out
    args = (lens.device, c, lens.data_ptr(), new.data_ptr(), page_table.data_ptr(), pool.free.data_ptr(),
            pool.state.data_ptr(), starts.data_ptr(), slots.data_ptr(), positions.data_ptr())
    if seen is None:
        _call("ca_cache_grow", *args)
    else:
        _call("ca_cache_grow_seen", *args, seen.data_ptr())
    _wrote(page_table, pool.state, starts, slots, positions, seen)
    return CacheStep(starts, slots, positions)


def cache_release(pool: PagePool, page_table, lens, *, left=-1, sinks=0, ws=None):
    """Gives the pages back that hold none of a sequence's lens[b] tokens, or with
    left >= 0 none that its next token sees with that window (the last `left` and
    the first `sinks`): all of a finished sequence (lens 0), those of
    rejected tokens (lens less than it was), those behind a window. Their entries
    become -1. page_table: int32 [B, max_pages], changed in place. A page that
    several rows share must not go back from two of them, nor from one while another
    holds it. Returns nothing."""
    _on_ints(pool.free, pool.state, page_table, lens)
    c, nbytes = _pages(pool.page, _geo(pool.free), _geo(pool.state), _geo(page_table), _geo(lens), None,
                       0, int(left), int(sinks), None)
    ws = _workspace(nbytes, lens, ws)
    _call("ca_cache_release", lens.device, c, lens.data_ptr(), page_table.data_ptr(),
          pool.free.data_ptr(), pool.state.data_ptr(), _ptr(ws), 0 if ws is None else ws.nbytes)
    _wrote(page_table, pool.free, pool.state)


def _on_ints(like, *tensors):
    """All on one GPU."""
    if not like.is_cuda:
        raise ValueError("expected tensors on the GPU")
    i = like.get_device()
    for t in tensors:
        if t.get_device() != i:
            raise ValueError(f"expected all tensors on {like.device}, got one on {t.device}")


@_kept
def _chunk(k_pages, v_pages, w, table, lens, starts, q, out, scale, k, v, slots):
    """(descriptor, bytes of workspace) of a cache_write (k, v and slots given) or an
    attention (w, table, lens, starts and q given)."""
    dtype = k_pages[2]
    dt = _dtype(dtype)
    (P, page, Hk, d), ks = _rows(k_pages, "k_pages", 4, dtype)
    vs = _rows(v_pages, "v_pages", 4, dtype, k_pages[0])[1]
    ks, vs, z = _I64x3(*ks[:3]), _I64x3(*vs[:3]), _I64x2()
    if k is not None:
        (T, h, x), kn = _rows(k, "k", 3, dtype)
        if (h, x) != (Hk, d):
            raise ValueError(f"k: expected shape [T, {Hk}, {d}], got {[T, h, x]}")
        vn = _rows(v, "v", 3, dtype, k[0])[1]
        if slots[2] != torch.int64 or tuple(slots[0]) != (T,) or (slots[1][0] != 1 and T > 1):
            raise ValueError(f"slots: expected a contiguous int64 tensor of [{T}]")
        return _lib.CaChunk(1, Hk, Hk, d, dt, page, P, 1, T, -1, -1, 0, 0, 0.0, 0, ks, vs, z, z,
                            _I64x2(*kn[:2]), _I64x2(*vn[:2])), 0
    (T, H, x), qs = _rows(q, "q", 3, dtype)
    if x != d:
        raise ValueError(f"q: expected a last dimension of {d}, got {x}")
    os = _rows(out or _dense(q), "out", 3, dtype, q[0])[1]
    if len(table[0]) != 2:
        raise ValueError("page_table: expected [B, max_pages]")
    B, width = table[0]
    _int32(table, "page_table", (B, width))
    _int32(lens, "lens", (B,))
    _int32(starts, "starts", (B + 1,))
    if (table[1][1] != 1 and width > 1) or (lens[1][0] != 1 and B > 1) or starts[1][0] != 1:
        raise ValueError("lens, starts and the rows of page_table must be contiguous")
    c = _lib.CaChunk(B, H, Hk, d, dt, page, P, width, T, _side(w.left), _side(w.right),
                     _int(min(w.sinks, _MOST), "sinks"), int(w.causal), 0.0 if scale is None else scale,
                     table[1][0] if B > 1 else 0, ks, vs, _I64x2(*qs[:2]), _I64x2(*os[:2]), z, z)
    return c, _bytes("ca_paged_chunk_workspace_size", c)


def cache_write(k, v, k_pages, v_pages, slots):
    """Writes the packed new keys and values k, v [T,Hk,d] (any strides) to their
    slots (int64 [T], as cache_grow gives them: page * its index + place in the
    page); rows with a slot outside the pools are left out, no two rows may have the
    same one. k_pages, v_pages: [pages, page, Hk, d], any strides. Returns nothing. Not
    recorded by autograd."""
    if _recording():
        _unrecorded((k, v), (k_pages, v_pages))
    _on(k, v, k_pages, v_pages, slots)
    c, _ = _chunk(_geo(k_pages), _geo(v_pages), None, None, None, None, None, None, None, _geo(k), _geo(v),
                  _geo(slots))
    _call("ca_cache_write", k.device, c, k.data_ptr(), v.data_ptr(), k_pages.data_ptr(),
          v_pages.data_ptr(), slots.data_ptr())
    _wrote(k_pages, v_pages)


def paged_chunk_attn(w: Window, q, k_pages, v_pages, page_table, lens, starts, *, scale=None,
                     want_lse=False, out=None, lse=None, ws=None):
    """Attention of the new tokens of each sequence, any number of them, over the
    sequence's cached keys, the new tokens' own (written before) included. q:
    [T,H,d] packed, any strides, rows starts[b] .. starts[b + 1] - 1 those of the
    last tokens of sequence b (starts: int32 [B + 1]); lens: int32 [B], all tokens of
    the sequences; k_pages, v_pages: [pages, page, Hk, d], any strides, Hk a
    divisor of H; page_table: int32 [B, max_pages]. Who sees whom is w, as in
    window_attn: Window(causal=True) for text, Window() where the new tokens see each
    other. Returns (out [T,H,d], lse [T,H] fp32 or None); a query that sees no key has
    0 and -inf. Rows before the first and behind the last sequence are left as they were
    (in new tensors: as they come). out may be q itself. Not recorded by autograd, and without a backward pass."""
    if _recording():
        _unrecorded((q, k_pages, v_pages), (out, lse))
    _on(q, k_pages, v_pages, page_table, lens, starts, out, lse)
    if q.dim() != 3:
        raise ValueError("q: expected [T, H, d]")
    c, nbytes = _chunk(_geo(k_pages), _geo(v_pages), w, _geo(page_table), _geo(lens), _geo(starts), _geo(q),
                       None if out is None else _geo(out), _scale(scale), None, None, None)
    if lse is not None and (lse.dtype != torch.float32 or lse.shape != q.shape[:2] or
                            not lse.is_contiguous()):
        raise ValueError(f"lse: expected a contiguous fp32 tensor of {list(q.shape[:2])}")
    o = _new(q) if out is None else out
    z = q.new_empty(q.shape[:2], dtype=torch.float32) if lse is None and want_lse else lse
    ws = _workspace(nbytes, q, ws)
    _call("ca_paged_chunk_attn", q.device, c, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
          page_table.data_ptr(), lens.data_ptr(), starts.data_ptr(), o.data_ptr(), _ptr(z), _ptr(ws),
          0 if ws is None else ws.nbytes)
    if out is not None or lse is not None:
        _wrote(out, lse)
    return o, z
