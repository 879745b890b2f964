"""Tensors with tangents (forward-mode derivatives) given to the sequence calls: told that the tangents end
there, also under no_grad, which does not end them; written ones are refused. No GPU needed: the calls refuse the
CPU tensors afterwards."""
import warnings

import pytest


def _calls():
    import torch
    import paper_2608_26965_amd as ca
    x, pool = torch.zeros(2, 3, 4, 64), torch.zeros(3, 16, 3, 64)
    table, lens, starts = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    slots, lse = torch.zeros(2, dtype=torch.int64), torch.zeros(2, 3, 4)
    r, w = ca.rope_axes((64,)), ca.Window()
    rows = torch.zeros(2, 3, 64)
    # (call of the tensor under test, that tensor without a tangent)
    read = [(lambda t: ca.rope(r, t, grid=(4,)), x), (lambda t: ca.rope(r, x, t, grid=(4,)), x),
            (lambda t: ca.window_attn(w, x, t, x), x), (lambda t: ca.window_attn_backward(w, t, x, x, x, x, lse), x),
            (lambda t: ca.window_attn_backward(w, x, x, x, t, x, lse), x), (lambda t: ca.cache_append(t, x, pool, pool, table, lens), x),
            (lambda t: ca.paged_attn(rows, t, pool, table, lens), pool), (lambda t: ca.cache_write(rows, t, pool, pool, slots), rows),
            (lambda t: ca.paged_chunk_attn(w, t, pool, pool, table, lens, starts), rows),
            (lambda t: ca.paged_chunk_attn(w, rows, pool, t, table, lens, starts), pool)]
    written = [(lambda t: ca.rope(r, x, grid=(4,), q_out=t), x), (lambda t: ca.window_attn(w, x, x, x, out=t), x),
               (lambda t: ca.window_attn_backward(w, x, x, x, x, x, lse, dk=t), x),
               (lambda t: ca.cache_append(x, x, pool, t, table, lens), pool), (lambda t: ca.paged_attn(rows, pool, pool, table, lens, out=t), rows),
               (lambda t: ca.cache_write(rows, rows, t, pool, slots), pool),
               (lambda t: ca.paged_chunk_attn(w, rows, pool, pool, table, lens, starts, out=t), rows)]
    return read, written


@pytest.mark.parametrize("grad", [True, False])
def test_tangents_that_would_be_lost(grad):
    import torch
    from torch.autograd import forward_ad as fw
    read, written = _calls()
    with torch.set_grad_enabled(grad):
        for call, t in read:
            with fw.dual_level():
                with pytest.warns(UserWarning, match="tangents"), pytest.raises(ValueError, match="GPU"):
                    call(fw.make_dual(t, torch.ones_like(t)))
                with warnings.catch_warnings(), pytest.raises(ValueError, match="GPU"):
                    warnings.simplefilter("error")
                    call(t)
        for call, t in written:
            with fw.dual_level(), pytest.raises(ValueError, match="tangent"):
                call(fw.make_dual(t, torch.ones_like(t)))
