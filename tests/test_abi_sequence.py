"""Refusals of the sequence operators, before anything is enqueued: the C
entry points with addresses that are never dereferenced, and the binding with
CPU tensors. No GPU needed."""
import ctypes

import pytest


def _lib():
    from paper_2608_26965_amd import _lib as L
    try:
        return L, L.load()
    except ImportError as e:  # pragma: no cover
        pytest.skip(str(e))


I3, I2, I4 = ctypes.c_int64 * 3, ctypes.c_int64 * 2, ctypes.c_int32 * 4
FAKE = 256


def _rope(**kw):
    from paper_2608_26965_amd import _lib as L
    st = I3(4 * 8 * 64, 8 * 64, 64)
    c = L.CaRope(batch=2, heads=4, heads_k=4, n=8, d=64, dtype=L.CA_BF16, axes=2, section=I4(16, 16), halves=0,
                 inverse=0, grid=I4(2, 4), start=I4(), pos_stride=I3(), q_stride=st, k_stride=st, q_out_stride=st,
                 k_out_stride=st, freq=(ctypes.c_double * 64)(*([0.5] * 64)))
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("kw,status,word", [
    (dict(dtype=9), 1, "dtype"), (dict(batch=0), 1, "batch"), (dict(heads=0), 1, "heads"), (dict(n=0), 1, "n must"),
    (dict(d=0), 1, "d must"), (dict(d=136), 1, "d must"), (dict(d=36), 2, "multiple"), (dict(axes=0), 1, "axes"),
    (dict(axes=5), 1, "axes"), (dict(section=I4(-1, 4)), 1, "section"), (dict(section=I4(0, 0)), 1, "section"),
    (dict(section=I4(16, 17)), 1, "section"), (dict(section=I4(2, 2), halves=1), 2, "halves"),
    (dict(grid=I4(2, 3)), 1, "grid"), (dict(grid=I4(0, 9)), 1, "grid"), (dict(start=I4(2**31 - 1)), 1, "start"),
    (dict(freq=(ctypes.c_double * 64)(float("nan"))), 1, "freq"), (dict(freq=(ctypes.c_double * 64)(1e9)), 1, "freq"), (dict(q_stride=I3(64, 64, 4)), 1, "q_stride[2]"),
    (dict(q_stride=I3(-64, 64, 64)), 1, "q_stride[0]"), (dict(k_stride=I3(64, 4, 64)), 1, "k_stride[1]"),
    (dict(q_out_stride=I3(2048, 0, 64)), 1, "q_out_stride[1]"), (dict(k_out_stride=I3(2048, 512, 0)), 1, "k_out_stride"),
])
def test_rope_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_rope(_rope(**kw), FAKE, FAKE, None, FAKE, FAKE, None) == status
    assert word in L.last_error()


def test_rope_pointers():
    L, lib = _lib()
    assert lib.ca_rope(None, FAKE, FAKE, None, FAKE, FAKE, None) == L.CA_E_INVALID
    for args in ((None, FAKE, FAKE, FAKE), (FAKE, None, FAKE, FAKE), (FAKE, FAKE, None, FAKE), (FAKE, FAKE, FAKE, None),
                 (FAKE + 8, FAKE, FAKE, FAKE), (FAKE, FAKE + 8, FAKE, FAKE), (FAKE, FAKE, FAKE + 8, FAKE),
                 (FAKE, FAKE, FAKE, FAKE + 8)):
        assert lib.ca_rope(_rope(), args[0], args[1], None, args[2], args[3], None) == L.CA_E_INVALID
    # given positions need no grid, but everything else
    assert lib.ca_rope(_rope(grid=I4(), dtype=7), FAKE, FAKE, FAKE, FAKE, FAKE, None) == L.CA_E_INVALID


def _window(**kw):
    from paper_2608_26965_amd import _lib as L
    st, sk = I3(8 * 100 * 64, 100 * 64, 64), I3(2 * 100 * 64, 100 * 64, 64)
    c = L.CaWindow(batch=2, heads=8, heads_k=2, nq=100, nk=100, d=64, dtype=L.CA_BF16, left=-1, right=-1, sinks=0,
                   causal=0, scale=0.0, q_stride=st, k_stride=sk, v_stride=sk, out_stride=st, dout_stride=st,
                   dq_stride=st, dk_stride=sk, dv_stride=sk)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


_BAD_WINDOW = [
    (dict(dtype=2), 1, "dtype"), (dict(heads_k=3), 1, "multiple of heads_k"), (dict(heads_k=0), 1, "heads_k"),
    (dict(batch=0), 1, "batch"), (dict(nq=0), 1, "nq"), (dict(nk=0), 1, "nk"), (dict(nk=(1 << 22) + 1), 1, "2^22"),
    (dict(d=96), 2, "64, 128"), (dict(d=192), 1, "d must"), (dict(dtype=0, d=62), 2, "fp32"), (dict(sinks=-1), 1, "sinks"),
    (dict(batch=8192), 2, "65535"), (dict(q_stride=I3(64, 64, 4)), 1, "q_stride[2]"),
    (dict(v_stride=I3(64, 4, 64)), 1, "v_stride[1]"), (dict(k_stride=I3(64, 64, 1 << 24)), 2, "2^23"),
    (dict(batch=1000, heads=64, nq=1 << 22), 2, "too large"), (dict(out_stride=I3(-64, 64, 64)), 1, "out_stride[0]"),
]


@pytest.mark.parametrize("kw,status,word", _BAD_WINDOW + [(dict(out_stride=I3(51200, 0, 64)), 1, "out_stride[1]")])
def test_window_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_window_attn(_window(**kw), FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, 1 << 40, None) == status
    assert word in L.last_error()


@pytest.mark.parametrize("kw,status,word", _BAD_WINDOW + [
    (dict(dout_stride=I3(64, 64, 4)), 1, "dout_stride"), (dict(dout_stride=I3(64, 64, 1 << 24)), 2, "2^23"), (dict(dq_stride=I3(64, 64, 0)), 1, "dq_stride[2]"),
    (dict(dk_stride=I3(0, 64, 64)), 1, "dk_stride[0]"), (dict(dv_stride=I3(64, 0, 64)), 1, "dv_stride[1]"),
])
def test_window_backward_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_window_attn_backward(_window(**kw), *[FAKE] * 6, None, None, FAKE, FAKE, FAKE, FAKE, 1 << 40,
                                       None) == status
    assert word in L.last_error()


def test_window_pointers_and_workspace():
    L, lib = _lib()
    n = ctypes.c_size_t(0)
    assert lib.ca_window_workspace_size(None, 0, n) == L.CA_E_INVALID
    assert lib.ca_window_workspace_size(_window(nk=100000), 0, n) == L.CA_OK and n.value > 0
    assert lib.ca_window_attn(_window(nk=100000), FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, n.value - 1, None) == \
        L.CA_E_WORKSPACE
    assert lib.ca_window_workspace_size(_window(), 1, n) == L.CA_OK and n.value >= 2 * 8 * 100 * 4
    for i in range(4):
        a = [FAKE, FAKE, FAKE, FAKE]
        for bad in (None, FAKE + 2):
            a[i] = bad
            assert lib.ca_window_attn(_window(), *a[:3], None, None, a[3], None, FAKE, n.value, None) == L.CA_E_INVALID
    for i in range(9):
        a = [FAKE] * 9
        a[i] = None
        assert lib.ca_window_attn_backward(_window(), *a[:6], None, None, *a[6:], FAKE, n.value, None) == L.CA_E_INVALID
    assert lib.ca_window_attn_backward(_window(), *[FAKE] * 6, None, None, *[FAKE] * 4, n.value - 1, None) == \
        L.CA_E_WORKSPACE
    assert lib.ca_window_attn_backward(_window(), *[FAKE] * 6, None, None, *[FAKE] * 3, None, n.value, None) == \
        L.CA_E_INVALID
    assert lib.ca_window_attn_backward(_window(), *[FAKE] * 6, None, None, *[FAKE] * 3, FAKE + 16, n.value, None) == \
        L.CA_E_INVALID


def _paged(**kw):
    from paper_2608_26965_amd import _lib as L
    st = I3(16 * 2 * 64, 2 * 64, 64)
    c = L.CaPaged(batch=2, heads=8, heads_k=2, d=64, dtype=L.CA_BF16, page=16, pages=10, max_pages=4, left=-1, sinks=0,
                  scale=0.0, table_stride=4, k_stride=st, v_stride=st, q_stride=I2(512, 64), out_stride=I2(512, 64),
                  n_new=1, k_new_stride=I3(128, 128, 64), v_new_stride=I3(128, 128, 64))
    for k, v in kw.items():
        setattr(c, k, v)
    return c


_BAD_PAGED = [
    (dict(dtype=5), 1, "dtype"), (dict(heads_k=3), 1, "heads_k"), (dict(d=80), 2, "64, 128"), (dict(page=0), 1, "page"),
    (dict(pages=0), 1, "pages"), (dict(max_pages=0), 1, "max_pages"), (dict(page=1 << 20, max_pages=1 << 10), 2, "2^30"),
    (dict(table_stride=-1), 1, "table_stride"), (dict(k_stride=I3(2048, 128, 4)), 1, "k_stride[2]"),
    (dict(v_stride=I3(2044, 128, 64)), 1, "v_stride[0]"),
]


@pytest.mark.parametrize("kw,status,word", _BAD_PAGED + [
    (dict(sinks=-2), 1, "sinks"), (dict(q_stride=I2(512, 4)), 1, "q_stride[1]"), (dict(out_stride=I2(0, 64)), 1, "overlap"),
])
def test_paged_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_paged_attn(_paged(**kw), *[FAKE] * 6, None, FAKE, 1 << 40, None) == status
    assert word in L.last_error()


@pytest.mark.parametrize("kw,status,word", _BAD_PAGED + [
    (dict(n_new=0), 1, "n_new"), (dict(k_new_stride=I3(128, 128, 4)), 1, "k_new_stride[2]"),
    (dict(v_new_stride=I3(128, -8, 64)), 1, "v_new_stride[1]"), (dict(k_stride=I3(0, 128, 64)), 1, "k_stride[0]"),
    (dict(v_stride=I3(2048, 0, 64)), 1, "v_stride[1]"),
])
def test_append_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_cache_append(_paged(**kw), *[FAKE] * 6, None) == status
    assert word in L.last_error()


def test_paged_pointers_and_workspace():
    L, lib = _lib()
    n = ctypes.c_size_t(0)
    assert lib.ca_paged_workspace_size(_paged(max_pages=4096), n) == L.CA_OK and n.value > 0
    big = _paged(max_pages=4096)
    for i in range(6):
        a = [FAKE] * 6
        a[i] = None
        assert lib.ca_paged_attn(big, *a, None, FAKE, n.value, None) == L.CA_E_INVALID
        assert lib.ca_cache_append(_paged(), *a, None) == L.CA_E_INVALID
    assert lib.ca_paged_attn(big, *[FAKE] * 6, None, FAKE, n.value - 1, None) == L.CA_E_WORKSPACE
    assert lib.ca_paged_attn(big, *[FAKE] * 6, None, None, n.value, None) == L.CA_E_INVALID


def test_binding_refuses_cpu_tensors_and_shapes():
    import torch
    import paper_2608_26965_amd as ca
    x = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    r = ca.rope_axes((32, 32))
    with pytest.raises(ValueError, match="GPU"):
        ca.rope(r, x, grid=(2, 2))
    with pytest.raises(ValueError, match="GPU"):
        ca.window_attn(ca.Window(), x, x, x)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ca.window_attn(ca.Window(), x.half(), x.half(), x.half())
    with pytest.raises(ValueError):
        ca.rope_axes((31, 33))
    with pytest.raises(ValueError):
        ca.Rope((2, 2), (1.0, 2.0, 3.0))
    with pytest.raises(ValueError):
        ca.Rope((2,), (1.0, 2.0), "pairs")
    with pytest.raises(ValueError, match="sections"):
        ca.Rope((2 ** 32 + 2, -2 ** 32), (1.0, 2.0))


def test_numbers_given_as_tensors_become_numbers():
    import torch
    import paper_2608_26965_amd as ca
    t = torch.tensor(3)
    w, r = ca.Window(left=t, sinks=t, causal=t), ca.Rope(torch.tensor([2, 1]), torch.tensor([1.0, 0.5, 0.25]))
    t.fill_(7)
    assert w == ca.Window(left=3, sinks=3, causal=True) and hash(w) == hash(ca.Window(3, -1, 3, True))
    assert r == ca.Rope((2, 1), (1.0, 0.5, 0.25)) and hash(r) == hash(ca.Rope((2, 1), (1.0, 0.5, 0.25)))


@pytest.mark.parametrize("kw", [{"rope_grid": (2, 2)}, {"rope_positions": 1}])
def test_forward_refuses_positions_without_rotary(kw):
    import torch
    import paper_2608_26965_amd as ca
    x = torch.zeros(1, 2, 4, 64)
    with pytest.raises(ValueError, match="go with rotary"):
        ca.forward(x, x, x, keep=0.5, **kw)


@pytest.mark.parametrize("call", [
    lambda ca, x: ca.rope(ca.rope_axes((32, 32)), x, grid=(2, 2)),
    lambda ca, x: ca.window_attn(ca.Window(), x, x, x),
    lambda ca, x: ca.cache_append(x, x, x.detach(), x.detach(), x.detach(), x.detach()),
    lambda ca, x: ca.paged_attn(x, x, x, x, x)])
def test_inputs_that_require_gradients_give_a_warning(call):
    """And the refusal of tensors off the GPU that the call gets without."""
    import warnings
    import torch
    import paper_2608_26965_amd as ca
    x = torch.zeros(1, 2, 4, 64, requires_grad=True)
    with pytest.warns(UserWarning, match="not recorded by autograd"), pytest.raises(ValueError, match="GPU"):
        call(ca, x)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with pytest.raises(ValueError, match="GPU"):
            call(ca, x.detach())
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call(ca, x)


@pytest.mark.parametrize("call", [
    lambda ca, x, y: ca.rope(ca.rope_axes((32, 32)), x, grid=(2, 2), q_out=y),
    lambda ca, x, y: ca.rope(ca.rope_axes((32, 32)), x, x, grid=(2, 2), k_out=y),
    lambda ca, x, y: ca.window_attn(ca.Window(), x, x, x, out=y),
    lambda ca, x, y: ca.window_attn_backward(ca.Window(), x, x, x, x, x, x, dk=y),
    lambda ca, x, y: ca.cache_append(x, x, x, y, x, x),
    lambda ca, x, y: ca.paged_attn(x, x, x, x, x, out=y)])
def test_tensors_that_require_gradients_are_not_written(call):
    import torch
    import paper_2608_26965_amd as ca
    x, y = torch.zeros(1, 2, 4, 64), torch.zeros(1, 2, 4, 64, requires_grad=True)
    for z in (y, y[:]):  # a leaf, and a view of one
        with pytest.raises(ValueError, match="requires gradients"):
            call(ca, x, z)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
        call(ca, x, y)


def test_rope_refuses_an_output_for_keys_that_are_not_given():
    import torch
    import paper_2608_26965_amd as ca
    x = torch.zeros(1, 2, 4, 64)
    with pytest.raises(ValueError, match="k_out goes with k"):
        ca.rope(ca.rope_axes((32, 32)), x, grid=(2, 2), k_out=x)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_window_backward_workspace_holds_cut_blocks_only(dt):
    """Two dense rows of 2^16 tokens a head, 16 sinks: partial sums of the keys' block that holds
    the sinks (of one block of 16 to 128 keys, at most 64 parts), not of every block."""
    L, lib = _lib()
    n = ctypes.c_size_t(0)
    N, H = 1 << 16, 4
    st = I3(H * N * 64, N * 64, 64)
    w = _window(dtype=L.CA_F32 if dt == "f32" else L.CA_BF16, batch=1, heads=H, heads_k=H, nq=N, nk=N, left=100, causal=1,
                sinks=16, **{x + "_stride": st for x in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")})
    assert lib.ca_window_workspace_size(w, 1, n) == L.CA_OK
    rows = 2 * H * N * 4  # at most two numbers a query
    assert n.value <= rows + H * 64 * 128 * 2 * 64 * 4 + 4096
    w.sinks = 0
    assert lib.ca_window_workspace_size(w, 1, n) == L.CA_OK and n.value <= rows + 4096
