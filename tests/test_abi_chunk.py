"""Refusals of the calls of chunks over the paged cache, before anything is enqueued: the C entry
points with addresses that are never dereferenced, and the binding with CPU tensors. No GPU
needed."""
import ctypes

import pytest


def _lib():
    from paper_2608_26965_amd import _lib as L
    try:
        return L, L.load()
    except ImportError as e:  # pragma: no cover
        pytest.skip(str(e))


I3, I2 = ctypes.c_int64 * 3, ctypes.c_int64 * 2
FAKE = 256


def _pages(**kw):
    from paper_2608_26965_amd import _lib as L
    c = L.CaPages(batch=3, page=16, pages=20, max_pages=5, tokens=9, left=-1, sinks=0, table_stride=5)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


_BAD_PAGES = [
    (dict(batch=0), 1, "batch"), (dict(batch=65536), 2, "65535"), (dict(page=0), 1, "page"), (dict(pages=0), 1, "pages"),
    (dict(max_pages=0), 1, "max_pages"), (dict(page=1 << 20, max_pages=1 << 10), 2, "2^30"),
    (dict(table_stride=4), 1, "table_stride"), (dict(table_stride=-5), 1, "table_stride"),
]


@pytest.mark.parametrize("kw,status,word", _BAD_PAGES + [(dict(tokens=0), 1, "tokens"), (dict(tokens=1 << 25), 1, "2^24")])
def test_grow_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_cache_grow(_pages(**kw), *[FAKE] * 8, None) == status
    assert word in L.last_error()


@pytest.mark.parametrize("kw,status,word", _BAD_PAGES + [(dict(sinks=-1), 1, "sinks")])
def test_release_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_cache_release(_pages(**kw), *[FAKE] * 5, 1 << 30, None) == status
    assert word in L.last_error()


def test_pages_pointers_and_workspace():
    L, lib = _lib()
    n = ctypes.c_size_t(0)
    assert lib.ca_cache_grow(None, *[FAKE] * 8, None) == L.CA_E_INVALID
    for i in range(8):
        a = [FAKE] * 8
        a[i] = None
        assert lib.ca_cache_grow(_pages(), *a, None) == L.CA_E_INVALID
    assert lib.ca_cache_release_workspace_size(None, n) == L.CA_E_INVALID
    assert lib.ca_cache_release_workspace_size(_pages(), None) == L.CA_E_INVALID
    assert lib.ca_cache_release_workspace_size(_pages(), n) == L.CA_OK and n.value >= 16
    assert lib.ca_cache_release(None, *[FAKE] * 5, n.value, None) == L.CA_E_INVALID
    for i in range(5):
        a = [FAKE] * 5
        a[i] = None
        assert lib.ca_cache_release(_pages(), *a, n.value, None) == L.CA_E_INVALID
    assert lib.ca_cache_release(_pages(), *[FAKE] * 5, n.value - 1, None) == L.CA_E_WORKSPACE
    assert lib.ca_cache_release(_pages(), *[FAKE] * 4, FAKE + 16, n.value, None) == L.CA_E_INVALID


def _chunk(**kw):
    from paper_2608_26965_amd import _lib as L
    st = I3(16 * 2 * 64, 2 * 64, 64)
    c = L.CaChunk(batch=3, heads=8, heads_k=2, d=64, dtype=L.CA_BF16, page=16, pages=20, max_pages=5, tokens=9, left=-1,
                  right=-1, sinks=0, causal=1, scale=0.0, table_stride=5, k_stride=st, v_stride=st, q_stride=I2(512, 64),
                  out_stride=I2(512, 64), k_new_stride=I2(128, 64), v_new_stride=I2(128, 64))
    for k, v in kw.items():
        setattr(c, k, v)
    return c


_BAD_CHUNK = [
    (dict(dtype=5), 1, "dtype"), (dict(heads_k=0), 1, "heads_k"), (dict(d=80), 2, "64, 128"), (dict(d=0), 1, "d must"),
    (dict(dtype=0, d=62), 2, "fp32"), (dict(page=0), 1, "page"), (dict(pages=0), 1, "pages"), (dict(tokens=0), 1, "tokens"),
    (dict(tokens=(1 << 24) + 1), 1, "2^24"), (dict(k_stride=I3(2048, 128, 4)), 1, "k_stride[2]"),
    (dict(v_stride=I3(2044, 128, 64)), 1, "v_stride[0]"), (dict(v_stride=I3(-2048, 128, 64)), 1, "v_stride[0]"),
]


@pytest.mark.parametrize("kw,status,word", _BAD_CHUNK + [
    (dict(heads_k=3), 1, "multiple of heads_k"), (dict(batch=0), 1, "batch"), (dict(batch=65536), 2, "65535"),
    (dict(heads=65536, heads_k=1), 2, "65535"), (dict(heads=65535, heads_k=65535, tokens=1 << 24), 2, "too large"),
    (dict(heads=64, heads_k=1, tokens=1 << 24), 2, "too large"), (dict(max_pages=0), 1, "max_pages"),
    (dict(page=1 << 20, max_pages=1 << 10), 2, "2^30"), (dict(sinks=-2), 1, "sinks"), (dict(table_stride=-1), 1, "table_stride"),
    (dict(q_stride=I2(512, 4)), 1, "q_stride[1]"), (dict(out_stride=I2(0, 64)), 1, "out_stride[0]"),
    (dict(out_stride=I2(512, 0)), 1, "out_stride[1]"), (dict(out_stride=I2(512, -64)), 1, "out_stride[1]"),
])
def test_chunk_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_paged_chunk_attn(_chunk(**kw), *[FAKE] * 7, None, FAKE, 1 << 40, None) == status
    assert word in L.last_error()


@pytest.mark.parametrize("kw,status,word", _BAD_CHUNK + [
    (dict(heads_k=65536), 1, "heads_k"), (dict(k_new_stride=I2(128, 4)), 1, "k_new_stride[1]"),
    (dict(v_new_stride=I2(-128, 64)), 1, "v_new_stride[0]"), (dict(k_stride=I3(0, 128, 64)), 1, "k_stride[0]"),
    (dict(v_stride=I3(2048, 0, 64)), 1, "v_stride[1]"), (dict(v_stride=I3(2048, 128, 0)), 1, "v_stride[2]"),
    (dict(tokens=1 << 24, heads_k=64), 2, "too large"),
])
def test_write_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_cache_write(_chunk(**kw), *[FAKE] * 5, None) == status
    assert word in L.last_error()


def test_chunk_pointers_and_workspace():
    L, lib = _lib()
    n = ctypes.c_size_t(0)
    assert lib.ca_paged_chunk_workspace_size(None, n) == L.CA_E_INVALID
    assert lib.ca_paged_chunk_workspace_size(_chunk(), None) == L.CA_E_INVALID
    wide = _chunk(max_pages=1 << 20)
    assert lib.ca_paged_chunk_workspace_size(wide, n) == L.CA_OK
    assert lib.ca_paged_chunk_attn(None, *[FAKE] * 7, None, FAKE, n.value, None) == L.CA_E_INVALID
    for i in range(7):
        a = [FAKE] * 7
        a[i] = None
        assert lib.ca_paged_chunk_attn(wide, *a, None, FAKE, n.value, None) == L.CA_E_INVALID
    if n.value:
        assert lib.ca_paged_chunk_attn(wide, *[FAKE] * 7, None, FAKE, n.value - 1, None) == L.CA_E_WORKSPACE
        assert lib.ca_paged_chunk_attn(wide, *[FAKE] * 7, None, FAKE + 16, n.value, None) == L.CA_E_INVALID
        assert lib.ca_paged_chunk_attn(wide, *[FAKE] * 7, None, None, n.value, None) == L.CA_E_INVALID
    for i in range(5):
        for bad in (None, FAKE + 8):
            a = [FAKE] * 5
            a[i] = bad
            if i < 4 or bad is None:
                assert lib.ca_cache_write(_chunk(), *a, None) == L.CA_E_INVALID


@pytest.mark.parametrize("kw", [dict(), dict(batch=1000, tokens=1 << 20), dict(heads=64, heads_k=1, tokens=1 << 23),
                                dict(dtype=0, d=100), dict(batch=65535, tokens=1 << 23, heads=64)])
def test_chunk_workspace_does_not_grow_with_the_table(kw):
    """At most what the launch's workgroups hold at once: some hundred MB, for tables of any width."""
    L, lib = _lib()
    got = []
    for width in (1 << 10, 1 << 25):
        n = ctypes.c_size_t(0)
        assert lib.ca_paged_chunk_workspace_size(_chunk(page=16, max_pages=width, **kw), n) == L.CA_OK
        got.append(n.value)
    assert got[1] <= 2 * got[0] + (1 << 20) or got[1] < (1 << 29)


def test_chunk_sinks_of_any_number_bound_the_tiles():
    """A window of few keys beside sinks without end is as long as the table."""
    L, lib = _lib()
    got = []
    for kw in (dict(), dict(left=100, sinks=2 ** 31 - 1), dict(left=100, sinks=2 ** 31 - 64), dict(left=100, sinks=1 << 24)):
        n = ctypes.c_size_t(0)
        assert lib.ca_paged_chunk_workspace_size(_chunk(max_pages=1 << 20, **kw), n) == L.CA_OK
        got.append(n.value)
    assert got[0] > 0 and got == got[:1] * 4


def _args(requires_grad=False):
    import torch
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, requires_grad=requires_grad)
    pool = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    return x, pool, torch.zeros(2, 2, dtype=torch.int32), i, torch.zeros(3, dtype=torch.int32)


def test_binding_refuses_cpu_tensors():
    import torch
    import paper_2608_26965_amd as ca
    x, pool, table, lens, starts = _args()
    p = ca.page_pool(3, 16, device="cpu")
    assert p.pages == 3 and p.free.tolist() == [2, 1, 0] and p.state.tolist() == [3, 0, 0]
    for call in (lambda: ca.cache_grow(p, table, lens, lens, 4), lambda: ca.cache_release(p, table, lens),
                 lambda: ca.cache_write(x, x, pool, pool, torch.zeros(4, dtype=torch.int64)),
                 lambda: ca.paged_chunk_attn(ca.Window(), x, pool, pool, table, lens, starts)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        ca.paged_chunk_attn(ca.Window(), x.half(), pool, pool, table, lens, starts)
    for bad in (lambda: ca.page_pool(0, 16, device="cpu"), lambda: ca.page_pool(4, 0, device="cpu"),
                lambda: ca.cache_grow(p, table, lens, lens, 0)):
        with pytest.raises(ValueError, match="out of range"):
            bad()


def test_what_autograd_records():
    import torch
    import paper_2608_26965_amd as ca
    x, pool, table, lens, starts = _args(True)
    slots = torch.zeros(4, dtype=torch.int64)
    write = lambda k, p: ca.cache_write(k, k, p, p, slots)  # noqa: E731
    attend = lambda q, **kw: ca.paged_chunk_attn(ca.Window(), q, pool, pool, table, lens, starts, **kw)  # noqa: E731
    for call in (lambda: write(x, pool), lambda: attend(x)):
        with pytest.warns(UserWarning, match="not recorded by autograd"), pytest.raises(ValueError, match="GPU"):
            call()
    p = pool.clone().requires_grad_()
    for call in (lambda: write(x.detach(), p), lambda: attend(x.detach(), out=x),
                 lambda: attend(x.detach(), lse=torch.zeros(4, 2, requires_grad=True))):
        with pytest.raises(ValueError, match="requires gradients"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call()
