"""Steps with fewer rows than new tokens: what the oracle says of them, and the refusals of the call
that reports how far the rows go. No GPU needed."""
import random

import pytest

from oracle import seq
from tests.test_abi_chunk import FAKE, _BAD_PAGES, _args, _lib, _pages


def test_rows_sit_where_the_attention_takes_them_for():
    """Row i of the lq of sequence b sits at place i + lens - lq for the attention, with the lengths that
    cache_grow reports for lens; rope and the slots go by the positions. Every token below that length is
    an older one or has a row."""
    r = random.Random(1)
    for _ in range(200):
        B, page, width = r.randrange(1, 6), r.choice((1, 4, 16)), 5
        lens = [r.randrange(-2, page * width + 9) for _ in range(B)]
        new = [r.randrange(-1, 30) for _ in range(B)]
        total = sum(min(max(m, 0), min(max(n, 0), page * width)) for n, m in zip(lens, new))
        tokens = max(1, r.choice((total, total + 3, total // 2, r.randrange(1, total + 2))))
        table, free = [[-1] * width for _ in range(B)], list(range(100))
        state, starts, slots, positions = seq.cache_grow(table, free, lens, new, page, 100, tokens)
        seen = seq.lens_with_rows(lens, new, page * width, tokens)
        assert sum(min(max(n, 0), page * width) for n in lens) - sum(seen) == state[2]
        for b in range(B):
            lq, n = starts[b + 1] - starts[b], min(max(lens[b], 0), page * width)
            assert positions[starts[b]:starts[b + 1]] == [i + seen[b] - lq for i in range(lq)]
            assert seen[b] - lq == n - min(max(new[b], 0), n)


@pytest.mark.parametrize("kw,status,word", _BAD_PAGES + [(dict(tokens=0), 1, "tokens"), (dict(tokens=1 << 25), 1, "2^24")])
def test_grow_seen_refusals(kw, status, word):
    L, lib = _lib()
    assert lib.ca_cache_grow_seen(_pages(**kw), *[FAKE] * 9, None) == status
    assert word in L.last_error()


def test_grow_seen_pointers():
    L, lib = _lib()
    assert lib.ca_cache_grow_seen(None, *[FAKE] * 9, None) == L.CA_E_INVALID
    for i in range(9):
        a = [FAKE] * 9
        a[i] = None
        assert lib.ca_cache_grow_seen(_pages(), *a, None) == L.CA_E_INVALID


def test_binding_refuses_lengths_in_place():
    import paper_2608_26965_amd as ca
    _, _, table, lens, _ = _args()
    p, new = ca.page_pool(3, 16, device="cpu"), lens.clone()
    for seen in (lens, new):
        with pytest.raises(ValueError, match="seen"):
            ca.cache_grow(p, table, lens, new, 4, seen=seen)
    with pytest.raises(ValueError, match="GPU"):
        ca.cache_grow(p, table, lens, new, 4, seen=lens.clone())
