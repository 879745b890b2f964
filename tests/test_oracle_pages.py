"""Pins of the page oracle (oracle/seq.py): cases by hand and invariants. CPU only."""
import random

from oracle import seq


def test_grow_by_hand():
    # pages of 4: sequence 0 goes on by one token into a new page, 1 has nothing new, 2 is a prompt of 6
    table, free = [[5, -1, -1], [7, 8, -1], [-1, -1, -1]], [0, 1, 2, 3]
    state, starts, slots, positions = seq.cache_grow(table, free, [5, 6, 6], [1, 0, 6], 4, 9, 9)
    assert table == [[5, 3, -1], [7, 8, -1], [2, 1, -1]] and free == [0]
    assert state == [1, 0, 0] and starts == [0, 1, 1, 7]
    assert slots == [12, 8, 9, 10, 11, 4, 5, -1, -1] and positions == [4, 0, 1, 2, 3, 4, 5, 0, 0]


def test_grow_that_lacks_pages_and_rows():
    table, free = [[-1, -1], [-1, -1]], [6]
    state, starts, slots, positions = seq.cache_grow(table, free, [3, 4], [3, 4], 2, 7, 5)
    assert table == [[6, -1], [-1, -1]] and state == [0, 3, 2]
    assert starts == [0, 3, 5] and slots == [12, 13, -1, -1, -1] and positions == [0, 1, 2, 0, 1]


def test_release_by_hand():
    table = [[1, 2, 3, 4], [5, 6, -1, 9], [7, -1, -1, -1]]
    free = [0]
    # window of 3 and one sink: of 10 tokens in pages of 3 the next sees 0 and 7, 8, 9
    seq.cache_release(table, free, [10, 3, 0], 3, 9, left=3, sinks=1)
    assert table == [[1, -1, 3, 4], [5, -1, -1, 9], [-1, -1, -1, -1]]  # 9 is no page
    assert free == [0, 7, 6, 2]


def test_release_undoes_grow_and_no_page_is_lost():
    r = random.Random(0)
    for _ in range(50):
        page, pages, B, width = r.choice((1, 3, 16)), 40, r.randrange(1, 6), 12
        table, free = [[-1] * width for _ in range(B)], list(range(pages))
        lens = [0] * B
        for _ in range(8):
            new = [r.choice((0, 1, r.randrange(2 * page + 1))) for _ in range(B)]
            lens = [min(a + n, width * page) for a, n in zip(lens, new)]
            before, spare = [list(x) for x in table], list(free)
            state, *_ = seq.cache_grow(table, free, lens, new, page, pages, 10 ** 6)
            held = [e for row in table for e in row if e >= 0]
            assert sorted(held + free) == list(range(pages)) and state[0] == len(free)
            if not state[1]:
                again = [list(x) for x in table], list(free)
                seq.cache_grow(table, free, lens, new, page, pages, 10 ** 6)
                assert (table, free) == again
                if r.random() < 0.3:
                    kept = [min(a, n) for a, n in zip(([a - n for a, n in zip(lens, new)]), lens)]
                    seq.cache_release(table, free, kept, page, pages)
                    assert (table, free) == (before, spare)
                    lens = kept
            if r.random() < 0.3:
                lens[r.randrange(B)] = 0
                seq.cache_release(table, free, lens, page, pages)
                assert sorted([e for row in table for e in row if e >= 0] + free) == list(range(pages))
