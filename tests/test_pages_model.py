"""The plain model of the pages by hand-worked cases (CPU)."""
import random

import pytest

from tests.pages_model import FULL, LENGTH, OK, RANGE, UNIT, PagesModel


def _rows(n, tag=0):
    return [(tag + i, -(tag + i)) for i in range(n)]


def test_append_takes_the_lowest_pages_in_entry_order():
    m = PagesModel(3, 4, 8, 16)
    assert m.append([2, 0], [_rows(17), _rows(16)]) == [OK, OK]
    assert m.table == [[2], [], [0, 1]] and m.lens == [16, 0, 17]
    assert m.append([0, 2], [_rows(1), _rows(15)]) == [OK, OK]
    assert m.table == [[2, 3], [], [0, 1]]
    assert m.slot(2, 16) == (16, -16)


def test_entries_past_the_free_pages_are_refused_and_those_that_need_none_go_ahead():
    m = PagesModel(4, 4, 2, 16)
    assert m.append([0, 1, 2], [_rows(16), _rows(17), _rows(1)]) == [OK, FULL, FULL]
    assert m.append([0, 1], [_rows(0), _rows(0)]) == [OK, OK]
    assert m.lens == [16, 0, 0, 0]


def test_fork_shares_full_pages_and_copies_the_last():
    m = PagesModel(3, 4, 8, 16)
    m.append([0], [_rows(20)])
    assert m.fork([0, 0], [1, 2]) == [OK, OK]
    assert m.table == [[0, 1], [0, 2], [0, 3]] and m.refs[:4] == [3, 1, 1, 1]
    assert m.slot(2, 19) == (19, -19)
    assert m.fork([0], [1]) == [UNIT]     # not empty
    m.free([0])
    assert m.refs[:4] == [2, 0, 1, 1]


def test_compact_keeps_the_prefix_and_the_picked():
    m = PagesModel(2, 4, 8, 16)
    m.append([0], [_rows(50)])
    assert m.compact([0], [0], [17], [[40, 20, 20]]) == [OK]
    assert m.lens[0] == 20 and [m.slot(0, s)[0] for s in (0, 16, 17, 18, 19)] == [0, 16, 40, 20, 20]
    assert m.table[0] == [0, 4]
    assert m.compact([0], [0], [18], [[]]) == [OK] and m.table[0] == [0, 4]
    assert m.compact([0], [0], [19], [[]]) == [RANGE]
    assert m.compact([0], [0], [0], [[0] * 80]) == [LENGTH]


@pytest.mark.parametrize("seed", range(5))
def test_every_page_is_counted(seed):
    rng = random.Random(seed)
    m = PagesModel(8, 6, 24, 16)
    for _ in range(200):
        us = [rng.randrange(8) for _ in range(3)]
        op = rng.randrange(4)
        if op == 0:
            m.append(us, [_rows(rng.randrange(40)) for _ in us])
        elif op == 1:
            m.fork(us, [rng.randrange(8) for _ in us])
        elif op == 2:
            keep = [rng.randint(0, m.lens[u]) for u in us]
            m.compact(us, us, keep, [[rng.randrange(max(1, m.lens[u])) for _ in range(rng.randrange(20))
                                      if m.lens[u]] for u in us])
        else:
            m.free(us[:1])
        held = [p for t in m.table for p in t]
        assert m.refs == [held.count(p) for p in range(24)]
        for u in range(8):
            assert len(m.table[u]) == -(-m.lens[u] // 16)
            if m.lens[u] % 16:
                assert m.refs[m.table[u][-1]] == 1   # a page that is not full is one unit's own


def test_a_unit_forked_to_itself_stays():
    m = PagesModel(3, 4, 8, 16)
    m.append([0, 1], [_rows(20), _rows(16)])
    before = [list(t) for t in m.table], list(m.refs)
    assert m.fork([0, 1, 2], [0, 1, 2]) == [OK, OK, OK]
    assert ([list(t) for t in m.table], m.refs) == before and m.lens == [20, 16, 0]
    assert m.fork([0, 0], [0, 2]) == [OK, UNIT]
