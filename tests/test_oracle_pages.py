"""CPU pins of the oracle's shared pages: the rules by hand, and what no run of calls may break: every page is held or on the stack, once, and
its count is that of its holders less one."""
import numpy as np
import pytest

from oracle import paged, pages


def test_fork_by_hand():
    P, free = 16, [7, 6, 5, 0, 0, 0, 0, 0]
    table = [[3, 1, -1], [9, 9, 9], [9, 9, 9], [2, -1, -1]]
    src, dst, n, top, shared, ok, t = pages.fork([0, 0, 3], [1, 2, 0], [20, 0, -4, 16], table, free, [2], [0] * 8, P)
    assert list(ok) == [1, 1, 0]                            # row 0 has tokens
    assert list(src) == [1, 1, -1] and list(dst) == [6, 7, -1] and list(top) == [0] and list(n) == [20, 20, 20, 16]
    assert list(t[1]) == [3, 6, 9] and list(t[2]) == [3, 7, 9] and list(shared) == [0, 0, 0, 2, 0, 0, 0, 0]
    # one page for two forks that need one; a whole page needs none, wherever it stands; the second that names a row is refused
    *_, top, shared, ok, t = pages.fork([0, 0, 3, 3], [1, 2, 2, 2], [20, 0, 0, 16], table, free, [1], [0] * 8, P)
    assert list(ok) == [1, 0, 0, 0] and list(top) == [0] and list(t[2]) == [9, 9, 9]
    *_, n, top, shared, ok, t = pages.fork([3, 0, 0], [2, 1, 5], [20, 0, 0, 16], table, free, [0], [0] * 8, P, n_tokens=[16, 16, 3])
    assert list(ok) == [1, 1, 0] and list(n) == [20, 16, 16, 16] and list(shared) == [0, 0, 1, 1, 0, 0, 0, 0]


def test_release_by_hand():
    table = [[3, 1], [3, 6], [3, 7], [0, 4]]
    n, top, shared, free = pages.release([1, 0, 1, 1], [20, 20, 20, 16], table, [5, 2, -1, -1, -1, -1, -1, -1], [2], [0, 0, 0, 2, 0, 0, 0, 0], 16)
    assert list(n) == [0, 20, 0, 0] and list(top) == [5] and list(free) == [5, 2, 0, 1, 7, -1, -1, -1] and list(shared) == [0] * 8
    n, top, shared, free = pages.release([1, 1, 1, 0], [20, 20, 20, 16], table, [5, 2, -1, -1, -1, -1, -1, -1], [2], [0, 0, 0, 2, 0, 0, 0, 0], 16)
    assert list(free[:6]) == [5, 2, 1, 3, 6, 7] and list(top) == [6]


def test_compact_by_hand():
    src, dst, t, free, shared = pages.compact([20, 16], [[6, 1], [6, 3]], [0, 7, 2, 5, 4, 9, 9, 9], [5], [0, 0, 0, 0, 0, 0, 1, 0], 16)
    assert list(src) == [3, 6, -1, -1] and list(dst) == [0, 2, -1, -1]
    assert t.tolist() == [[2, 1], [2, 3]]                   # (the second row's second entry is not held)
    assert list(free) == [7, 6, 5, 4, 3, -1, -1, -1] and list(shared) == [0, 0, 1, 0, 0, 0, 0, 0]


@pytest.mark.parametrize("seed", range(12))
def test_pages_are_held_or_free_and_contents_follow(seed):
    """A serving loop of all calls over a pool of marks: what every sequence reads through its row stays what it was."""
    rng = np.random.default_rng(seed)
    B, P, width, n_pages = 9, 16, 6, 30
    table, free, n_free, shared, lens = np.full((B, width), -1), np.arange(n_pages), np.array([n_pages]), np.zeros(n_pages, int), np.zeros(B, int)
    pool, marks, mark = np.zeros((n_pages, P), int), {b: [] for b in range(B)}, 0
    for _ in range(60):
        what = rng.integers(4)
        if what == 0:
            new = np.where(rng.random(B) < 0.4, rng.integers(0, 40, B), 0)
            slots, lens, n_free, granted, table, free = paged.page_map(lens, new, table, free, n_free, P, max_new=40)
            for b in range(B):
                for j in range(new[b] if granted[b] else 0):
                    mark += 1
                    pool[slots[b, j] // P, slots[b, j] % P] = mark
                    marks[b].append(mark)
        elif what == 1:
            src, dst = rng.integers(-1, B + 1, 3), rng.integers(-1, B + 1, 3)
            n = np.array([rng.integers(-1, max(1, lens[s]) + 2) if 0 <= s < B else 1 for s in src])
            cs, cd, lens, n_free, shared, ok, table = pages.fork(src, dst, lens, table, free, n_free, shared, P, n_tokens=n)
            pool = pages.copy(pool, cs, cd)
            old = {b: list(m) for b, m in marks.items()}
            for f in range(3):
                if ok[f]:
                    marks[int(dst[f])] = old[int(src[f])][:n[f]]
        elif what == 2:
            ended = rng.random(B) < 0.3
            lens, n_free, shared, free = pages.release(ended, lens, table, free, n_free, shared, P)
            marks = {b: [] if ended[b] else m for b, m in marks.items()}
        else:
            cs, cd, table, free, shared = pages.compact(lens, table, free, n_free, shared, P)
            pool = pages.copy(pool, cs, cd)
        holders = np.zeros(n_pages, int)
        for b in range(B):
            row = table[b, :-(-lens[b] // P)]
            np.add.at(holders, row, 1)
            assert [pool[row[t // P], t % P] for t in range(lens[b])] == marks[b]
        top = int(n_free[0])
        assert sorted(list(free[:top]) + list(np.flatnonzero(holders))) == list(range(n_pages))
        assert np.array_equal(shared, np.maximum(holders - 1, 0))
