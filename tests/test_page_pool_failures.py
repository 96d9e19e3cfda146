"""PagePool when a device call or an allocation fails midway (on the CPU): the pool is as it was, and a second try works."""

import numpy as np
import pytest
import torch

from test_page_pool import make, pools, rows, write          # noqa: F401 (a fixture)


class Failure(RuntimeError):
    pass


def state(pool):
    return (list(pool._free), [None if p is None else list(p) for p in pool._pages], pool._refs.tolist(), pool._len.tolist(),
            pool._shared, pool.page_table.tolist(), pool.lengths.tolist(), pool.free_pages)


def failing(monkeypatch, owner, name, at):
    """The at-th call of owner.name raises (counted from 0)."""
    real, calls = getattr(owner, name), []

    def call(*a, **kw):
        calls.append(1)
        if len(calls) == at + 1:
            raise Failure(name)
        return real(*a, **kw)
    monkeypatch.setattr(owner, name, call)


def keep(*at):
    return torch.tensor(at, dtype=torch.int32)


def filled(pools):
    pool = make(pools)
    a, b = pool.add(6), pool.add(9)
    write(pool, a, 0, range(10, 16))
    write(pool, b, 0, range(20, 29))
    return pool, a, b, pool.fork(a)


OPERATIONS = {
    "add": lambda pool, a, b, c: pool.add(7),
    "extend": lambda pool, a, b, c: pool.extend([a, c, b], 5),       # a copy of a shared page, and new pages
    "prune": lambda pool, a, b, c: pool.prune([a, b], keep(1, 2, 6, 9, 14), [2, 3]),
    "prune in place": lambda pool, a, b, c: pool.prune([b], keep(2, 3, 8), [3], in_place=True),
    "take": lambda pool, a, b, c: pool.take(pool._cache_of([pool.pages(b)]), [3], keep_idx=keep(0, 4, 5)),
}


def contents(pool):
    """Every sequence's keys (-1 where no one has written yet)."""
    return [[float(pool.k[0, p[r // pool.page_tokens], r % pool.page_tokens, 0, 0]) for r in range(pool.length(s))]
            for s, p in enumerate(pool._pages) if p is not None]


def expected(pools, op):
    pool, *seqs = filled(pools)
    OPERATIONS[op](pool, *seqs)
    return state(pool), contents(pool)


@pytest.mark.parametrize("op", OPERATIONS)
@pytest.mark.parametrize("where", ["copy", "move", "array", "table"])
def test_a_failure_changes_nothing(pools, monkeypatch, op, where):      # noqa: F811
    want = expected(pools, op)
    reached = 0
    for at in range(12):
        pool, *seqs = filled(pools)
        before = state(pool)
        with monkeypatch.context() as m:
            if where == "copy":
                failing(m, pools, "apack_copy_pages", at)
            elif where == "move":
                failing(m, pools, "apack_paged_compact", at)
            elif where == "array":
                failing(m, pool, "_device", at)
            else:
                failing(m, pools, "PagedCache", at)
            try:
                OPERATIONS[op](pool, *seqs)
                break
            except Failure:
                reached += 1
        assert state(pool) == before
        assert rows(pool, seqs[0]) == list(range(10, 16)) and rows(pool, seqs[1]) == list(range(20, 29))
        OPERATIONS[op](pool, *seqs)                                    # the second try
        assert (state(pool), contents(pool)) == want
    else:
        pytest.fail("the operation never succeeds")
    assert reached or (op, where) not in {("extend", "copy"), ("prune", "move"), ("prune in place", "move"), ("take", "move"),
                                         ("add", "array"), ("extend", "array"), ("prune", "array"), ("take", "array")}


@pytest.mark.parametrize("op", ["fork", "free"])
@pytest.mark.parametrize("where", ["page_table", "lengths"])
def test_a_failing_table_changes_nothing(pools, op, where):            # noqa: F811
    class Broken:
        def __getitem__(self, at):
            raise Failure(where)

    pool, a, b, c = filled(pools)
    before, real = state(pool), getattr(pool, where)
    setattr(pool, where, Broken())
    with pytest.raises(Failure):
        getattr(pool, op)(b)
    setattr(pool, where, real)
    assert state(pool)[:5] == before[:5]
    if op == "fork":
        new = pool.fork(b)
        assert rows(pool, new) == rows(pool, b)
    else:
        pool.free(b)
        assert pool.free_pages == len(before[0]) + 3


def test_a_failed_copy_does_not_hand_a_shared_page_to_two_writers(pools, monkeypatch):   # noqa: F811
    pool, a, b, c = filled(pools)
    with monkeypatch.context() as m:
        failing(m, pools, "apack_copy_pages", 0)
        with pytest.raises(Failure):
            pool.extend([a])
    first = pool.extend([a]).tolist()
    assert first == [6] and pool.pages(a)[-1] != pool.pages(c)[-1]
    write(pool, a, 6, [99])
    pool.extend([c])
    write(pool, c, 6, [77])
    assert rows(pool, a) == [10, 11, 12, 13, 14, 15, 99] and rows(pool, c) == [10, 11, 12, 13, 14, 15, 77]
    assert np.all(pool._refs >= 0)
