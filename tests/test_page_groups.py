"""PagePool.groups on the CPU: which sequences share their first pages, and how many rows."""

import pytest
import torch


@pytest.fixture()
def pool(monkeypatch):
    import __graft_entry__
    __graft_entry__.build()
    from paper_2608_08794_gb300 import paged
    monkeypatch.setattr(paged, "apack_copy_pages", lambda *a, **k: None)
    return paged.PagePool(1, 40, 4, 1, 64, 12, dtype=torch.float16, device="cpu")


def test_groups(pool):
    a, b, empty = pool.add(10), pool.add(8), pool.add(0)
    kid = pool.fork(a)
    assert [x if isinstance(x, list) else x.tolist() for x in pool.groups([a, kid])] == [[a, kid], [0, 2], [10]]
    grown, of_b = pool.fork(a), pool.fork(b)
    pool.extend([grown], 3)                                   # its copy of a's last page: 8 rows are still the same
    pool.extend([of_b], 1)                                    # a page of its own behind b's two
    order, bounds, prefix = pool.groups([of_b, grown, empty, a, b, kid])
    assert order == [of_b, b, grown, a, kid, empty] and bounds.tolist() == [0, 2, 5, 6] and prefix.tolist() == [8, 8, 0]
    order, bounds, prefix = pool.groups([empty])
    assert order == [empty] and bounds.tolist() == [0, 1] and prefix.tolist() == [0]
    assert pool.groups([])[0] == [] and pool.groups([])[1].tolist() == [0]
    with pytest.raises(ValueError):
        pool.groups([a, a])
    with pytest.raises(ValueError):
        pool.groups([11])
