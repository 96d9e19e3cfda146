"""Page tables kept on the device: calls without a list of pages to copy, and lists that are other sequences' lengths."""

import pytest
import torch

from oracle.paged_oracle import PageLists
from test_gpu_pages import i32, state, ws

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


@pytest.mark.parametrize("page,pages,room", [(16, 40, 60), (16, 40, 9000), (2, 20000, 40000)])    # one kernel, two, a cluster
def test_extension_without_pairs(ap, page, pages, room):
    """A call that would have a page to copy and has nowhere to say so changes nothing; others need no pairs."""
    t, ref, w = ap.PageTables.new(6, 9, pages, page), PageLists(6, 9, pages, page), ws()
    n = 2 * page + 1                                                           # a last page of one row

    def extend(seqs, grow, fails, pairs=None):
        cu, rows, before = i32([9] * (len(seqs) + 1)), torch.full((room,), 9, dtype=torch.int32, device="cuda"), state(t)
        ap.apack_pages_extend(t, i32(grow), cu, rows, seqs=i32(seqs), pairs=pairs, ws=w)
        if fails:
            assert ap.apack_device_error(w) == ap.APACK_EDEVICE
            assert all(torch.equal(a, b) for a, b in zip(before, state(t)))
            assert cu.tolist() == [0] * (len(seqs) + 1) and (rows == -1).all()
            return
        want = ref.extend(seqs, grow)
        assert ap.apack_device_error(w) == 0 and cu.tolist() == want[0]
        assert rows[:len(want[1])].tolist() == want[1] and (rows[len(want[1]):] == -1).all()
        assert pairs is not None or all(p == (0, 0) for p in want[4])
        assert t.page_table.tolist() == ref.table and t.lengths.tolist() == ref.lengths and t.refs.tolist() == ref.refs

    extend([0, 5], [n, 3], False)
    ap.apack_pages_fork(t, i32([0, 0, 0]), i32([1, 2, 3]), ws=w)
    ref.fork([0, 0, 0], [1, 2, 3])
    extend([1], [1], True)
    extend([5, 2], [1, 1], True)
    extend([0, 1, 2, 3], [1, 1, 1, 1], True)                                   # all holders: all but the last would copy
    extend([0, 1, 2, 3, 5], [0, 0, 0, 0, 2], False)                            # no rows, no copy
    extend([1, 2], [1, 1], False, pairs=i32([[9, 9]] * 2))
    extend([0], [1], True)
    ap.apack_pages_release(t, i32([0]), seqs=i32([0]), ws=w)
    ref.release([0], [0])
    extend([3, 1], [1, page], False)                                           # the last holder writes where it is
    ap.apack_pages_release(t, i32([2 * page]), seqs=i32([2]), ws=w)
    ref.release([2], [2 * page])
    ap.apack_pages_fork(t, i32([2]), i32([4]), ws=w)
    ref.fork([2], [4])
    extend([2, 4], [1, 1], False)                                              # whole pages are shared and not written to


@pytest.mark.parametrize("seqs,width", [(150, 90), (300, 90), (1500, 40)])                       # one CTA, a cluster
@pytest.mark.parametrize("shared", [False, True])
def test_lists_that_are_other_lengths(ap, seqs, width, shared):
    """Every sequence is cut to, or grows by, the length that the one before it has before the call."""
    pages = seqs * width
    t, ref, w = ap.PageTables.new(seqs + 1, width, pages, 16), PageLists(seqs + 1, width, pages, 16), ws()
    order = list(range(seqs))
    grow = [1 + 300 * b // seqs + b % 2 * 20 for b in order]
    grow = sorted(grow)
    cu, pairs = i32([0] * (seqs + 1)), i32([[0, 0]] * seqs)
    rows = i32([0] * (sum(grow) + 3))
    ap.apack_pages_extend(t, i32(grow), cu, rows, seqs=i32(order), ws=w)
    ref.extend(order, grow)
    if shared:
        ap.apack_pages_fork(t, i32([seqs - 1]), i32([seqs]), ws=w)
        ref.fork([seqs - 1], [seqs])
    behind = order[1:]
    ap.apack_pages_release(t, t.lengths[:seqs - 1], seqs=i32(behind), ws=w)
    ref.release(behind, grow[:-1])
    assert ap.apack_device_error(w) == 0
    assert t.lengths.tolist() == ref.lengths and t.page_table.tolist() == ref.table and t.refs.tolist() == ref.refs
    assert t.free_list[:int(t.free_count)].tolist() == ref.free
    now = t.lengths[:seqs - 1].tolist()
    ap.apack_pages_extend(t, t.lengths[:seqs - 1], cu[:seqs], rows, seqs=i32(behind), pairs=pairs[:seqs - 1], ws=w)
    want = ref.extend(behind, now)
    assert ap.apack_device_error(w) == 0 and cu[:seqs].tolist() == want[0] and rows[:len(want[1])].tolist() == want[1]
    assert t.lengths.tolist() == ref.lengths and t.page_table.tolist() == ref.table and t.refs.tolist() == ref.refs
