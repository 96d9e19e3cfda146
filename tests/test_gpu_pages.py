"""Page tables kept on the device against lists on the host: whole numbers, equal."""

import numpy as np
import pytest
import torch

from oracle.paged_oracle import PageLists

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def ws():
    return torch.zeros(1024, dtype=torch.uint8, device="cuda")


class Pair:
    """The same calls on the device and on lists."""

    def __init__(self, ap, seqs, width, pages, page):
        self.ap, self.ws = ap, ws()
        self.t = ap.PageTables.new(seqs, width, pages, page)
        self.ref = PageLists(seqs, width, pages, page)
        self.pages = pages

    def same(self):
        count = int(self.t.free_count)
        assert self.t.page_table.tolist() == self.ref.table
        assert self.t.lengths.tolist() == self.ref.lengths
        assert self.t.refs.tolist() == self.ref.refs
        assert self.t.free_list[:count].tolist() == self.ref.free
        assert self.ap.apack_device_error(self.ws) == 0

    def release(self, seqs, keep):
        self.ap.apack_pages_release(self.t, i32(keep), seqs=i32(seqs), ws=self.ws)
        self.ref.release(seqs, keep)

    def fork(self, parents, seqs):
        self.ap.apack_pages_fork(self.t, i32(parents), i32(seqs), ws=self.ws)
        self.ref.fork(parents, seqs)

    def extend(self, seqs, grow, spare=5):
        n, cap = len(seqs), sum(grow) + spare
        cu, rows, owners = i32([9] * (n + 1)), i32([9] * cap), i32([9] * cap)
        slots, pairs = torch.full((cap,), 9, dtype=torch.int64, device="cuda"), i32([[9, 9]] * n).view(n, 2)
        self.ap.apack_pages_extend(self.t, i32(grow), cu, rows, seqs=i32(seqs), row_seqs=owners, slots=slots, pairs=pairs,
                                   ws=self.ws)
        want = self.ref.extend(seqs, grow)
        pad = [-1] * spare
        assert cu.tolist() == want[0]
        assert rows.tolist() == want[1] + pad
        assert owners.tolist() == want[2] + pad
        assert slots.tolist() == want[3] + pad
        assert [tuple(p) for p in pairs.tolist()] == want[4]


@pytest.mark.parametrize("page,seqs,most", [(16, 9, 70), (1, 5, 30), (7, 40, 40), (64, 61, 900), (128, 300, 200)])
def test_random_steps(ap, page, seqs, most):
    rng = np.random.default_rng(page)
    width = -(-4 * most // page) + 1
    p = Pair(ap, seqs, width, seqs * width, page)
    for step in range(25):
        order = rng.permutation(seqs).tolist()
        if step % 3 == 0:
            some = order[:rng.integers(1, seqs + 1)]
            p.release(some, [int(rng.integers(0, p.ref.lengths[b] + 1)) if rng.random() < 0.7 else 0 for b in some])
            p.same()
        empty = [b for b in order if p.ref.lengths[b] == 0]
        held = [b for b in order if p.ref.lengths[b] > 0]
        if held and empty and step % 2:
            children = empty[:rng.integers(1, len(empty) + 1)]
            p.fork([held[i] for i in rng.integers(0, min(3, len(held)), len(children))], children)
            p.same()
        some = [b for b in rng.permutation(seqs).tolist() if p.ref.lengths[b] < 3 * most][:rng.integers(1, seqs + 1)]
        grow = [int(rng.integers(0, most)) if rng.random() < 0.8 else 0 for _ in some]
        p.extend(some, grow, spare=int(rng.integers(0, 9)))
        p.same()


def test_many_entries_and_a_long_map(ap):
    """All 4,096 sequences, then a slot map that a second kernel writes."""
    p = Pair(ap, 4096, 12, 4096 * 12, 16)
    seqs = np.random.default_rng(3).permutation(4096).tolist()
    grow = [1 + (7 * b) % 90 for b in seqs]
    p.extend(seqs, grow)
    p.same()
    p.release(seqs, [g // 2 for g in grow])
    p.same()
    p.extend(seqs[::-1], [1] * 4096)
    p.same()
