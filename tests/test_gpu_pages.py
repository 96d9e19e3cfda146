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


def test_many_shared_pages(ap):
    """Lists of more pages than one CTA takes, with shared pages in them, given up in parts."""
    rng = np.random.default_rng(8)
    p = Pair(ap, 60, 400, 6000, 16)
    p.extend([0, 1, 2], [5000, 6399, 4100])
    p.same()
    kids = list(range(3, 60))
    parents = [int(x) for x in rng.integers(0, 3, len(kids))]
    p.fork(parents, kids)
    p.same()
    p.extend(kids, [int(x) for x in rng.integers(0, 1, len(kids))])               # no rows: nothing is copied
    p.same()
    p.release(kids[::2], [int(rng.integers(0, p.ref.lengths[b] + 1)) for b in kids[::2]])
    p.same()
    p.extend(kids, [1 if p.ref.lengths[b] < 6400 else 0 for b in kids])
    p.same()
    p.release([0, 1, 2] + kids[1::2], [0, 17, 0] + [0] * len(kids[1::2]))           # the last holders of most pages
    p.same()
    p.release(list(range(60)), [0] * 60)
    p.same()
    assert int(p.t.free_count) == 6000


def state(t):
    return [x.clone() for x in (t.page_table, t.lengths, t.refs, t.free_list, t.free_count)]


@pytest.mark.parametrize("seqs,width", [(6, 4), (60, 400)])                         # one CTA, a cluster
def test_what_cannot_be_carried_out_changes_nothing(ap, seqs, width):
    pages = 24
    t = ap.PageTables.new(seqs, width, pages, 16)
    w = ws()
    cu, rows = i32([9] * 4), i32([9] * 200)
    ap.apack_pages_extend(t, i32([40, 16, 1]), cu, rows, seqs=i32([0, 1, 2]), ws=w)
    assert cu.tolist() == [0, 40, 56, 57] and ap.apack_device_error(w) == 0
    before = state(t)

    def unchanged(n=None):
        assert ap.apack_device_error(w) == ap.APACK_EDEVICE
        assert all(torch.equal(a, b) for a, b in zip(before, state(t)))
        if n is not None:
            assert cu.tolist() == [0] * (n + 1) and (rows == -1).all() and (pairs == 0).all()

    for seq, grow in (([0, 1, 0], [1, 1, 1]),                    # named twice
                      ([0, 1, seqs], [1, 1, 1]), ([0, -1, 2], [1, 1, 1]),
                      ([0, 1, 2], [1, -1, 1]),
                      ([0, 1, 2], [1, width * 16, 1]),            # more rows than its part of the table
                      ([3, 4, 5], [60, 60, 81]),                  # more rows than the map takes
                      ([3, 4, 5], [1, 1, 2 ** 31 - 1])):
        pairs = i32([[9, 9]] * 3)
        rows.fill_(9)
        ap.apack_pages_extend(t, i32(grow), cu, rows, seqs=i32(seq), pairs=pairs, ws=w)
        unchanged(3)
    if width > pages:
        big, c4 = torch.empty(9000, dtype=torch.int32, device="cuda"), i32([9, 9])
        ap.apack_pages_extend(t, i32([16 * 21]), c4, big, seqs=i32([3]), ws=w)       # more pages than are free (19)
        assert ap.apack_device_error(w) == ap.APACK_EDEVICE and (big == -1).all() and c4.tolist() == [0, 0]
        assert all(torch.equal(a, b) for a, b in zip(before, state(t)))
    for seq, keep in (([0, 0], [1, 1]), ([0, seqs], [1, 0]), ([0, 1], [41, 1]), ([0, 1], [1, -1]), ([0, 3], [1, 1])):
        ap.apack_pages_release(t, i32(keep), seqs=i32(seq), ws=w)
        unchanged()
    for parent, seq in (([0, 1], [3, 3]), ([0, seqs], [3, 4]), ([0, -1], [3, 4]), ([0, 0], [3, 1]), ([3, 0], [3, 4])):
        ap.apack_pages_fork(t, i32(parent), i32(seq), ws=w)
        unchanged()
    # tables that disagree with the counts: a page that nobody holds, one outside the pool
    t.refs[int(t.page_table[0, 0])] = 0
    before = state(t)
    ap.apack_pages_release(t, i32([0]), seqs=i32([0]), ws=w)
    unchanged()
    ap.apack_pages_fork(t, i32([0]), i32([3]), ws=w)
    unchanged()
    t.refs[int(t.page_table[0, 0])] = 1
    t.page_table[1, 0] = pages
    before = state(t)
    ap.apack_pages_release(t, i32([0]), seqs=i32([1]), ws=w)
    unchanged()
    t.free_list[int(t.free_count) - 1] = -4
    before = state(t)
    pairs = i32([[9, 9]])
    c2 = i32([9, 9])
    ap.apack_pages_extend(t, i32([20]), c2, rows, seqs=i32([3]), pairs=pairs, ws=w)
    assert ap.apack_device_error(w) == ap.APACK_EDEVICE and c2.tolist() == [0, 0] and (rows == -1).all()
    assert all(torch.equal(a, b) for a, b in zip(before, state(t)))
    # without a workspace the same, unrecorded
    ap.apack_pages_release(t, i32([99]), seqs=i32([2]))
    assert all(torch.equal(a, b) for a, b in zip(before, state(t))) and ap.apack_device_error(w) == 0


def test_no_entries_and_no_rows(ap):
    t = ap.PageTables.new(3, 4, 9, 16)
    cu, rows = i32([9]), i32([9] * 5)
    none = i32([])
    ap.apack_pages_extend(t, none, cu, rows, seqs=none)
    assert cu.tolist() == [0] and rows.tolist() == [-1] * 5
    ap.apack_pages_extend(t, i32([0, 0, 0]), i32([9] * 4), i32([]))
    assert t.lengths.tolist() == [0, 0, 0] and int(t.free_count) == 9
    ap.apack_pages_extend(t, i32([16, 1, 0]), i32([9] * 4), i32([9] * 17))              # seqs None: entry i is sequence i
    assert t.lengths.tolist() == [16, 1, 0] and t.page_table[:, 0].tolist() == [0, 1, -1]
    ap.apack_pages_release(t, i32([16, 0, 0]))
    assert t.lengths.tolist() == [16, 0, 0] and int(t.free_count) == 8


def test_padding_copies_nothing_beside_a_page_that_is_written(ap):
    """Pairs of page 0 with itself, as apack_pages_extend leaves them, beside a pair that writes page 0."""
    k = torch.randn(3, 6, 16, 2, 64, device="cuda").half()
    v = torch.randn_like(k)
    cache = ap.PagedCache(k, v, i32([[0]]))
    want = k.clone(), v.clone()
    for x in want:
        x[:, 0] = x[:, 4]
    ap.apack_copy_pages(cache, i32([[0, 0]] * 40 + [[4, 0]] + [[0, 0]] * 40))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_rows_of_a_wider_table(ap):
    """Tables whose rows lie apart: what lies between them stays."""
    p = Pair(ap, 40, 500, 20000, 16)                         # (40 x 500 entries: a cluster)
    wide = torch.full((40, 517), 77, dtype=torch.int32, device="cuda")
    wide[:, 9:509] = -1
    t = p.t
    p.t = ap.PageTables(wide[:, 9:509], t.lengths, t.refs, t.free_list, t.free_count, 16)
    seqs = np.random.default_rng(2).permutation(40).tolist()
    p.extend(seqs[:30], [1 + (997 * b) % 8000 for b in seqs[:30]])
    p.same()
    p.fork(seqs[:5], seqs[30:35])
    p.same()
    p.release(seqs[3:33], [p.ref.lengths[b] // 2 for b in seqs[3:33]])
    p.same()
    p.extend(seqs[:33], [3] * 33)
    p.same()
    assert (wide[:, :9] == 77).all() and (wide[:, 509:] == 77).all()


def test_lists_that_are_the_lengths(ap):
    """The pool's own lengths as the rows to keep, and as the rows to add."""
    t, ref = ap.PageTables.new(300, 90, 27000, 16), PageLists(300, 90, 27000, 16)
    w, grow = ws(), [(37 * b) % 700 for b in range(300)]
    cu = i32([0] * 301)
    ap.apack_pages_extend(t, i32(grow), cu, i32([0] * sum(grow)), ws=w)
    ref.extend(list(range(300)), grow)
    ap.apack_pages_release(t, t.lengths, ws=w)
    assert t.lengths.tolist() == grow
    rows = i32([0] * sum(grow))
    ap.apack_pages_extend(t, t.lengths, cu, rows, ws=w)
    want = ref.extend(list(range(300)), grow)
    assert cu.tolist() == want[0] and rows.tolist() == want[1]
    assert t.page_table.tolist() == ref.table and t.lengths.tolist() == ref.lengths and ap.apack_device_error(w) == 0


@pytest.mark.parametrize("most", [90, 9000])
def test_a_captured_step_follows_its_inputs(ap, most):
    """Release, fork and extension in one graph; a map by the first kernel, and one by the second."""
    n, width, page = 12, 64, 16
    t, ref, w = ap.PageTables.new(2 * n, width, 2 * n * width, page), PageLists(2 * n, width, 2 * n * width, page), ws()
    seqs, parents, keep, grow = (i32([0] * n) for _ in range(4))
    seqs.copy_(i32(range(n)))
    kids, none = i32(range(n, n + 4)), i32([0] * 4)
    cu, rows, owners = i32([0] * (n + 1)), i32([0] * most), i32([0] * most)
    slots, pairs = torch.zeros(most, dtype=torch.int64, device="cuda"), i32([0] * (2 * n)).view(n, 2)

    def step():
        ap.apack_pages_release(t, keep, seqs=seqs, ws=w)
        ap.apack_pages_release(t, none, seqs=kids, ws=w)
        ap.apack_pages_fork(t, parents[:4], kids, ws=w)
        ap.apack_pages_extend(t, grow, cu, rows, seqs=seqs, row_seqs=owners, slots=slots, pairs=pairs, ws=w)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()                                                # (all empty)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
    torch.cuda.current_stream().wait_stream(s)
    rng = np.random.default_rng(most)
    for _ in range(12):
        order = rng.permutation(n).tolist()
        from_ = rng.permutation(n)[:4].tolist()
        kept = [int(rng.integers(0, ref.lengths[b] + 1)) if rng.random() < 0.5 else ref.lengths[b] for b in order]
        after = dict(zip(order, kept))
        more = [min(int(rng.integers(0, most // n)), width * page - after[b]) for b in order]
        seqs.copy_(i32(order)), keep.copy_(i32(kept)), grow.copy_(i32(more)), parents[:4].copy_(i32(from_))
        g.replay()
        ref.release(order, kept)
        ref.release(list(range(n, n + 4)), [0] * 4)
        ref.fork(from_, list(range(n, n + 4)))
        want = ref.extend(order, more)
        pad = [-1] * (most - sum(more))
        assert ap.apack_device_error(w) == 0
        assert t.page_table.tolist() == ref.table and t.lengths.tolist() == ref.lengths and t.refs.tolist() == ref.refs
        assert t.free_list[:int(t.free_count)].tolist() == ref.free
        assert cu.tolist() == want[0] and rows.tolist() == want[1] + pad and owners.tolist() == want[2] + pad
        assert slots.tolist() == want[3] + pad and [tuple(x) for x in pairs.tolist()] == want[4]
