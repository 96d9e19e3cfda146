"""Refusals of the calls on shared rows and page tables, before anything is launched (no device work), and pins of their
oracles."""

import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def status(ap, call):
    with pytest.raises(ap.ApackError) as e:
        call()
    return e.value.status


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def cache(ap, heads=4, dim=128, dtype=torch.bfloat16, seqs=3):
    k = torch.zeros(2, 6, 16, heads, dim, dtype=dtype)
    return ap.PagedCache(k, torch.zeros_like(k), i32(seqs, 3))


def workspace(n):
    raw = torch.zeros(n + 256, dtype=torch.uint8)
    return raw[(-raw.data_ptr()) % 256:][:n]


def test_workspace_sizes(ap):
    c = cache(ap)
    small, large = (ap.apack_paged_group_workspace_size(c, 28, 3, n) for n in (3, 300))
    assert 0 < small < large
    assert ap.apack_paged_group_workspace_size(c, 28, 3, 0) > 0
    assert ap.apack_paged_group_workspace_size(cache(ap, heads=1), 1024, 3, 5) > 0
    for heads, seqs, n in ((0, 3, 3), (30, 3, 3), (1028, 3, 3), (28, 0, 3), (28, 4097, 3), (28, 3, -1), (28, 3, 2 ** 24 + 1),
                           (28, 3, 10 ** 7)):
        assert status(ap, lambda: ap.apack_paged_group_workspace_size(c, heads, seqs, n)) == ap.APACK_EINVAL


def test_plan_arguments(ap):
    c = cache(ap)
    ws = workspace(ap.apack_paged_group_workspace_size(c, 28, 3, 7))
    lens = i32(3)

    def plan(cache=c, lens=lens, heads=28, n_q=3, ws=ws, **kw):
        ap.apack_paged_group_plan(cache, lens, heads, n_q, ws, stream=0, **kw)

    assert status(ap, lambda: plan(n_q=4)) == ap.APACK_EINVAL                  # one each without cu_q
    assert status(ap, lambda: plan(seqs=i32(4), n_q=3)) == ap.APACK_EINVAL
    assert status(ap, lambda: plan(ws=ws[:1024])) == ap.APACK_EWORKSPACE
    assert status(ap, lambda: plan(ws=ws[64:])) == ap.APACK_EINVAL
    assert status(ap, lambda: plan(heads=30)) == ap.APACK_EINVAL
    assert status(ap, lambda: plan(cu_groups=i32(5), prefix=i32(4))) == ap.APACK_EINVAL     # more groups than entries
    for bad in (dict(lens=i32(2)), dict(lens=torch.zeros(3, dtype=torch.int64)), dict(cu_q=i32(3)), dict(cu_groups=i32(2)),
                dict(prefix=i32(1)), dict(cu_groups=i32(3), prefix=i32(1)), dict(seqs=i32(3, 1)), dict(seqs=i32(6)[::2])):
        with pytest.raises(ValueError):
            plan(**bad)


def test_attention_arguments(ap):
    c = cache(ap)
    ws = workspace(ap.apack_paged_group_workspace_size(c, 28, 3, 5))
    q = torch.zeros(5, 30, 128, dtype=torch.bfloat16)
    out = torch.zeros(5, 28, 128, dtype=torch.bfloat16)

    def attend(layer=0, q=q[:, :28], out=out, ws=ws, **kw):
        ap.apack_paged_group_attention(c, layer, q, out, ws, stream=0, **kw)

    for layer in (-1, 2):
        assert status(ap, lambda: attend(layer)) == ap.APACK_EINVAL
    for scale in (0.0, -1.0, math.nan, math.inf, 3e38):
        assert status(ap, lambda: attend(scale=scale)) == ap.APACK_EINVAL
    assert status(ap, lambda: attend(ws=ws[:2048])) == ap.APACK_EWORKSPACE
    assert status(ap, lambda: attend(ws=ws[16:])) == ap.APACK_EINVAL
    same = torch.zeros(5, 28, 128, dtype=torch.bfloat16)
    assert status(ap, lambda: attend(q=same, out=same)) == ap.APACK_EINVAL     # over its own queries
    assert status(ap, lambda: attend()) == ap.APACK_EINVAL                     # host memory
    empty = torch.zeros(0, 28, 128, dtype=torch.bfloat16)
    attend(q=empty, out=empty)                                                 # no tokens: nothing to do
    for bad in (dict(q=q[:, :28].half()), dict(q=q[:, :28, :64]), dict(q=q[:, ::2]), dict(out=out.float()),
                dict(out=out[:4]), dict(lse=torch.zeros(5, 27)), dict(lse=torch.zeros(5, 28, dtype=torch.float64))):
        with pytest.raises(ValueError):
            attend(**bad)


def tables(ap, seqs=4, width=3, pages=9, page=16):
    return ap.PageTables.new(seqs, width, pages, page, device="cpu")


def test_page_table_arguments(ap):
    t = tables(ap)
    assert t.free_list.tolist() == list(range(8, -1, -1)) and int(t.free_count) == 9 and t.page_tokens == 16
    cu, rows = i32(5), i32(8)
    calls = (lambda t, n, **kw: ap.apack_pages_release(t, i32(n), stream=0, **kw),
             lambda t, n, **kw: ap.apack_pages_extend(t, i32(n), i32(n + 1), rows, stream=0, **kw),
             lambda t, n, **kw: ap.apack_pages_fork(t, i32(n), i32(n), stream=0, **kw))
    for call in calls:
        for field, value in (("page_table", None), ("lengths", None), ("refs", None), ("free_list", None),
                             ("free_count", None), ("num_seqs", 0), ("num_seqs", 4097), ("max_pages", 0), ("num_pages", 0),
                             ("page_tokens", 0), ("page_tokens", 2 ** 30 + 1), ("table_stride", 2)):
            bad = tables(ap)
            setattr(bad.struct, field, value)
            assert status(ap, lambda: call(bad, 2)) == ap.APACK_EINVAL, field
        assert status(ap, lambda: call(t, 4097)) == ap.APACK_EINVAL
        assert status(ap, lambda: call(t, 2, ws=torch.zeros(32, dtype=torch.uint8)[1:])) == ap.APACK_EINVAL
    for call in calls[:2]:
        assert status(ap, lambda: call(t, 5)) == ap.APACK_EINVAL                # more entries than sequences
    ap.apack_pages_release(t, i32(0), stream=0)
    ap.apack_pages_fork(t, i32(0), i32(0), stream=0)
    for bad in (lambda: ap.apack_pages_release(t, i32(4).long(), stream=0),
                lambda: ap.apack_pages_release(t, i32(4), seqs=i32(3), stream=0),
                lambda: ap.apack_pages_fork(t, i32(4), i32(8)[::2], stream=0),
                lambda: ap.apack_pages_extend(t, i32(4), i32(4), rows, stream=0),
                lambda: ap.apack_pages_extend(t, i32(4), cu, i32(2, 4), stream=0),
                lambda: ap.apack_pages_extend(t, i32(4), cu, rows, row_seqs=i32(7), stream=0),
                lambda: ap.apack_pages_extend(t, i32(4), cu, rows, slots=i32(8), stream=0),
                lambda: ap.apack_pages_extend(t, i32(4), cu, rows, pairs=i32(3, 2), stream=0),
                lambda: ap.PageTables(i32(4, 3), i32(3), i32(9), i32(9), i32(1), 16),
                lambda: ap.PageTables(i32(4, 3), i32(4), i32(9), i32(8), i32(1), 16),
                lambda: ap.PageTables(i32(4, 6)[:, ::2], i32(4), i32(9), i32(9), i32(1), 16),
                lambda: ap.PageTables(i32(4, 3), i32(4), i32(9), i32(9), i32(2), 16)):
        with pytest.raises(ValueError):
            bad()


# ---------------------------------------------------------------- pins of the oracles


def test_group_oracle_is_the_decode_oracle_of_every_token():
    rng = np.random.default_rng(5)
    k, v = rng.standard_normal((2, 7, 4, 2, 8))
    table = np.array([[3, 1, 6], [0, 2, 5]])
    lens, new = [11, 6], [4, 2]
    q = rng.standard_normal((6, 6, 8))
    got = po.group_attention(q, k, v, table, lens, [1, 0], [2, 4], 0.4)
    at = 0
    for b, m in ((1, 2), (0, 4)):
        for i in range(m):
            want = po.paged_decode(q[at:at + 1], k, v, table[b:b + 1], [lens[b] - m + i + 1], 0.4)
            for x, y in zip(got, want):
                np.testing.assert_allclose(x[at], y[0], rtol=1e-13)
            at += 1
    # more tokens than rows: the first see nothing
    out, lse, _, _ = po.group_attention(q[:3], k, v, table, [2, 6], [0], [3], 0.4)
    assert np.isneginf(lse[0]).all() and (out[0] == 0).all() and np.isfinite(lse[1:]).all()
    np.testing.assert_allclose(out[1], np.repeat(v[3, 0], 3, axis=0), rtol=1e-13)       # one row: its value


def test_page_lists_by_hand():
    p = po.PageLists(4, 4, 8, 4)                      # free: 7 .. 0, 0 on top
    assert p.extend([2, 0], [6, 3]) == ([0, 6, 9], [0, 1, 2, 3, 4, 5, 0, 1, 2], [2] * 6 + [0] * 3,
                                        [0, 1, 2, 3, 4, 5, 8, 9, 10], [(0, 0), (0, 0)])
    assert p.table[2][:2] == [0, 1] and p.table[0][:1] == [2] and p.free == [7, 6, 5, 4, 3]
    p.fork([2], [3])
    assert p.refs == [2, 2, 1, 0, 0, 0, 0, 0] and p.lengths == [3, 0, 6, 6]
    # both write into the shared last page: the first gets a copy, the last holder keeps it
    assert p.extend([3, 2], [3, 1])[3:] == ([14, 15, 16, 6], [(1, 3), (0, 0)])
    assert p.table[3] == [0, 3, 4, -1] and p.refs == [2, 1, 1, 1, 1, 0, 0, 0] and p.free == [7, 6, 5]
    p.release([3, 2], [0, 5])
    assert p.table[3] == [-1] * 4 and p.refs == [1, 1, 1, 0, 0, 0, 0, 0] and p.free == [7, 6, 5, 4, 3]
    p.release([2, 0], [0, 0])
    assert p.free == [7, 6, 5, 4, 3, 2, 1, 0] and p.refs == [0] * 8
