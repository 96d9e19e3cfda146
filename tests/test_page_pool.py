"""PagePool's bookkeeping on the CPU: pages, reference counts and lengths against a model that keeps every
sequence's rows as a list, with the two device calls replaced by the oracle's moves."""

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po


@pytest.fixture()
def pools(monkeypatch):
    import __graft_entry__
    __graft_entry__.build()
    from paper_2608_08794_gb300 import paged

    def copy_pages(cache, pairs, ws=None, stream=None):
        p = pairs.long()
        assert len(set(p[:, 1].tolist())) == len(p) and not set(p[:, 0].tolist()) & set(p[:, 1].tolist())
        for x in (cache.k, cache.v):
            x[:, p[:, 1]] = x[:, p[:, 0]]

    def compact(src, dst, cu_dst, n_out, keep_idx=None, cu_src=None, src_layer=0, dst_layer=0, num_layers=None, ws=None, stream=None):
        n = min(src.num_layers - src_layer, dst.num_layers - dst_layer) if num_layers is None else num_layers
        assert n_out == int(cu_dst[-1])
        for a, b in ((src.k, dst.k), (src.v, dst.v)):
            got = po.move_rows(a[src_layer:src_layer + n].double().numpy(), b[dst_layer:dst_layer + n].double().numpy(),
                               src.page_table.numpy(), dst.page_table.numpy(), cu_dst.tolist(),
                               None if keep_idx is None else keep_idx.tolist(), None if cu_src is None else cu_src.tolist())
            b[dst_layer:dst_layer + n] = torch.from_numpy(got).to(b.dtype)

    monkeypatch.setattr(paged, "apack_copy_pages", copy_pages)
    monkeypatch.setattr(paged, "apack_paged_compact", compact)
    return paged


def make(paged, pages=40, tokens=4, seqs=8, **kw):
    pool = paged.PagePool(2, pages, tokens, 1, 64, seqs, dtype=torch.float16, device="cpu", **kw)
    pool.k.fill_(-1)
    pool.v.fill_(-1)
    return pool


def write(pool, seq, first, values):
    for i, x in enumerate(values):
        page = pool.pages(seq)[(first + i) // pool.page_tokens]
        pool.k[:, page, (first + i) % pool.page_tokens] = x
        pool.v[:, page, (first + i) % pool.page_tokens] = -x


def rows(pool, seq):
    """The sequence as the operators read it: through the device's table and lengths."""
    n = int(pool.lengths[seq])
    page = pool.page_table[seq].tolist()
    out = [float(pool.k[1, page[r // pool.page_tokens], r % pool.page_tokens, 0, 0]) for r in range(n)]
    assert out == [-float(pool.v[0, page[r // pool.page_tokens], r % pool.page_tokens, 0, 63]) for r in range(n)]
    return out


@pytest.mark.parametrize("seed", range(6))
def test_random_operations_against_a_model(pools, seed):
    rng = np.random.default_rng(seed)
    pool = make(pools, heads_first=bool(seed % 2))
    model, value = {}, 0
    for _ in range(150):
        op = rng.choice(["add", "extend", "extend", "fork", "fork", "free", "prune", "prune", "take"])
        held = list(model)
        free, before = pool.free_pages, {s: rows(pool, s) for s in held}
        try:
            if op == "add":
                n = int(rng.integers(0, 14))
                s = pool.add(n)
                model[s] = [value + i for i in range(n)]
                write(pool, s, 0, model[s])
                value += n
            elif op == "take":
                lens = [int(x) for x in rng.integers(1, 9, 2)]
                kept = [int(rng.integers(0, n + 1)) for n in lens]
                import paper_2608_08794_gb300 as ap
                k = torch.zeros(2, 1, sum(lens), 1, 64, dtype=torch.float16)
                k[:, 0, :, 0] = (torch.arange(sum(lens)) + value)[None, :, None].half()
                src = ap.PagedCache(k, -k, torch.zeros(2, 1, dtype=torch.int32))
                keep = np.concatenate([np.sort(rng.permutation(n)[:m]) + o for n, m, o in zip(lens, kept, [0, lens[0]])])
                new = pool.take(src, kept, keep_idx=torch.tensor(keep, dtype=torch.int32))
                at = 0
                for s, m in zip(new, kept):
                    model[s] = [value + int(x) for x in keep[at:at + m]]
                    at += m
                value += sum(lens)
            elif not held:
                continue
            elif op == "extend":
                some = [int(x) for x in rng.permutation(held)[:rng.integers(1, len(held) + 1)]]
                n = int(rng.integers(0, 6))
                first = pool.extend(some, n)
                for s, f in zip(some, first.tolist()):
                    assert f == len(model[s])
                    model[s] = model[s] + [value + i for i in range(n)]
                    write(pool, s, f, model[s][f:])
                    value += n
            elif op == "fork":
                s = int(rng.choice(held))
                model[pool.fork(s)] = list(model[s])
            elif op == "free":
                s = int(rng.choice(held))
                pool.free(s)
                del model[s]
            else:
                some = [int(x) for x in rng.permutation(held)[:rng.integers(1, len(held) + 1)]]
                kept = [int(rng.integers(0, len(model[s]) + 1)) for s in some]
                picks = [np.sort(rng.permutation(len(model[s]))[:m]) for s, m in zip(some, kept)]
                at = np.concatenate([[0], np.cumsum([len(model[s]) for s in some])])
                keep = np.concatenate([p + o for p, o in zip(picks, at)]) if some else []
                own = all(pool._refs[p] == 1 for s in some for p in pool.pages(s))
                where = [s for s in some if own], [list(pool.pages(s)) for s in some]
                way = rng.choice([None, True] if own else [None])
                pool.prune(some, torch.tensor(keep, dtype=torch.int32), kept, in_place=way)
                if way:                                 # the first of their own pages
                    assert all(pool.pages(s) == p[:len(pool.pages(s))] for s, p in zip(*where))
                for s, p in zip(some, picks):
                    model[s] = [model[s][i] for i in p]
        except MemoryError:
            assert pool.free_pages == free and {s: rows(pool, s) for s in held} == before     # nothing has changed
        value %= 2000                                   # exact in fp16
        for s in model:
            assert rows(pool, s) == model[s] and pool.length(s) == len(model[s])
            assert len(pool.pages(s)) == -(-len(model[s]) // pool.page_tokens)
        refs = np.zeros(40, int)
        for s in model:
            refs[pool.pages(s)] += 1
        assert np.array_equal(refs, pool._refs) and sorted(pool._free) == np.flatnonzero(refs == 0).tolist()
    assert value or model


def test_refusals_change_nothing(pools):
    pool = make(pools, pages=3, tokens=4, seqs=2, max_pages=3)
    a = pool.add(9)
    b = pool.fork(a)
    with pytest.raises(MemoryError):
        pool.fork(a)                                    # no row of the table
    with pytest.raises(MemoryError):
        pool.extend([a, b], 1)                          # one of the two needs a copy of the last page
    for bad in (lambda: pool.add(-1), lambda: pool.extend([a], 40), lambda: pool.extend([a, a]), lambda: pool.extend([a], -1),
                lambda: pool.free(5), lambda: pool.length(-1), lambda: pool.prune([a, a], None, [1, 1]),
                lambda: pool.prune([], None, []), lambda: pool.prune([a], None, [1], in_place=True), lambda: pool.prune([a], None, [99]), lambda: pool.take(pool.cache, [1])):
        before = (pool.free_pages, [list(p or []) for p in pool._pages], pool._len.tolist())
        with pytest.raises(ValueError):
            bad()
        assert before == (pool.free_pages, [list(p or []) for p in pool._pages], pool._len.tolist())
    pool.free(b)
    with pytest.raises(ValueError):
        pool.free(b)
    pool.free(a)
    assert pool.free_pages == 3 and int(pool.lengths.sum()) == 0 and int(pool.page_table.max()) == -1


def test_device_tables_follow_the_host(pools):
    """After every call the device's table holds a sequence's pages and -1 behind them, and its length."""
    pool = make(pools)

    def check():
        for s, pages in enumerate(pool._pages):
            pages = pages or []
            assert pool.page_table[s].tolist() == pages + [-1] * (pool.max_pages - len(pages))
        assert pool.lengths.tolist() == pool._len.tolist() and pool.lengths.dtype == torch.int32

    a, b = pool.add(9), pool.add(0)
    check()
    c = pool.fork(a)
    check()
    assert pool.extend([]).tolist() == []
    assert pool.extend((c, b, a), 11).tolist() == [9, 0, 9]       # a copy, new pages of three sequences
    check()
    assert pool.extend(np.array([b]), 0).tolist() == [11]
    pool.prune([a, b], torch.arange(31, dtype=torch.int32)[[0, 19, 20, 30]], [2, 2])
    check()
    pool.prune([c], torch.tensor([3, 4], dtype=torch.int32), [2], in_place=True)
    check()
    pool.free(a)
    pool.free(b)
    pool.free(c)
    check()
    assert pool.free_pages == 40 and pool._shared == 0
