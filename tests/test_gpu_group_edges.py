"""Attention over shared rows where it can go wrong: masked values that are no numbers, growing maxima, long caches, captured
calls that follow their inputs, what the device finds wrong, and a pool's calls together as a server makes them."""

import math
import os
import re
import subprocess
import sys

import numpy as np
import pytest
import torch

from test_gpu_group import Batch, DT, f64, i32, workspace

pytestmark = pytest.mark.gpu

NAN = float("nan")


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def slot(b, seq, row):
    page = b.k.shape[2]
    return int(b.table[seq][row // page]), row % page


@pytest.mark.parametrize("heads,dim,page", [("28/4", 128, 16), ("8/8", 64, 32), ("4/2", 128, 7)])
@pytest.mark.parametrize("bad", [NAN, math.inf, -math.inf])
def test_what_a_token_does_not_see_may_be_no_number(ap, heads, dim, page, bad):
    """The second sequence's last two keys and values: its tokens before them, and every other sequence, are as they were."""
    b = Batch(ap, heads, dim, "bf16", page, [(70, [(90, 3), (140, 6), (75, 1)]), (0, [(33, 5)])], seed=3)
    b.plan()
    want = b.attend()
    n, seq = b.seqlens[b.seqs[1]], b.seqs[1]
    keep = []
    for row in (n - 1, n - 2):
        p, s = slot(b, seq, row)
        for x in (b.k, b.v):
            keep.append(x[0, p, s].clone())
            x[0, p, s] = bad
    out, lse = b.attend()
    sees = list(range(0, 7)) + list(range(9, sum(b.new)))                # all but the two tokens that see them
    b2 = Batch(ap, heads, dim, "bf16", page, [(70, [(90, 3), (140, 6), (75, 1)]), (0, [(33, 5)])], seed=3)
    b2.check(out, lse, rows=sees)
    assert torch.isnan(out[7:9]).all() or not math.isnan(bad)
    assert not torch.equal(out[7:9], want[0][7:9])
    assert ap.apack_device_error(b.ws) == 0


def test_a_number_that_is_none_reaches_those_that_see_it(ap):
    b = Batch(ap, "8/2", 128, "bf16", 16, [(64, [(80, 1), (90, 2)])], seed=4)
    p, s = slot(b, b.seqs[0], 10)                                        # a shared row
    b.v[0, p, s] = NAN
    b.plan()
    out, _ = b.attend()
    assert torch.isnan(out[:sum(b.new)]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rising", [True, False])
def test_growing_and_falling_maxima(ap, dtype, rising):
    """Scores that grow tile by tile (a new reference in each), and ones that end far below the first."""
    b = Batch(ap, "8/2", 128, dtype, 64, [(1024, [(1100, 2), (1024 + 33, 1)]), (0, [(900, 40)])], seed=5, scale=0.5)
    longest = 1200
    for seq in b.seqs:
        n = int(b.seqlens[seq])
        for row in range(0, n):
            p, s = slot(b, seq, row)
            level = (row if rising else longest - row) / longest * 3.0
            b.k[0, p, s] = (b.k[0, p, s].float() * 0.1 + level).to(b.dt)
    b.q.copy_((b.q.float().abs() * 0.3 + 0.2).to(b.dt))
    b.plan()
    b.check(*b.attend())


def reference(b, layer=0):
    """fp64 on the GPU, for sizes that the oracle's loops take too long for."""
    page, real = b.k.shape[2], sum(b.new)
    out = torch.zeros(real, b.hq, b.dim, dtype=torch.float64, device="cuda")
    lse = torch.full((real, b.hq), -math.inf, dtype=torch.float64, device="cuda")
    g, at = b.hq // b.hkv, 0
    for seq, m in zip(b.seqs, b.new):
        n = int(b.seqlens[seq])
        pages = torch.tensor(b.table[seq][:-(-n // page)], device="cuda")
        for h in range(b.hkv if m and n else 0):
            k = b.k[layer, pages, :, h].flatten(0, 1)[:n].double()
            v = b.v[layer, pages, :, h].flatten(0, 1)[:n].double()
            q = b.q[layer, at:at + m, h * g:(h + 1) * g].double().transpose(0, 1)
            x = q @ k.T * b.scale
            seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - m, n, device="cuda")[:, None]
            x = x.masked_fill(~seen, -math.inf)
            z = torch.logsumexp(x, -1)
            x = x.masked_fill(~seen.any(1)[:, None], 0.0) - z.masked_fill(torch.isneginf(z), math.inf)[..., None]
            lse[at:at + m, h * g:(h + 1) * g] = z.T
            out[at:at + m, h * g:(h + 1) * g] = (x.exp() @ v).transpose(0, 1)
        at += m
    return out, lse


def near(b, out, lse, rows=slice(None)):
    """Every row within 4 of the type's roundings of the reference's norm (the output's, the weights' and as much again for their
    sums), lse within 2^-14."""
    real = sum(b.new)
    ref, ref_lse = reference(b)
    u = torch.finfo(b.dt).eps / 2
    far = torch.linalg.norm(out[:real].double() - ref, dim=-1) - 4 * u * torch.linalg.norm(ref, dim=-1)
    assert (far[rows] <= 1e-3).all(), far[rows].max()
    off = (lse[:real].double() - ref_lse)[rows]
    assert (off[torch.isfinite(ref_lse[rows])].abs() <= 2.0 ** -14).all()
    assert torch.equal(torch.isneginf(lse[:real][rows]), torch.isneginf(ref_lse[rows]))
    assert (out[real:] == 7).all() and (lse[real:] == 7).all()


@pytest.mark.parametrize("heads,dim,dtype,page,groups", [
    ("28/4", 128, "bf16", 16, [(40000, [(40100, 1), (40001, 3)])]),              # many runs of keys
    ("8/1", 128, "bf16", 64, [(30000, [(30030, 30)])]),
    ("28/4", 128, "bf16", 64, [(3000, [(3000 + m, m) for m in range(1, 60, 2)])]),   # many runs of rows
    ("8/8", 64, "fp16", 32, [(2000, [(2000 + m, m) for m in (1, 2, 5, 300)])]),
    ("16/2", 128, "fp16", 24, [(0, [(5000, 1500)])]),
    ("28/4", 64, "bf16", 128, [(0, [(300, 300)]), (999, [(1300, 301)] * 3)]),
    ("12/2", 128, "bf16", 16, [(200 + i, [(200 + i + j, 1) for j in range(1, 1 + i % 5)]) for i in range(1, 60)]),
    ("3/1", 128, "bf16", 16, [(0, [(5 + i, 1)]) for i in range(700)]),             # many sequences, nothing shared
])
def test_long_and_large(ap, heads, dim, dtype, page, groups):
    b = Batch(ap, heads, dim, dtype, page, groups, seed=len(groups))
    b.plan()
    out, lse = b.attend()
    ref, ref_lse = reference(b)
    real = sum(b.new)
    u = torch.finfo(b.dt).eps / 2
    # values and keys are standard normal (1.3 for keys): |v| <= 6 and sum_i |q_i k_i| <= 6 * 8 * sqrt(dim)
    assert torch.linalg.norm(out[:real].double() - ref) <= 2 * u * torch.linalg.norm(ref)
    rows = torch.linalg.norm(out[:real].double() - ref, dim=-1)
    assert (rows <= 4 * u * torch.linalg.norm(ref, dim=-1) + 1e-3).all()
    assert (lse[:real].double() - ref_lse).abs().max() <= 2.0 ** -14
    assert ap.apack_device_error(b.ws) == 0


def test_draws(ap):
    """Batches at random, against 64 bits."""
    rng = np.random.default_rng(11)
    for i in range(40):
        heads = ("28/4", "16/2", "8/8", "5/1", "32/8", "9/3")[rng.integers(6)]
        groups = []
        for _ in range(rng.integers(1, 6)):
            shared = int(rng.integers(0, 700))
            members = []
            for _ in range(rng.integers(1, 9)):
                m = int(rng.choice([0, 1, 1, 1, 2, 7, 40]))
                members.append((shared + m + int(rng.integers(0, 200)), m))
            groups.append((shared, members))
        b = Batch(ap, heads, int(rng.choice([64, 128])), str(rng.choice(["bf16", "fp16"])), int(rng.choice([1, 8, 16, 24, 64, 128, 512])),
                  groups, order=str(rng.choice(["nhd", "hnd", "inside"])), seed=100 + i, pad=int(rng.integers(0, 4)))
        if sum(b.new) == 0:
            continue
        b.plan()
        out, lse = b.attend()
        ref, ref_lse = reference(b)
        real = sum(b.new)
        u = torch.finfo(b.dt).eps / 2
        rows = torch.linalg.norm(out[:real].double() - ref, dim=-1)
        assert (rows <= 4 * u * torch.linalg.norm(ref, dim=-1) + 1e-3).all(), i
        assert (lse[:real].double() - ref_lse).abs().max() <= 2.0 ** -14, i
        assert (out[real:] == 7).all() and (lse[real:] == 7).all()
        assert ap.apack_device_error(b.ws) == 0


def test_queries_out_of_a_projection_and_layers(ap):
    b = Batch(ap, "28/4", 128, "bf16", 16, [(100, [(130, 2), (101, 1)])], layers=3, seed=6)
    b.plan()
    wide = torch.randn(b.n_q, 28 + 8, 128, device="cuda").bfloat16()
    for layer in (2, 0, 1):
        wide[:, :28] = b.q[layer]
        out, lse = b.outputs()
        ap.apack_paged_group_attention(b.cache, layer, wide[:, :28], out, b.ws, lse=lse)
        b.check(out, lse, layer)
    one = Batch(ap, "8/2", 64, "fp16", 16, [(0, [(9, 1)])], seed=7)
    one.plan()
    out, _ = one.outputs()
    ap.apack_paged_group_attention(one.cache, 0, one.q[0], out, one.ws)                 # no lse
    assert torch.equal(out, one.attend()[0])
    one.scale = 0.31
    out, lse = one.outputs()
    ap.apack_paged_group_attention(one.cache, 0, one.q[0], out, one.ws, scale=0.31, lse=lse)
    one.check(out, lse)


def test_captured_calls_follow_their_inputs(ap):
    """A plan and two layers in one graph, with room for more tokens than there are: lengths, tokens and groups change under it."""
    b = Batch(ap, "28/4", 128, "bf16", 16, [(300, [(340, 6), (310, 5), (333, 7)]), (0, [(200, 4)])], layers=2, seed=8, pad=5)
    outs = [b.outputs() for _ in range(2)]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            b.plan()
            for layer in range(2):
                ap.apack_paged_group_attention(b.cache, layer, b.q[layer], outs[layer][0], b.ws, lse=outs[layer][1])
    full, lens = list(b.new), b.seqlens.copy()
    for cut, grouped in ((0, True), (2, True), (4, False), (1, True)):
        b.new = [max(m - cut, 0) for m in full]
        b.seqlens = lens.copy()
        for seq, m, was in zip(b.seqs, b.new, full):
            b.seqlens[seq] -= was - m
        b.cu_q.copy_(i32(np.concatenate([[0], np.cumsum(b.new)])))
        b.lens.copy_(i32(b.seqlens))
        b.prefix.copy_(i32([300 if grouped else 0, 0]))
        for o, l in outs:
            o.fill_(7)
            l.fill_(7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for layer in range(2):
            b.check(*outs[layer], layer)
    assert ap.apack_device_error(b.ws) == 0


def test_a_workspace_takes_one_plan_after_another(ap):
    big = Batch(ap, "28/4", 128, "bf16", 16, [(500, [(600, 9), (505, 2)])], seed=9)
    small = Batch(ap, "28/4", 128, "bf16", 16, [(16, [(17, 1), (20, 1)])], seed=10)
    small.ws = big.ws
    for _ in range(2):
        for b in (big, small):
            b.plan()
            b.check(*b.attend())
    # a plan of other sizes than the call's is refused on the device, and nothing is written
    small.plan()
    out, lse = big.attend()
    assert (out == 7).all() and (lse == 7).all() and ap.apack_device_error(big.ws) == ap.APACK_EDEVICE
    fresh = workspace(big.ws.numel())
    big.ws = fresh                                                       # no plan at all
    out, lse = big.attend()
    assert (out == 7).all() and (lse == 7).all() and ap.apack_device_error(fresh) == ap.APACK_EDEVICE
    big.plan()
    big.check(*big.attend())
    assert ap.apack_device_error(fresh) == 0


def test_what_the_device_finds_wrong(ap):
    def fresh():
        b = Batch(ap, "8/2", 128, "bf16", 16, [(64, [(80, 3), (70, 2)]), (0, [(30, 1)])], seed=12)
        return b
    # offsets that do not rise, or pass n_q: no plan, nothing written
    for cu in ([0, 3, 2, 6], [1, 3, 5, 6], [0, 3, 5, 7], [0, 3, 5, -1]):
        b = fresh()
        b.cu_q = i32(cu)
        b.plan()
        assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
        out, lse = b.attend()
        assert (out == 7).all() and (lse == 7).all()
        assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
    for cu in ([0, 2, 4], [0, -1, 3], [2, 1, 3]):
        b = fresh()
        b.cu_g = i32(cu)
        b.plan()
        assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
    # an entry outside the cache gives zeros, the others are right
    b = fresh()
    b.seqs_d = b.seqs_d.clone()
    b.seqs_d[2] = 99
    b.plan()
    assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
    out, lse = b.attend()
    assert (out[5] == 0).all() and torch.isneginf(lse[5]).all()
    b.check(out, lse, rows=slice(0, 5))
    # a prefix beyond the first entry's rows, below 0, and a length beyond the table: the nearest in range
    b = fresh()
    b.prefix = i32([10 ** 6, 0])
    b.plan(grouped=True)
    assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
    b = fresh()
    b.prefix = i32([-5, 0])
    b.plan()
    assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
    b.check(*b.attend())
    b = fresh()
    b.lens[int(b.seqs[2])] = -3
    b.plan()
    assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
    out, lse = b.attend()
    assert (out[5] == 0).all() and torch.isneginf(lse[5]).all()
    b.check(out, lse, rows=slice(0, 5))
    # more tokens than rows: the first see nothing
    b = fresh()
    b.seqlens[b.seqs[2]] = 0
    b.lens[int(b.seqs[2])] = 0
    b.plan()
    assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
    b.check(*b.attend())
    # a page outside the pool reads as zeros
    for page in (16, 7):
        b = Batch(ap, "8/2", 128, "bf16", page, [(0, [(40, 2)])], seed=13)
        table = b.table.copy()
        table[b.seqs[0], 1] = 10 ** 6
        b.cache = ap.PagedCache(b.k, b.v, i32(table))
        b.plan()
        out, lse = b.attend()
        assert ap.apack_device_error(b.ws) == ap.APACK_EDEVICE
        p = int(b.table[b.seqs[0], 1])
        b.k[:, p], b.v[:, p] = 0, 0
        b.check(out, lse)


@pytest.mark.parametrize("members,shared", [([(900, 1)] * 2 + [(880, 3)], True), ([(1000, 300), (980, 290), (950, 200)], False)])
def test_rows_are_read_together_where_that_saves_products(ap, members, shared):
    """A NaN in the shared rows of the second sequence's own pages shows whose were read: the first's for all, or each its own."""
    b = Batch(ap, "8/2", 128, "bf16", 64, [(640, members)], seed=14)
    b.plan()
    b.check(*b.attend())
    page = next(i for i in range(b.k.shape[1]) if i not in b.table)               # a page of nobody
    table = b.table.copy()
    table[b.seqs[1], 3] = page
    b.k[:, page], b.v[:, page] = 0.0, NAN
    b.cache = ap.PagedCache(b.k, b.v, i32(table))
    b.plan()
    out, _ = b.attend()
    m0, m1 = b.new[0], b.new[1]
    assert not torch.isnan(out[:m0]).any() and not torch.isnan(out[m0 + m1:sum(b.new)]).any()
    assert torch.isnan(out[m0:m0 + m1]).all() == (not shared)


def test_rows_of_one_part_are_written_out_at_once(ap):
    """Sequences that share nothing and are short: no part, the same rules (tails, masks, what is no number, tokens that see nothing)."""
    cases = [("28/4", 128, "bf16", 16, [(0, [(200 + 40 * i, 60 + 10 * i)]) for i in range(40)]),
             ("8/8", 64, "fp16", 32, [(0, [(300 + i, 290 + i % 9)]) for i in range(60)]),
             ("5/1", 128, "fp16", 7, [(0, [(260, 260)]) for i in range(80)])]
    for heads, dim, dtype, page, groups in cases:
        b = Batch(ap, heads, dim, dtype, page, groups, seed=15, pad=2)
        b.plan()
        segs = b.ws[1024 + (b.n_q * 16 + 255) // 256 * 256:].view(torch.int32)[:8 * int(b.ws[256:352].view(torch.int32)[9])]
        assert (segs.view(-1, 8)[:, 7] == -1).any()            # some are
        near(b, *b.attend())
        seq = b.seqs[3]
        p, s = slot(b, seq, int(b.seqlens[seq]) - 1)
        b.v[0, p, s] = NAN
        at = sum(b.new[:3])
        out, lse = b.attend()
        assert torch.isnan(out[at + b.new[3] - 1]).all()
        b.v[0, p, s] = 0.0
        near(b, out, lse, rows=[i for i in range(sum(b.new)) if i != at + b.new[3] - 1])
        b.lens[int(b.seqs[5])] = b.new[5] - 4                  # its first four tokens see nothing
        b.seqlens[b.seqs[5]] = b.new[5] - 4
        b.plan()
        near(b, *b.attend())


@pytest.mark.parametrize("page", [16, 7])
def test_pages_beyond_four_gigabytes(ap, page):
    """TMA boxes and rows by the lanes, from the end of a pool of 5 GB of keys.

    Per value: half a step of bf16 for each probability, half a step for the output, and as much again for fp32's sums and exponentials.
    """
    n, pages = 300, 5 * 2 ** 30 // (page * 4 * 128 * 2)
    k, v = (torch.empty(1, pages, page, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    need = -(-n // page)
    used = torch.arange(pages - need, pages, device="cuda").flip(0)
    for x in (k, v):
        x[0, used] = torch.randn(need, page, 4, 128, device="cuda").bfloat16()
    cache = ap.PagedCache(k, v, used.to(torch.int32)[None].repeat(2, 1))
    q = torch.randn(5, 28, 128, device="cuda").bfloat16()
    out = torch.empty_like(q)
    ws = workspace(ap.apack_paged_group_workspace_size(cache, 28, 2, 5))
    ap.apack_paged_group_plan(cache, i32([n, n]), 28, 5, ws, cu_q=i32([0, 2, 5]), cu_groups=i32([0, 2]), prefix=i32([n - 40]))
    ap.apack_paged_group_attention(cache, 0, q, out, ws)
    assert ap.apack_device_error(ws) == 0
    kk, vv = (x[0, used].flatten(0, 1)[:n].double() for x in (k, v))
    for t, seen in enumerate((n - 1, n, n - 2, n - 1, n)):
        for h in range(28):
            p = torch.softmax(kk[:seen, h // 7] @ q[t, h].double() / math.sqrt(128), 0)
            ref = p @ vv[:seen, h // 7]
            assert ((out[t, h].double() - ref).abs() <= 2.0 ** -8 * (ref.abs() + 2 * (p @ vv[:seen, h // 7].abs()))).all()


FIRST = r"""
import sys, threading
import torch
sys.path.insert(0, sys.argv[1])
import __graft_entry__
__graft_entry__.build()
import paper_2608_08794_gb300 as ap
torch.manual_seed(0)
n, hq, hkv, dim = 300, 16, 4, int(sys.argv[2])
dt = torch.bfloat16 if sys.argv[3] == "bf16" else torch.float16
k, v = (torch.randn(1, 20, 16, hkv, dim, device="cuda").to(dt) for _ in range(2))
cache = ap.PagedCache(k, v, torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20) % 20)
lens, cu, pre = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([n, n - 3], [0, 2], [256]))
ws = torch.zeros(ap.apack_paged_group_workspace_size(cache, hq, 2, 2), dtype=torch.uint8, device="cuda")
q = torch.randn(2, hq, dim, device="cuda").to(dt)
out = torch.empty_like(q)
tables = ap.PageTables.new(3, 4, 9, 16)
grow, cu_new, rows = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([20, 3, 0], [0] * 4, [0] * 30))
torch.cuda.synchronize()
assert ap.apack_launch_count() == 0
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    ap.apack_pages_release(tables, lens.new_zeros(3))
    ap.apack_pages_extend(tables, grow, cu_new, rows)
    ap.apack_paged_group_plan(cache, lens, hq, 2, ws, cu_groups=cu, prefix=pre)
    ap.apack_paged_group_attention(cache, 0, q, out, ws)
for _ in range(3):
    g.replay()
torch.cuda.synchronize()
want = out.clone()
assert tables.lengths.tolist() == [20, 3, 0] and cu_new.tolist() == [0, 20, 23, 23], (tables.lengths, cu_new)
assert rows.tolist() == list(range(20)) + [0, 1, 2] + [-1] * 7
go, errors, outs = threading.Barrier(2), [], {}
def work(i):
    try:
        torch.cuda.set_device(0)
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            w, o = ws.clone(), torch.empty_like(out)
            s.synchronize()
            go.wait()
            for _ in range(50):
                ap.apack_paged_group_plan(cache, lens, hq, 2, w, cu_groups=cu, prefix=pre)
                ap.apack_paged_group_attention(cache, 0, q, o, w)
            s.synchronize()
        outs[i] = o
    except Exception as e:
        errors.append(e)
ts = [threading.Thread(target=work, args=(i,)) for i in range(2)]
for t in ts: t.start()
for t in ts: t.join()
assert not errors, errors
assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
assert ap.apack_device_error(ws) == ap.APACK_OK
print("first calls ok")
"""


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (64, "bf16"), (128, "fp16"), (64, "fp16")])
def test_first_calls_captured_and_from_two_threads(dim, dtype):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST, root, str(dim), dtype], capture_output=True, text=True, cwd=root, timeout=600)
    assert r.returncode == 0 and "first calls ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


def test_the_readme_step_of_questions(ap):
    """README's step over a DevicePool, run as written, against 64 bits."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        block, = [x for x in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "DevicePool" in x]
    torch.manual_seed(3)
    n, m = 333, [5, 1, 12]
    n_q = sum(m)
    k, v = (torch.randn(28, n, 4, 128, device="cuda").bfloat16() for _ in range(2))
    new = torch.randn(28, n_q, 36, 128, device="cuda").bfloat16()
    q_rot, out = (torch.empty(n_q, 28, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    names = dict(ap=ap, torch=torch, k=k, v=v, n=n, n_q=n_q, q_rot=q_rot, out=out, video=i32([0]), video_rows=i32([n]),
                 parents=i32([0, 0, 0]), questions=i32([1, 2, 3]), new_rows=i32(m), bounds=i32([0, 3]), nothing=i32([0, 0, 0]),
                 rotary=ap.Rotary(128), positions=i32([n + i for x in m for i in range(x)]),
                 project=lambda layer: (new[layer][:, :28], new[layer][:, 28:32], new[layer][:, 32:]))
    exec(block, names)
    pool = names["pool"]
    assert ap.apack_device_error(names["ws"]) == 0
    assert pool.lengths.tolist()[:5] == [n, 0, 0, 0, 0] and int(pool.tables.free_count) == 4096 - -(-n // 16)
    x = new[27].double()
    turn = torch.zeros(n_q, 32, 128, dtype=torch.float64, device="cuda")
    angle = names["positions"].double()[:, None] * torch.tensor(names["rotary"].frequencies, device="cuda")[None]
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    turn[..., :64], turn[..., 64:] = x[:, :32, :64] * c - x[:, :32, 64:] * s, x[:, :32, 64:] * c + x[:, :32, :64] * s
    at = 0
    for count in m:
        kk = torch.cat([k[27].double(), turn[at:at + count, 28:].bfloat16().double()])
        vv = torch.cat([v[27].double(), x[at:at + count, 32:]])
        for i in range(count):
            for h in range(28):
                q = q_rot[at + i, h].double()
                p = torch.softmax(kk[:n + i + 1, h // 7] @ q / math.sqrt(128), 0)
                ref = p @ vv[:n + i + 1, h // 7]
                # 4 roundings of bf16 (output, weights, and the new keys, whose own may fall the other way) of sums of |v|
                tol = 2.0 ** -8 * (ref.abs() + 3 * (p @ vv[:n + i + 1, h // 7].abs()))
                assert ((out[at + i, h].double() - ref).abs() <= tol).all()
        at += count


def test_the_pool_of_the_host_names_its_groups(ap):
    from paper_2608_08794_gb300.paged import PagePool
    pool = PagePool(1, 60, 16, 2, 128, 12)
    a, c = pool.add(100), pool.add(33)
    for x in (pool.k, pool.v):
        x.normal_()
    kids = [pool.fork(a) for _ in range(3)]
    pool.extend(kids + [c])                                              # copies of a's last page
    order, bounds, prefix = pool.groups([c, kids[2], kids[0], kids[1]])
    assert order == [c, kids[2], kids[0], kids[1]] and bounds.tolist() == [0, 1, 4] and prefix.tolist() == [0, 96]
    q = torch.randn(4, 8, 128, device="cuda").bfloat16()
    outs = []
    for grouped in (True, False):
        ws = workspace(ap.apack_paged_group_workspace_size(pool.cache, 8, 4, 4))
        out = torch.empty_like(q)
        ap.apack_paged_group_plan(pool.cache, pool.lengths, 8, 4, ws, seqs=i32(order), cu_groups=bounds if grouped else None,
                                  prefix=prefix if grouped else None)
        ap.apack_paged_group_attention(pool.cache, 0, q, out, ws)
        assert ap.apack_device_error(ws) == 0
        outs.append(out.float())
    # and beside the one-token call of the same rows
    full = torch.zeros(12, 8, 128, dtype=torch.bfloat16, device="cuda")
    full[torch.tensor(order, device="cuda")] = q
    dec = torch.empty(12, 8, 128, dtype=torch.bfloat16, device="cuda")
    ws = workspace(ap.apack_paged_decode_workspace_size(pool.cache, 8))
    ap.apack_paged_decode_attention(pool.cache, 0, pool.lengths, full, dec, ws)
    outs.append(dec[torch.tensor(order, device="cuda")].float())
    # |v| <= 6: an output is a mean of values; two roundings of its own and of the weights on either side
    assert (outs[0] - outs[1]).abs().max() <= 4 * 2.0 ** -8 * 6 and (outs[0] - outs[2]).abs().max() <= 4 * 2.0 ** -8 * 6
