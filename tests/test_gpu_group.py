"""Attention over shared rows on the GPU against the fp64 oracle.

Tolerances (u = eps/2 of the type, its rounding; A = sum_r p_r |v_r|, d = 2^-20 max_r scale sum_i |q_i k_i|):

out   |got - ref| <= u |ref| + A (u + 2^-16 + n 2^-23 + 2 d): the output's rounding, P as one 16-bit number (u of each), exp2
      and the factors of partial sums (2^-16), n = ceil(rows / 16) + 400 sequential fp32 additions (parts among them), and
      logits that are off by d (8 fp32 accumulations that may truncate, the scale, log2 units).  fp16: + rows 2^-36
      max |v|, the spacing of its smallest numbers against probabilities of up to 2^11 and more, and 2^-25, the
      spacing of its smallest outputs.
lse   |got - ref| <= 2 d + n 2^-23 + 2^-21 (1 + |ref|).
"""

import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def f64(t):
    return t.detach().cpu().double().numpy()


def workspace(n):
    raw = torch.zeros(n + 256, dtype=torch.uint8, device="cuda")
    return raw[(-raw.data_ptr()) % 256:][:n]


class Batch:
    """Sequences in groups that share pages: groups is a list of (shared rows, [(length, new tokens), ...]).

    The first shared rows // page pages of a group are the same; prefix says all shared rows (the rest is the same by
    value).  Every slot that holds no row is NaN, and so is a whole page of its own; entries behind a sequence's pages
    are -1."""

    def __init__(self, ap, heads, dim, dtype, page, groups, order="nhd", layers=1, seed=0, scale=1.3, spare_rows=2, pad=0):
        rng = np.random.default_rng(seed)
        hq, hkv = map(int, heads.split("/"))
        dt = DT[dtype]
        tables, lens, new, prefix, cu_g, total, copies = [], [], [], [], [0], 1, []
        for shared, members in groups:
            first = len(tables)
            for x, (n, m) in enumerate(members):
                common = min(shared, n) // page if len(members) > 1 else 0
                if x == 0:
                    mine = list(range(total, total - (-n // page)))
                    total += -(-n // page)
                else:
                    need = -(-n // page) - common
                    mine = tables[first][:common] + list(range(total, total + need))
                    total += need
                    if common * page < min(shared, n):        # the rows of the last shared page that is not whole
                        copies.append((tables[first][common], mine[common], min(shared, n) - common * page))
                tables.append(mine)
                lens.append(n)
                new.append(m)
            prefix.append(shared)
            cu_g.append(len(tables))
        total += 2
        perm = rng.permutation(total)
        place = rng.permutation(len(tables) + spare_rows)[:len(tables)]
        width = max(1, max(len(t) for t in tables))
        table = np.full((len(tables) + spare_rows, width), -1)
        seqlens = np.zeros(len(tables) + spare_rows, np.int64)
        shape = (layers, total, page, hkv, dim)
        k = (rng.standard_normal(shape) * scale).astype(np.float32)
        v = rng.standard_normal(shape).astype(np.float32)
        written = np.zeros((total, page), bool)
        for t, n, b in zip(tables, lens, place):
            table[b, :len(t)] = perm[t]
            seqlens[b] = n
            for c, p in enumerate(t):
                written[perm[p], :min(page, n - c * page)] = True
        for a, b, rows in copies:
            k[:, perm[b], :rows], v[:, perm[b], :rows] = k[:, perm[a], :rows], v[:, perm[a], :rows]
        k[:, ~written] = np.nan
        v[:, ~written] = np.inf
        def pool(x):
            t = torch.from_numpy(x).to(dt).cuda()
            if order == "hnd":
                return t.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
            if order == "inside":                          # layers inside pages, a gap behind every token
                wide = torch.full((total, layers, page, hkv + 1, dim), float("nan"), dtype=dt, device="cuda")
                wide[:, :, :, :hkv] = t.transpose(0, 1)
                return wide.transpose(0, 1)[:, :, :, :hkv]
            return t
        self.ap, self.hq, self.hkv, self.dim, self.dt, self.layers = ap, hq, hkv, dim, dt, layers
        self.k, self.v = pool(k), pool(v)
        self.table, self.seqlens, self.seqs, self.new = table, seqlens, place, new
        self.cache = ap.PagedCache(self.k, self.v, i32(table))
        self.n_q = sum(new) + pad
        self.q = torch.from_numpy(rng.standard_normal((layers, self.n_q, hq, dim)).astype(np.float32)).to(dt).cuda()
        self.cu_q = i32(np.concatenate([[0], np.cumsum(new)]))
        self.cu_g, self.prefix = i32(cu_g), i32(prefix)
        self.lens, self.seqs_d = i32(seqlens), i32(place)
        self.ws = workspace(ap.apack_paged_group_workspace_size(self.cache, hq, len(place), self.n_q))
        self.scale = 1.0 / math.sqrt(dim)

    def plan(self, grouped=True):
        self.ap.apack_paged_group_plan(self.cache, self.lens, self.hq, self.n_q, self.ws, cu_q=self.cu_q, seqs=self.seqs_d,
                                       cu_groups=self.cu_g if grouped else None, prefix=self.prefix if grouped else None)

    def outputs(self):
        out = torch.full((self.n_q, self.hq, self.dim), 7.0, dtype=self.dt, device="cuda")
        return out, torch.full((self.n_q, self.hq), 7.0, dtype=torch.float32, device="cuda")

    def attend(self, layer=0):
        out, lse = self.outputs()
        self.ap.apack_paged_group_attention(self.cache, layer, self.q[layer], out, self.ws, lse=lse)
        return out, lse

    def expected(self, layer=0):
        clean = [np.nan_to_num(f64(x[layer]), nan=0.0, posinf=0.0, neginf=0.0) for x in (self.k, self.v)]
        return po.group_attention(f64(self.q[layer]), clean[0], clean[1], self.table, self.seqlens, self.seqs, self.new,
                                  self.scale)

    def check(self, out, lse, layer=0, rows=slice(None)):
        real = sum(self.new)
        ref, ref_lse, spread, size = self.expected(layer)
        longest = int(self.seqlens.max())
        u = torch.finfo(self.dt).eps / 2
        n = math.ceil(longest / 16) + 400
        d = 2.0 ** -20 * size
        tol = u * np.abs(ref) + spread * (u + 2.0 ** -16 + n * 2.0 ** -23 + 2 * d[..., None])
        if self.dt == torch.float16:
            tol = tol + longest * 2.0 ** -36 * 6 + 2.0 ** -25
        got, got_lse = f64(out), f64(lse)
        assert np.all(got[real:] == 7.0) and np.all(got_lse[real:] == 7.0)          # behind the last sequence
        sel = np.arange(real)[rows]
        err = np.abs(got - ref)[sel]
        assert np.all(err <= tol[sel]), (np.nanmax(err / tol[sel]), np.argwhere(~(err <= tol[sel]))[:5])
        empty = np.isneginf(ref_lse[sel])
        assert np.all(np.isneginf(got_lse[sel]) == empty)
        assert np.all(got[sel][empty] == 0)
        with np.errstate(invalid="ignore"):
            far = np.abs(got_lse - ref_lse)[sel]
            bound = (2 * d + n * 2.0 ** -23 + 2.0 ** -21 * (1 + np.abs(ref_lse)))[sel]
        assert np.all((far <= bound) | empty), np.nanmax(far - bound)


CASES = [
    ("28/4", 128, "bf16", 16, [(0, [(1, 1)])]),
    ("28/4", 128, "bf16", 16, [(64, [(70, 1), (65, 1)])]),
    ("28/4", 128, "bf16", 16, [(473, [(500, 1), (474, 1), (600, 1)]), (0, [(17, 1)]), (33, [(33, 1), (40, 3)])]),
    ("28/4", 128, "bf16", 64, [(1000, [(1001 + 7 * i, 1) for i in range(40)])]),
    ("28/4", 128, "bf16", 64, [(700, [(700 + m, m) for m in (1, 12, 60, 33)])]),
    ("28/4", 128, "fp16", 16, [(0, [(700, 300)])]),
    ("28/4", 128, "bf16", 16, [(0, [(300, 300)]), (0, [(129, 2)]), (0, [(1, 1)])]),
    ("16/2", 128, "fp16", 16, [(300, [(300 + i, 1 + i % 3) for i in range(1, 20)]), (128, [(128, 1), (200, 5)])]),
    ("8/8", 64, "fp16", 32, [(100, [(100 + i, 1) for i in range(1, 15)]), (257, [(300, 4), (270, 5)])]),
    ("8/8", 64, "bf16", 128, [(256, [(256 + 5, 5), (257, 1)])]),
    ("12/2", 128, "bf16", 8, [(127, [(140, 2), (131, 3)]), (0, [(128, 1)])]),
    ("8/1", 64, "bf16", 24, [(100, [(111, 2), (120, 1), (104, 4)])]),
    ("3/3", 128, "fp16", 1, [(40, [(50, 1), (45, 2)]), (0, [(7, 7)])]),
    ("40/1", 128, "bf16", 7, [(60, [(66, 3), (61, 1)])]),
    ("33/11", 64, "fp16", 1000, [(900, [(1500, 2), (901, 1)])]),
    ("32/8", 128, "bf16", 256, [(512, [(512 + 30, 30), (513, 1), (700, 2)]), (0, [(5, 0)]), (0, [(0, 0)])]),
    ("2/2", 128, "bf16", 16, [(2000, [(2048 + i, 1) for i in range(3)])]),
]


@pytest.mark.parametrize("order", ["nhd", "hnd", "inside"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-p{c[3]}-{len(c[4])}")
def test_against_the_oracle(ap, case, order):
    heads, dim, dtype, page, groups = case
    b = Batch(ap, heads, dim, dtype, page, groups, order, seed=len(groups) + page, pad=3)
    b.plan()
    b.check(*b.attend())
    assert ap.apack_device_error(b.ws) == 0
    first = b.attend()
    again = b.attend()
    assert all(torch.equal(x, y) for x, y in zip(first, again))                  # the same bits in every call
    b.plan(grouped=False)
    b.check(*b.attend())
    assert ap.apack_device_error(b.ws) == 0
