"""Calls at the edges of what the paged-cache entry points allow, on the GPU."""

from fractions import Fraction
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
import test_gpu_paged as base

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def workspace(n=0):
    raw = torch.zeros(max(n, 1024) + 256, dtype=torch.uint8, device="cuda")
    return raw[(-raw.data_ptr()) % 256:][:max(n, 1024)]


@pytest.mark.parametrize("lens,kept", [([40, 0, 25], [11, 0, 25]), ([300], [200]), ([5] * 1500, [3] * 1500)])
@pytest.mark.parametrize("in_place", [False, True])
def test_rows_bound_above_the_offsets(ap, lens, kept, in_place):
    """n_out above cu_dst[B], with an index that ends there: what lies behind it names no row, and is not used."""
    rng = np.random.default_rng(len(lens))
    tokens, layers, spare = 8, 2, 700
    cu_src, cu_dst = (np.concatenate([[0], np.cumsum(x)]) for x in (lens, kept))
    keep = np.concatenate([np.sort(rng.permutation(n)[:m]) + o for n, m, o in zip(lens, kept, cu_src)])
    need = [-(-n // tokens) for n in lens]
    perm, at = rng.permutation(sum(need)), 0
    table = np.full((len(lens), max(need)), -1)
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    k, v = (torch.randn(layers, sum(need), tokens, 2, 64, device="cuda").bfloat16() for _ in range(2))
    src = ap.PagedCache(k, v, i32(table))
    dst = src if in_place else ap.PagedCache(torch.zeros_like(k), torch.zeros_like(v), i32(table))
    want = [po.move_rows(a.double().cpu().numpy(), b.double().cpu().numpy(), table, table, cu_dst, keep, cu_src)
            for a, b in ((k, dst.k), (v, dst.v))]
    longer = i32(np.concatenate([keep, rng.choice([-5, 2 ** 31 - 1, -2 ** 31, 10 ** 6], spare)]))
    ws, cu_src, cu_dst = workspace(), i32(cu_src), i32(cu_dst)
    status = ap._lib.apack_paged_compact(src._address, dst._address, 0, 0, layers, longer.data_ptr(), cu_src.data_ptr(),
                                         cu_dst.data_ptr(), len(keep) + spare, ws.data_ptr(), None)
    assert status == ap.APACK_OK and ap.apack_device_error(ws) == ap.APACK_OK
    torch.cuda.synchronize()
    assert np.array_equal(dst.k.double().cpu().numpy(), want[0]) and np.array_equal(dst.v.double().cpu().numpy(), want[1])


PI = Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)


@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_of_any_frequency(ap, interleaved):
    """cos and sin of position * frequency (the pair (1, 0), fp32) against exact reductions: the angle to 2^-24 of a turn,
    sincospif to 2 ulp below 1 (2^-23), and products with 1 and 0 that are exact."""
    freq = np.array([0.3, 1.0, 3.0, 5.0, 2 * math.pi, -0.1, -1.0, -1e-12, 1e-7, 1000.0, 1e5, -12345.678, 2.0 ** 40, 0.0, 0.9, -2.9])
    pos = [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 7, 2 ** 30 + 12345, -2 ** 30 - 99, 10 ** 6, 1, 0, -1] + [2 ** 31 - 1 - 1000 * i for i in range(55)]
    pairs, n = len(freq), len(pos)
    x = torch.zeros(n, 1, 2 * pairs, device="cuda")
    lo = slice(0, None, 2) if interleaved else slice(0, pairs)
    hi = slice(1, None, 2) if interleaved else slice(pairs, None)
    x[:, :, lo] = 1
    out = torch.empty_like(x)
    ap.apack_rotary(ap.Rotary(2 * pairs, interleaved=interleaved, frequencies=freq), x, i32(pos), out)
    turns = [[float(p * Fraction(f) / (2 * PI) - math.floor(p * Fraction(f) / (2 * PI))) for f in freq.tolist()] for p in pos]
    angle = 2 * math.pi * np.array(turns)
    tol = 2 * math.pi * 2.0 ** -24 + 2.0 ** -23
    got = out.double().cpu().numpy()[:, 0]
    assert float(np.abs(got[:, lo] - np.cos(angle)).max()) <= tol
    assert float(np.abs(got[:, hi] - np.sin(angle)).max()) <= tol


@pytest.mark.parametrize("hq,hkv,h", [(251, 251, 1), (244, 244, 4), (5 * 47, 5 * 47, 5), (17 * 60, 60, 4)])
def test_work_beyond_the_list_is_reported(ap, hq, hkv, h):
    """4096 sequences over one shared page, one tile beyond 2^31 - 1025 entries by the formula of the header: nothing is
    computed but the empty sequence's zeros.  (One tile below the limit would be work of seconds.)"""
    B, tokens, tile, limit = 4096, 2048, 32, 2 ** 31 - 1025
    cost, groups = 24 // h, hkv // h
    full = B - 2                                              # sequences of as many tiles, one shorter, one empty
    tiles = (limit + cost) // groups // (full + 1) - cost
    lens = np.full(B, tiles * tile)
    lens[7] = 0
    rest = (limit + cost) // groups - full * (tiles + cost)   # entries per group left for the last sequence
    lens[-1] = (rest + 1 - cost) * tile
    total = sum(groups * (-(-int(n) // tile) + cost) for n in lens if n) - cost
    assert 0 <= limit - (total - groups) < groups and total > limit
    columns = -(-int(lens.max()) // tokens)
    k = torch.zeros(1, 1, tokens, hkv, 64, dtype=torch.bfloat16, device="cuda")
    cache = ap.PagedCache(k, k.clone(), torch.zeros(B, columns, dtype=torch.int32, device="cuda"))
    q = torch.zeros(B, hq, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.full((B, hq, 64), 3.5, dtype=torch.bfloat16, device="cuda")
    ws = workspace(ap.apack_paged_decode_workspace_size(cache, hq))
    ap.apack_paged_decode_attention(cache, 0, i32(lens), q, out, ws)
    assert ap.apack_device_error(ws) == ap.APACK_EDEVICE
    assert not out[7].any() and bool((out[:7] == 3.5).all()) and bool((out[8:] == 3.5).all())


def test_outputs_between_the_rows_that_are_read(ap):
    """Slices of one buffer that share no byte, although their ranges do: as written elsewhere."""
    torch.manual_seed(0)
    n, rot, pos = 37, ap.Rotary(64), i32(np.arange(37) * 977)
    wide = torch.randn(n, 12, 64, device="cuda").bfloat16()
    x, want = wide[:, 2:6], torch.empty(n, 4, 64, dtype=torch.bfloat16, device="cuda")
    ap.apack_rotary(rot, x, pos, want)
    for out in (wide[:, 6:10], wide[:, 8:12]):
        before = wide.clone()
        ap.apack_rotary(rot, x, pos, out)
        assert torch.equal(out, want)
        out.copy_(before[:, out.storage_offset() // 64:][:, :4])
        assert torch.equal(wide, before)
    # behind the last row read, with another stride
    flat = torch.randn(4000 + n * 64, device="cuda").bfloat16()
    x, out = flat[:13 * 300].view(13, 300)[:, :64].view(13, 1, 64), flat[13 * 300 - 236:][:13 * 64].view(13, 1, 64)
    want = torch.empty(13, 1, 64, dtype=torch.bfloat16, device="cuda")
    ap.apack_rotary(rot, x, pos[:13], want)
    ap.apack_rotary(rot, x, pos[:13], out)
    assert torch.equal(out, want)
    # the append: queries into the heads behind the values, and one token's queries in place under another stride
    k, v = (torch.zeros(1, n, 1, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = ap.PagedCache(k, v, torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1))
    zeros = torch.zeros(n, dtype=torch.int32, device="cuda")
    q_want = torch.empty(n, 4, 64, dtype=torch.bfloat16, device="cuda")
    ap.apack_rotary_append(rot, cache, 0, wide[:, :4], wide[:, 4:6], wide[:, 6:8], q_want, pos, zeros)
    k_want, v_want = k.clone(), wide[:, 6:8].clone()
    k.zero_(), v.zero_()
    ap.apack_rotary_append(rot, cache, 0, wide[:, :4], wide[:, 4:6], wide[:, 6:8], wide[:, 8:], pos, zeros)
    assert torch.equal(wide[:, 8:], q_want) and torch.equal(k, k_want) and torch.equal(v.flatten(0, 2), v_want)


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
def test_attention_output_between_query_rows(ap, out_dtype):
    """Query rows far apart, the contiguous output in a gap between them: no byte is shared, and the call is taken."""
    torch.manual_seed(1)
    k, v = (torch.randn(1, 4, 16, 2, 64, device="cuda").bfloat16() for _ in range(2))
    cache = ap.PagedCache(k, v, i32([[0, 1], [2, 3]]))
    rows = torch.randn(12, 4, 64, device="cuda").bfloat16()
    q = rows[::7][:2]                                           # rows 0 and 7
    ws = workspace(ap.apack_paged_decode_workspace_size(cache, 4))
    want = torch.empty(2, 4, 64, dtype=out_dtype, device="cuda")
    ap.apack_paged_decode_attention(cache, 0, i32([20, 31]), q, want, ws)
    size = 2 if out_dtype == torch.bfloat16 else 4
    for first in (1, 7 - size, 8):
        before = rows.clone()
        out = rows[first:first + size].view(out_dtype).reshape(-1).view(2, 4, 64)
        ap.apack_paged_decode_attention(cache, 0, i32([20, 31]), q, out, ws)
        assert torch.equal(out, want)
        rows[first:first + size] = before[first:first + size]
        assert torch.equal(rows, before)
    for first in (0, 7 - size + 1, 7):
        out = rows[first:first + size].view(out_dtype).reshape(-1).view(2, 4, 64)
        with pytest.raises(ap.ApackError) as e:
            ap.apack_paged_decode_attention(cache, 0, i32([20, 31]), q, out, ws)
        assert e.value.status == ap.APACK_EINVAL


@pytest.mark.parametrize("n", [1, 5, 700])
def test_positions_that_the_axes_share(ap, n):
    """One row of positions expanded over three axes: what three equal rows give."""
    torch.manual_seed(n)
    rot = ap.Rotary(128, sections=[16, 24, 24])
    x = torch.randn(n, 8, 128, device="cuda").bfloat16()
    pos = torch.randint(0, 2 ** 30, (n,), dtype=torch.int32, device="cuda")
    outs = []
    for p in (pos.expand(3, n).contiguous(), pos.expand(3, n), pos.view(1, n).expand(3, n)):
        out = torch.empty_like(x)
        ap.apack_rotary(rot, x, p, out)
        k, v = (torch.zeros(1, n, 1, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache = ap.PagedCache(k, v, torch.arange(n, dtype=torch.int32, device="cuda").view(1, n))
        q = torch.empty_like(x[:, :4])
        ap.apack_rotary_append(rot, cache, 0, x[:, :4], x[:, 4:6], x[:, 6:], q, p,
                               torch.arange(n, dtype=torch.int32, device="cuda"), seqs=torch.zeros(n, dtype=torch.int32, device="cuda"))
        outs.append((out, q, k, v))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))
    assert torch.equal(outs[0][0][:, :4], outs[0][1]) and torch.equal(outs[0][2].flatten(0, 2), outs[0][0][:, 4:6])


def test_scales_at_the_ends_of_fp32(ap):
    """The kernel works with scale * log2(e): what overflows there is refused, and the largest and smallest scales that do
    not give logits of any size (here 0 and ln 2: the softmax is 1/3 and 2/3)."""
    k = torch.zeros(1, 1, 16, 1, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    v[0, 0, 1] = 3
    cache = ap.PagedCache(k, v, i32([[0]]))
    ws = workspace(ap.apack_paged_decode_workspace_size(cache, 1))
    q, out = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(1, 1, 64, device="cuda")
    for scale in (3e38, 2.4e38):
        with pytest.raises(ap.ApackError) as e:
            ap.apack_paged_decode_attention(cache, 0, i32([2]), q, out, ws, scale=scale)
        assert e.value.status == ap.APACK_EINVAL
    for scale in (2.0 ** 127, 2.0 ** -100, 1.0):
        # ln 2 = scale q k for a power of two of the scale, q k a bf16 number: 0.69140625 of it
        e = -round(math.log2(scale))
        k[0, 0, 1, 0, 0] = 0.69140625 * 2.0 ** (e // 2)
        q[0, 0, 0] = 2.0 ** (e - e // 2)
        ap.apack_paged_decode_attention(cache, 0, i32([2]), q, out, ws, scale=scale)
        p = math.exp(0.69140625)
        assert abs(float(out[0, 0, 0]) - 3 * p / (1 + p)) <= 2.0 ** -19 * 3


@pytest.mark.parametrize("dim,tokens,group", [(64, 8, 2), (64, 24, 5), (128, 24, 7), (64, 40, 20), (128, 8, 32)])
def test_bad_pages_in_boxes_of_eight_tokens(ap, dim, tokens, group):
    """A page outside the pool is read as zeros, for the rows of it that the sequence has, and is reported."""
    rng = np.random.default_rng(15)
    lens = [3 * tokens - 5, tokens + 1]
    table, pages = base.make_table(rng, lens, tokens)
    k, v = (base.normal(rng, (1, pages + 1, tokens, 2, dim), torch.bfloat16) for _ in range(2))
    k[0, pages], v[0, pages] = 0, 0
    q = base.normal(rng, (2, 2 * group, dim), torch.bfloat16)

    def run(t):
        cache = ap.PagedCache(k, v, i32(t))
        ws = workspace(ap.apack_paged_decode_workspace_size(cache, 2 * group))
        out, lse = torch.empty(2, 2 * group, dim, device="cuda"), torch.empty(2, 2 * group, device="cuda")
        ap.apack_paged_decode_attention(cache, 0, i32(lens), q, out, ws, lse=lse)
        return out, lse, ap.apack_device_error(ws)

    for at in ((0, 0), (0, 1), (0, 2), (1, 1)):
        zeros = table.copy()
        zeros[at] = pages
        want, want_lse, code = run(zeros)
        assert code == ap.APACK_OK and torch.isfinite(want).all()
        for page in (-1, pages + 1, 2 ** 31 - 1, -2 ** 31):
            bad = table.copy()
            bad[at] = page
            out, lse, code = run(bad)
            assert code == ap.APACK_EDEVICE and torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens", [8, 24, 56, 104])
def test_attention_over_pages_of_eight_tokens(ap, dim, tokens):
    """Sequences that end anywhere in a box, a page or a tile, behind which NaN and infinities lie."""
    rng = np.random.default_rng(dim + tokens)
    lens = list(range(1, 42)) + [tokens * i + j for i in (1, 2, 5) for j in (-1, 0, 1)] + [0, 777]
    base.check_attention(ap, rng, lens, 12, 4, dim, tokens, "bf16", "hnd", "fp32")
    base.check_attention(ap, rng, lens[::3], 40, 2, dim, tokens, "fp16", "nhd")
