"""The paged-cache operators on the GPU against the fp64 oracle.

Tolerances (u = eps/2 of the output's type, its rounding):

rotary     |got - ref| <= u |ref| + 2^-20 m (|a| + |b|) + angle * 2^-51 m (|a| + |b|), with (a, b) the pair.  The phase
           is cut to 32 bits of a turn and rounded to fp32 (below 2^-23 of a radian), sincospif is off by 2 ulp, two
           products and a sum add 3 roundings: below 2^-20 in all; a frequency is known to 2^-52 of itself, and so is the
           oracle's angle.
attention  |got - ref| <= u |ref| + A (2^-16 + n 2^-23 + 2 d), A = sum_r p_r |v_r|: P as two 16-bit numbers (2^-17),
           exp2 (2^-22), n = 2 ceil(len / 16) + 64 sequential fp32 additions at most, and logits that are off by
           d = 2^-20 * max_r scale sum_i |q_i k_i| (8 fp32 accumulations that may truncate, the scale, log2 units).
           fp16: + len 2^-36 max |v|, the spacing of its smallest numbers against probabilities of up to 2^11 and more.
lse        |got - ref| <= 2 d + n 2^-23 + 2^-21 (1 + |ref|).
moves      bit for bit.
"""

import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def unit(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return t.detach().cpu().double().numpy()


def normal(rng, shape, dtype, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dtype).cuda()


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def workspace(n):
    raw = torch.zeros(max(n, 1024) + 256, dtype=torch.uint8, device="cuda")
    return raw[(-raw.data_ptr()) % 256:][:max(n, 1024)]


def make_pool(rng, layers, pages, tokens, heads, dim, dtype, order="nhd", scale=1.0):
    if order == "hnd":
        return normal(rng, (layers, pages, heads, tokens, dim), dtype, scale).permute(0, 1, 3, 2, 4)
    if order == "inside":                       # layers inside pages, and a gap behind every token
        p = normal(rng, (pages, layers, tokens, heads + 1, dim), dtype, scale)
        return p.transpose(0, 1)[:, :, :, :heads]
    return normal(rng, (layers, pages, tokens, heads, dim), dtype, scale)


def make_table(rng, lens, tokens, spare=3):
    need = [-(-n // tokens) for n in lens]
    pages = sum(need) + spare
    perm = rng.permutation(pages)
    table = np.full((len(lens), max(1, max(need))), -1)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, pages


# ---------------------------------------------------------------- rotary


def rotary_bound(x, freq, positions, sections, interleaved, m, ref, dtype):
    n, h, d = x.shape
    pairs = len(freq)
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = np.abs(positions[axis].T.astype(np.float64) * freq)                   # [n, pairs]
    tol = unit(dtype) * np.abs(ref) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    for i in range(pairs):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        pair = m * (np.abs(x[:, :, lo]) + np.abs(x[:, :, hi])) * (2.0 ** -20 + angle[:, i] * 2.0 ** -51)[:, None]
        tol[:, :, lo] += pair
        tol[:, :, hi] += pair
    return tol


@pytest.mark.parametrize("n,heads,dim,rdim,dtype,interleaved,sections,scaling,far", [
    (1, 1, 128, 128, "bf16", False, None, "none", 10),
    (5, 32, 128, 128, "bf16", False, [16, 24, 24], "none", 200000),
    (700, 3, 128, 64, "fp16", True, None, "yarn", 1000000),
    (611, 33, 64, 64, "bf16", False, [32, 0], "linear", 5000),
    (7, 5, 256, 256, "fp32", True, [0, 100, 28], "ntk", 2 ** 31 - 1),
    (9, 2, 80, 20, "bf16", False, None, "none", 1000),       # halves that are not whole 16-byte pieces
    (9, 3, 6, 2, "fp16", True, None, "none", 1000),
    (33, 3, 100, 100, "fp32", False, None, "none", 2 ** 31 - 1),
    (620, 7, 128, 32, "fp32", False, None, "none", 99999),
    (3, 70, 256, 2, "bf16", False, None, "none", 70),
])
@pytest.mark.parametrize("transpose", [False, True])
def test_rotary(ap, n, heads, dim, rdim, dtype, interleaved, sections, scaling, far, transpose):
    rng = np.random.default_rng(n + heads + dim)
    dt = DT[dtype]
    rot = ap.Rotary(rdim, base=1e6, interleaved=interleaved, scaling=scaling, factor=4.0 if scaling != "none" else 1.0,
                    original_len=4096, sections=sections)
    sec = [rdim // 2] if sections is None else sections
    wide = normal(rng, (n, heads + 2, dim), dt)
    x = wide[:, 1:heads + 1]                                                  # rows with a gap, start inside one
    pos = rng.integers(-far, far, (len(sec), n))
    pos[:, 0] = far
    pos_d = i32(pos) if len(sec) > 1 else i32(pos[0])
    out = torch.full((n, heads, dim), math.nan, dtype=dt, device="cuda")
    before = wide.clone()
    ap.apack_rotary(rot, x, pos_d, out, transpose=transpose)
    ref = po.rotary(f64(x), pos, rot.frequencies, sec, interleaved, rot.magnitude, transpose)
    tol = rotary_bound(f64(x), rot.frequencies, pos, sec, interleaved, rot.magnitude, ref, dt)
    assert np.all(np.abs(f64(out) - ref) <= tol)
    assert torch.equal(out[..., rdim:], x[..., rdim:])
    ap.apack_rotary(rot, x, pos_d, x, transpose=transpose)                 # in place
    assert torch.equal(x, out) and torch.equal(wide[:, 0], before[:, 0]) and torch.equal(wide[:, -1], before[:, -1])


def test_rotary_gradient_by_differences(ap):
    """The transposed map against central differences of the forward map, in fp32."""
    rng = np.random.default_rng(3)
    rot = ap.Rotary(32, base=100.0, interleaved=True, magnitude=1.25)
    x, w = normal(rng, (2, 3, 48), torch.float32), normal(rng, (2, 3, 48), torch.float32)
    pos = i32([5, 90])
    grad, y = torch.empty_like(x), torch.empty_like(x)
    ap.apack_rotary(rot, w, pos, grad, transpose=True)

    def loss(z):
        ap.apack_rotary(rot, z, pos, y)
        return float((y.double() * w.double()).sum())

    for t, h, i in [(0, 0, 0), (1, 2, 31), (0, 1, 7), (1, 0, 32), (1, 1, 47)]:
        e = torch.zeros_like(x)
        e[t, h, i] = 1.0                        # the map is linear: any step is exact but for fp32 rounding
        diff = (loss(x + e) - loss(x - e)) / 2
        # 288 products of magnitudes below 5 * 1.25 * 5, each off by 2^-20 of itself
        assert abs(diff - float(grad[t, h, i])) <= 288 * 32 * 2.0 ** -20


# ---------------------------------------------------------------- rotary and the write into pages


@pytest.mark.parametrize("prompt", [False, True])
@pytest.mark.parametrize("heads,dim,rdim,dtype,tokens,order,interleaved,sections", [
    ((28, 4), 128, 128, "bf16", 16, "nhd", False, [16, 24, 24]),
    ((8, 8), 64, 32, "fp16", 5, "hnd", True, None),
    ((5, 1), 128, 36, "bf16", 1, "inside", False, None),         # narrow accesses
    ((0, 3), 64, 64, "bf16", 48, "inside", False, [20, 12]),     # keys and values alone
    ((6, 2), 128, 0, "fp16", 7, "nhd", False, None),              # no rotation
])
def test_rotary_append(ap, prompt, heads, dim, rdim, dtype, tokens, order, interleaved, sections):
    hq, hkv = heads
    rng = np.random.default_rng(dim + tokens + hq)
    dt = DT[dtype]
    if prompt:                                   # three sequences' tokens in one call, in any order
        lens = [0, 700, 33]
        seqs = np.concatenate([np.full(m, b) for b, m in enumerate(lens)])
        rows = np.concatenate([np.arange(m) for m in lens])
        order_ = rng.permutation(len(seqs))
        seqs, rows = seqs[order_], rows[order_]
        skip = rng.random(len(rows)) < 0.1
        rows[skip] = -1
    else:
        lens = [1, 40, 17, 3, 90]
        seqs, rows = None, np.array([0, 39, -5, 2, 89])
    n = len(rows)
    table, pages = make_table(rng, lens, tokens)
    layers, layer = 3, 1
    kp, vp = (make_pool(rng, layers, pages, tokens, hkv, dim, dt, order) for _ in range(2))
    cache = ap.PagedCache(kp, vp, i32(table))
    qkv = normal(rng, (n, hq + 2 * hkv, dim), dt)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    rot = None if rdim == 0 else ap.Rotary(rdim, base=1e4, interleaved=interleaved, sections=sections)
    sec = sections or [rdim // 2]
    pos = rng.integers(0, 300000, (len(sec), n))
    k0, v0 = kp.clone(), vp.clone()
    q_out = torch.full((n, hq, dim), math.nan, dtype=dt, device="cuda") if hq else None
    ws = workspace(0)
    ap.apack_rotary_append(rot, cache, layer, q if hq else None, k, v, q_out, i32(pos) if sections else i32(pos[0]),
                           i32(rows), seqs=None if seqs is None else i32(seqs), ws=ws)
    assert ap.apack_device_error(ws) == ap.APACK_OK
    for x, got in ((q, q_out), (k, None)):
        if x.shape[1] == 0:
            continue
        if rot is None:
            ref, tol = f64(x), np.zeros(x.shape)
        else:
            ref = po.rotary(f64(x), pos, rot.frequencies, sec, interleaved)
            tol = rotary_bound(f64(x), rot.frequencies, pos, sec, interleaved, 1.0, ref, dt)
        if got is not None:
            assert np.all(np.abs(f64(got) - ref) <= tol)
    k_now, v_now, v_in = f64(kp), f64(vp), f64(v)
    k_want, v_want, allowed = f64(k0), f64(v0), np.zeros(tuple(kp.shape))
    for t in range(n):
        if rows[t] >= 0:
            b = t if seqs is None else seqs[t]
            p, s = table[b, rows[t] // tokens], rows[t] % tokens
            k_want[layer, p, s], v_want[layer, p, s], allowed[layer, p, s] = ref[t], v_in[t], tol[t]
    assert np.all(np.abs(k_now - k_want) <= allowed)             # the rows of the call, and no other
    assert np.array_equal(v_now, v_want)
    if hq:                                                        # queries in place
        ap.apack_rotary_append(rot, cache, layer, q, k, v, q, i32(pos) if sections else i32(pos[0]), i32(rows),
                               seqs=None if seqs is None else i32(seqs))
        assert torch.equal(q, q_out)


def test_append_reports_rows_and_pages_outside(ap):
    rng = np.random.default_rng(4)
    kp, vp = (make_pool(rng, 1, 4, 8, 2, 64, torch.bfloat16) for _ in range(2))
    cache = ap.PagedCache(kp, vp, i32([[0, 1], [2, 9], [-1, 3]]))
    k0, v0 = kp.clone(), vp.clone()
    kv = normal(rng, (1, 2, 64), torch.bfloat16)
    ws = workspace(0)
    for seq, row in ((0, 16), (0, 2 ** 31 - 1), (1, 8), (2, 0), (3, 0), (-1, 0)):
        ap.apack_rotary_append(None, cache, 0, None, kv, kv, None, None, i32([row]), seqs=i32([seq]), ws=ws)
        assert ap.apack_device_error(ws) == ap.APACK_EDEVICE, (seq, row)
        ap.apack_rotary_append(None, cache, 0, None, kv, kv, None, None, i32([row]), seqs=i32([seq]))
    torch.cuda.synchronize()
    assert torch.equal(kp, k0) and torch.equal(vp, v0)


# ---------------------------------------------------------------- attention


def check_attention(ap, rng, lens, hq, hkv, dim, tokens, dtype, order="nhd", out_dtype=None, scale=None, k_scale=1.5,
                    poison=True, layers=1, layer=0):
    dt = DT[dtype]
    table, pages = make_table(rng, lens, tokens)
    kp, vp = (make_pool(rng, layers, pages, tokens, hkv, dim, dt, order, s) for s in (k_scale, 1.0))
    if poison:                                    # what lies behind the last row must not be seen
        bad = torch.tensor([math.nan, math.inf, -math.inf], dtype=dt, device="cuda")
        used = np.zeros((pages, tokens), bool)
        for b, n in enumerate(lens):
            for r in range(n):
                used[table[b, r // tokens], r % tokens] = True
        free = torch.from_numpy(~used).cuda()
        for pool in (kp, vp):
            rows = pool[layer][free]
            pool[layer][free] = bad[torch.arange(rows.numel(), device="cuda").view(rows.shape) % 3]
    q = normal(rng, (len(lens), hq + 3, dim), dt)[:, 2:hq + 2]
    out = torch.full((len(lens), hq, dim), math.nan, dtype=DT[out_dtype or dtype], device="cuda")
    lse = torch.full((len(lens), hq), math.nan, device="cuda")
    cache = ap.PagedCache(kp, vp, i32(table))
    ws = workspace(ap.apack_paged_decode_workspace_size(cache, hq))
    ap.apack_paged_decode_attention(cache, layer, i32(lens), q, out, ws, scale=scale, lse=lse)
    assert ap.apack_device_error(ws) == ap.APACK_OK
    s = 1 / math.sqrt(dim) if scale is None else scale
    ref, ref_lse, spread, size = po.paged_decode(f64(q), f64(kp[layer]), f64(vp[layer]), table, lens, s)
    d = 2.0 ** -20 * size
    n = (2 * -(-np.array(lens) // 16) + 64)[:, None]
    tol = unit(out.dtype) * np.abs(ref) + spread * (2.0 ** -16 + n * 2.0 ** -23 + 2 * d)[..., None]
    if dt == torch.float16:
        tol += np.array(lens)[:, None, None] * 2.0 ** -36 * 6
    if out.dtype == torch.float16:
        tol += 2.0 ** -25
    assert np.all(np.abs(f64(out) - ref) <= tol), float((np.abs(f64(out) - ref) / (tol + 1e-300)).max())
    got = f64(lse)
    empty = np.array(lens) == 0
    assert np.all(got[empty] == -np.inf) and np.all(f64(out)[empty] == 0)
    err = np.abs(got[~empty] - ref_lse[~empty])
    assert np.all(err <= (2 * d + n * 2.0 ** -23 + 2.0 ** -21 * (1 + np.abs(ref_lse)))[~empty])
    again, lse2 = torch.empty_like(out), torch.empty_like(lse)
    ap.apack_paged_decode_attention(cache, layer, i32(lens), q, again, ws, scale=scale, lse=lse2)
    assert torch.equal(again, out) and torch.equal(lse2, lse)               # the same bits again
    ap.apack_paged_decode_attention(cache, layer, i32(lens), q, again, ws, scale=scale)
    assert torch.equal(again, out)


@pytest.mark.parametrize("lens,hq,hkv,dim,tokens,dtype,order,out_dtype", [
    ([1], 28, 4, 128, 16, "bf16", "nhd", None),
    ([0], 4, 4, 64, 16, "bf16", "nhd", None),
    ([15, 16, 17, 31, 33], 28, 4, 128, 16, "bf16", "nhd", "fp32"),
    ([7, 64, 65, 1000, 0, 4099], 28, 4, 128, 64, "bf16", "nhd", None),
    ([5000, 333], 16, 2, 128, 16, "fp16", "hnd", "fp32"),
    ([2000], 8, 8, 64, 32, "fp16", "hnd", None),
    ([3000, 2], 8, 1, 128, 128, "bf16", "nhd", "fp32"),
    ([1500, 1, 0, 77], 32, 1, 128, 16, "bf16", "nhd", None),     # 32 query rows of one KV head
    ([900, 40], 30, 3, 64, 16, "fp16", "inside", "fp32"),        # ten of each of three
    ([500, 16], 5, 5, 128, 16, "bf16", "inside", None),
    ([100, 2000, 60], 48, 24, 64, 16, "bf16", "nhd", None),       # three groups of KV heads
    ([300, 299], 40, 10, 128, 16, "fp16", "hnd", None),
    ([301, 12], 64, 8, 128, 24, "bf16", "nhd", None),             # page sizes of every kind
    ([37, 45, 200], 28, 4, 128, 1, "bf16", "nhd", "fp32"),
    ([37, 45, 200], 12, 4, 64, 7, "fp16", "hnd", None),
    ([100, 3, 250], 16, 2, 128, 4, "bf16", "inside", None),
    ([130, 8, 90], 22, 2, 128, 40, "bf16", "nhd", "fp32"),
    ([257], 17, 1, 64, 1000, "fp16", "nhd", None),
    ([100, 47, 33, 16], 12, 4, 64, 48, "fp16", "nhd", None),
    ([1000, 18], 32, 1, 64, 16, "bf16", "hnd", None),
    ([700, 45, 3000], 64, 4, 128, 16, "bf16", "nhd", None),
    ([333, 1, 90], 96, 4, 64, 8, "fp16", "nhd", "fp32"),
])
def test_paged_attention(ap, lens, hq, hkv, dim, tokens, dtype, order, out_dtype):
    rng = np.random.default_rng(sum(lens) + hq + tokens)
    check_attention(ap, rng, lens, hq, hkv, dim, tokens, dtype, order, out_dtype, layers=2, layer=1)


@pytest.mark.parametrize("group", [1, 3, 9])
@pytest.mark.parametrize("hkv", [1, 3, 5, 6, 7, 9, 12, 24])
def test_paged_attention_head_counts(ap, hkv, group):
    """Head counts that are no powers of two share a CTA's warps in other ways: what the warps of a head hold is summed
    among them, whichever warps they are."""
    rng = np.random.default_rng(100 * hkv + group)
    check_attention(ap, rng, [5, 130, 0, 47, 700], group * hkv, hkv, 128, 16, "bf16", out_dtype="fp32")
    check_attention(ap, rng, [60] * 20, group * hkv, hkv, 64, 5, "fp16")


def test_paged_attention_of_many_sequences(ap):
    rng = np.random.default_rng(8)
    lens = [int(x) for x in rng.integers(0, 60, 300)]
    lens[5], lens[130], lens[299] = 2000, 0, 700
    check_attention(ap, rng, lens, 4, 2, 64, 16, "bf16")
    check_attention(ap, rng, [1] * 700, 2, 2, 64, 16, "fp16")
    check_attention(ap, rng, [int(x) for x in rng.integers(0, 4, 4095)] + [900], 1, 1, 64, 16, "fp16")
    check_attention(ap, rng, [0] * 64 + [1, 0, 40], 12, 12, 64, 16, "bf16")


@pytest.mark.parametrize("k_scale,scale", [(8.0, None), (30.0, None), (0.0, None), (1.5, 1e-3), (1.5, 1.0)])
def test_paged_attention_logits_of_any_size(ap, k_scale, scale):
    rng = np.random.default_rng(9)
    check_attention(ap, rng, [700, 33], 28, 4, 128, 16, "bf16", scale=scale, k_scale=k_scale, out_dtype="fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_paged_attention_long_tail(ap, dtype):
    """One key takes nearly all of the weight and has the value 0; what comes out is the tail, each of its keys about
    2^-25 of the largest."""
    n, dim, dt = 30000, 64, DT[dtype]
    pages = -(-n // 16)
    k = torch.zeros(1, pages, 16, 1, dim, dtype=dt, device="cuda")
    v = torch.ones_like(k)
    for at in (0, 16111, n - 1):                       # seen first, in the middle, last
        kk, vv = k.clone(), v.clone()
        kk.view(-1, dim)[at, 0] = 17.25
        vv.view(-1, dim)[at] = 0
        vv.view(-1, dim)[n:] = math.nan
        q = torch.zeros(1, 3, dim, dtype=dt, device="cuda")
        q[0, :, 0] = 1.0
        cache = ap.PagedCache(kk, vv, i32([list(range(pages))]))
        out, lse = torch.empty(1, 3, dim, device="cuda"), torch.empty(1, 3, device="cuda")
        ws = workspace(ap.apack_paged_decode_workspace_size(cache, 3))
        ap.apack_paged_decode_attention(cache, 0, i32([n]), q, out, ws, scale=1.0, lse=lse)
        w = (n - 1) * math.exp(-17.25)
        want = w / (1 + w)
        tol = want * (2.0 ** -16 + (2 * pages + 64) * 2.0 ** -23 + 2 * 2.0 ** -20 * 17.25)
        if dtype == "fp16":
            tol += n * 2.0 ** -36
        assert float((out.double() - want).abs().max()) <= tol
        assert float((lse.double() - 17.25 - math.log1p(w)).abs().max()) <= 2 * 2.0 ** -20 * 17.25 + (2 * pages + 64) * 2.0 ** -23 + 2.0 ** -16


def test_paged_attention_reference_that_grows(ap):
    """Keys in rising order of their logit: every tile raises the maximum, and its step is above the threshold or
    below it; and in falling order."""
    rng = np.random.default_rng(10)
    for step in (0.01, 0.3, 3.0):
        for sign in (1, -1):
            n, dim = 900, 64
            q = torch.zeros(1, 2, dim, dtype=torch.float16, device="cuda")
            q[0, :, 0] = 1.0
            k = normal(rng, (1, 57, 16, 1, dim), torch.float16, 0.1)
            k.view(-1, dim)[:n, 0] = (torch.arange(n, device="cuda") * step * sign).half()
            v = normal(rng, (1, 57, 16, 1, dim), torch.float16)
            cache = ap.PagedCache(k, v, i32([list(range(57))]))
            out = torch.empty(1, 2, dim, device="cuda")
            ws = workspace(ap.apack_paged_decode_workspace_size(cache, 2))
            ap.apack_paged_decode_attention(cache, 0, i32([n]), q, out, ws, scale=1.0)
            ref, _, spread, size = po.paged_decode(f64(q), f64(k[0]), f64(v[0]), np.arange(57)[None], [n], 1.0)
            tol = spread * (2.0 ** -16 + (2 * 57 + 64) * 2.0 ** -23 + 2.0 ** -19 * size)[..., None]
            assert np.all(np.abs(f64(out) - ref) <= tol)


def test_paged_attention_nan_and_infinite_rows_of_the_sequence(ap):
    """What a sequence does attend to is not hidden: a NaN or an infinity among its values or keys reaches the heads
    that read it, and no other.  An infinite value may come out as a NaN: a probability is the sum of two 16-bit
    numbers, of which the second may be 0 or negative, and infinity + (0 or -x) * infinity is NaN."""
    rng = np.random.default_rng(11)
    k, v = (normal(rng, (1, 3, 16, 2, 64), torch.bfloat16) for _ in range(2))
    k[0, 1, 3, 0, 5] = math.nan
    v[0, 2, 1, 1, 7] = math.inf
    q = normal(rng, (1, 4, 64), torch.bfloat16)
    cache = ap.PagedCache(k, v, i32([[0, 1, 2]]))
    out, lse = torch.empty(1, 4, 64, device="cuda"), torch.empty(1, 4, device="cuda")
    ws = workspace(ap.apack_paged_decode_workspace_size(cache, 4))
    ap.apack_paged_decode_attention(cache, 0, i32([48]), q, out, ws, lse=lse)
    assert torch.isnan(out[0, :2]).all() and torch.isnan(lse[0, :2]).all()
    assert not torch.isfinite(out[0, 2:, 7]).any() and torch.isfinite(lse[0, 2:]).all()
    assert torch.isfinite(out[0, 2:, :7]).all() and torch.isfinite(out[0, 2:, 8:]).all()


def test_paged_attention_bad_lengths_and_pages(ap):
    """Lengths outside the table are read as the nearest, pages outside the pool as zeros; both are reported."""
    rng = np.random.default_rng(12)
    k, v = (normal(rng, (1, 4, 16, 2, 64), torch.bfloat16) for _ in range(2))
    q = normal(rng, (2, 4, 64), torch.bfloat16)
    cache = ap.PagedCache(k, v, i32([[0, 1], [2, 3]]))
    ws = workspace(ap.apack_paged_decode_workspace_size(cache, 4))

    def run(lens, c=cache):
        out = torch.empty(2, 4, 64, device="cuda")
        ap.apack_paged_decode_attention(c, 0, i32(lens), q, out, ws)
        return out, ap.apack_device_error(ws)

    good, code = run([32, 0])
    assert code == ap.APACK_OK
    for lens in ([33, 0], [2 ** 31 - 1, 0], [32, -1], [32, -2 ** 31]):
        out, code = run(lens)
        assert code == ap.APACK_EDEVICE and torch.equal(out, good)
    kz, vz = k.clone(), v.clone()
    kz[0, 1], vz[0, 1] = 0, 0
    want, _ = run([20, 5], ap.PagedCache(kz, vz, cache.page_table))
    for page in (-1, 4, 2 ** 31 - 1, -2 ** 31):
        out, code = run([20, 5], ap.PagedCache(k, v, i32([[0, page], [2, 3]])))
        assert code == ap.APACK_EDEVICE and torch.equal(out, want)
    assert run([32, 0])[1] == ap.APACK_OK


@pytest.mark.parametrize("dim,tokens,group", [(128, 1, 2), (64, 5, 2), (128, 8, 12), (64, 2, 20)])
def test_paged_attention_bad_pages_of_few_tokens(ap, dim, tokens, group):
    """A page outside the pool is a page of zeros here too, for the rows of it that the sequence has, and is reported."""
    rng = np.random.default_rng(15)
    lens = [43, 17]
    table, pages = make_table(rng, lens, tokens)
    k, v = (normal(rng, (1, pages + 1, tokens, 2, dim), torch.bfloat16) for _ in range(2))
    k[0, pages], v[0, pages] = 0, 0
    q = normal(rng, (2, 2 * group, dim), torch.bfloat16)

    def run(t):
        cache = ap.PagedCache(k, v, i32(t))
        ws = workspace(ap.apack_paged_decode_workspace_size(cache, 2 * group))
        out, lse = torch.empty(2, 2 * group, dim, device="cuda"), torch.empty(2, 2 * group, device="cuda")
        ap.apack_paged_decode_attention(cache, 0, i32(lens), q, out, ws, lse=lse)
        return out, lse, ap.apack_device_error(ws)

    for at in ((0, 0), (0, 42 // tokens), (1, 1)):
        zeros = table.copy()
        zeros[at] = pages
        want, want_lse, code = run(zeros)
        assert code == ap.APACK_OK and torch.isfinite(want).all()
        for page in (-1, pages + 1, 2 ** 31 - 1, -2 ** 31):
            bad = table.copy()
            bad[at] = page
            out, lse, code = run(bad)
            assert code == ap.APACK_EDEVICE and torch.equal(out, want) and torch.equal(lse, want_lse)


def test_paged_attention_refuses_an_output_over_its_queries(ap):
    rng = np.random.default_rng(14)
    k, v = (normal(rng, (1, 3, 16, 2, 64), torch.bfloat16) for _ in range(2))
    both = normal(rng, (5, 4, 64), torch.bfloat16)
    cache = ap.PagedCache(k, v, i32([[0, 1], [2, 2]]))
    ws = workspace(ap.apack_paged_decode_workspace_size(cache, 4))
    for q, out in ((both[:2], both[:2]), (both[:2], both[1:3]), (both[1:3], both[:2]), (both[::2][:2], both[1:3])):
        with pytest.raises(ap.ApackError) as e:
            ap.apack_paged_decode_attention(cache, 0, i32([20, 3]), q, out, ws)
        assert e.value.status == ap.APACK_EINVAL
    want, q = torch.empty(2, 4, 64, device="cuda").bfloat16(), both[:2].clone()
    ap.apack_paged_decode_attention(cache, 0, i32([20, 3]), q, want, ws)
    for out in (both[2:4], both[3:5]):                  # beside them
        ap.apack_paged_decode_attention(cache, 0, i32([20, 3]), both[:2], out, ws)
        assert torch.equal(out, want)


def test_paged_attention_agrees_with_the_contiguous_call(ap):
    """One page that holds the whole packed cache of a sequence: the numbers of apack_decode_attention."""
    rng = np.random.default_rng(13)
    n = 4644
    k, v = (normal(rng, (1, 1, n, 4, 128), torch.bfloat16) for _ in range(2))
    q = normal(rng, (1, 28, 128), torch.bfloat16)
    cu = np.array([0, n], np.int32)
    a, b = torch.empty(1, 28, 128, device="cuda"), torch.empty(1, 28, 128, device="cuda")
    ws = workspace(ap.apack_decode_workspace_size(cu, 28, 4))
    ap.apack_decode_attention(cu, q, k, v, 1024, 28, 4, a, ws)
    cache = ap.PagedCache(k, v, i32([[0]]))
    ws2 = workspace(ap.apack_paged_decode_workspace_size(cache, 28))
    ap.apack_paged_decode_attention(cache, 0, i32([n]), q, b, ws2)
    # both are within 2^-16 + n 2^-23 + ... of the same sums of values below 5: far inside 1e-3
    assert float((a - b).abs().max()) < 1e-3


# ---------------------------------------------------------------- moves


def planes(pool, l0, n):
    return f64(pool[l0:l0 + n].float())


@pytest.mark.parametrize("lens,heads,dim,dtype,src,dst", [
    ([900], 4, 128, "bf16", ("slab", 0), ("nhd", 16)),
    ([300, 0, 77, 1000], 2, 128, "bf16", ("nhd", 16), ("nhd", 64)),
    ([300, 1, 77], 8, 64, "fp16", ("hnd", 5), ("inside", 16)),
    ([64, 65], 3, 64, "fp16", ("inside", 32), ("hnd", 1)),
    ([10, 20], 1, 64, "bf16", ("nhd", 7), ("nhd", 7)),
])
@pytest.mark.parametrize("indexed", [True, False])
def test_paged_compact(ap, lens, heads, dim, dtype, src, dst, indexed):
    rng = np.random.default_rng(sum(lens) + heads)
    dt = DT[dtype]
    B = len(lens)
    kept = [int(rng.integers(0, n + 1)) for n in lens]
    kept[0] = max(1, kept[0])
    cu_src, cu_dst = (np.concatenate([[0], np.cumsum(x)]) for x in (lens, kept))
    keep = np.concatenate([np.sort(rng.permutation(n)[:m]) + cu_src[b] for b, (n, m) in enumerate(zip(lens, kept))])
    if src[0] == "slab":
        ks, vs = (normal(rng, (3, 1, sum(lens), heads, dim), dt) for _ in range(2))
        table = np.zeros((B, 1), int)
    else:
        table, pages = make_table(rng, lens, src[1])
        ks, vs = (make_pool(rng, 3, pages, src[1], heads, dim, dt, src[0]) for _ in range(2))
    to, pages = make_table(rng, kept, dst[1])
    kd, vd = (make_pool(rng, 4, pages, dst[1], heads, dim, dt, dst[0]) for _ in range(2))
    a, b = ap.PagedCache(ks, vs, i32(table)), ap.PagedCache(kd, vd, i32(to))
    k0, v0 = kd.clone(), vd.clone()
    ws = workspace(0)
    packed = src[0] == "slab"
    ap.apack_paged_compact(a, b, i32(cu_dst), int(cu_dst[-1]) + (0 if indexed else 40),
                           keep_idx=i32(keep) if indexed else None,
                           cu_src=i32(cu_src) if indexed and not packed else None, src_layer=1, dst_layer=2, num_layers=2, ws=ws)
    assert ap.apack_device_error(ws) == ap.APACK_OK
    for s, d, d0 in ((ks, kd, k0), (vs, vd, v0)):
        want = po.move_rows(planes(s, 1, 2), planes(d0, 2, 2), table, to, cu_dst, keep if indexed else None,
                            cu_src if indexed and not packed else None)
        assert np.array_equal(planes(d, 2, 2), want) and torch.equal(d[:2], d0[:2])


@pytest.mark.parametrize("lens,heads,dim,tokens,order", [
    ([1000], 4, 128, 16, "nhd"), ([300, 0, 77, 1000, 5], 2, 64, 5, "hnd"), ([130, 64], 3, 128, 32, "inside"),
    ([2500, 31, 33], 1, 64, 1, "nhd"),
])
@pytest.mark.parametrize("ratio", [0.02, 0.5, 0.97, 1.0])
def test_paged_compact_in_place(ap, lens, heads, dim, tokens, order, ratio):
    check_in_place(ap, lens, heads, dim, tokens, order, ratio)


def test_paged_compact_in_place_of_batches(ap):
    """Batches large enough for 64 and 128 bytes of a row per warp, sequences of several steps."""
    check_in_place(ap, [400, 270] * 20, 4, 128, 16, "nhd", 0.9)
    check_in_place(ap, [300, 1000] * 10, 4, 128, 16, "nhd", 0.6)
    check_in_place(ap, [500] * 22, 5, 64, 7, "hnd", 0.95)


def check_in_place(ap, lens, heads, dim, tokens, order, ratio):
    rng = np.random.default_rng(sum(lens) + heads)
    kept = [int(round(n * ratio)) for n in lens]
    cu_src, cu_dst = (np.concatenate([[0], np.cumsum(x)]) for x in (lens, kept))
    keep = np.concatenate([np.sort(rng.permutation(n)[:m]) + cu_src[b] for b, (n, m) in enumerate(zip(lens, kept))])
    table, pages = make_table(rng, lens, tokens)
    k, v = (make_pool(rng, 3, pages, tokens, heads, dim, torch.bfloat16, order) for _ in range(2))
    k0, v0 = k.clone(), v.clone()
    cache = ap.PagedCache(k, v, i32(table))
    ws = workspace(0)
    ap.apack_paged_compact(cache, cache, i32(cu_dst), int(cu_dst[-1]), keep_idx=i32(keep), cu_src=i32(cu_src),
                           src_layer=1, dst_layer=1, ws=ws)
    assert ap.apack_device_error(ws) == ap.APACK_OK
    for pool, before in ((k, k0), (v, v0)):
        want = po.move_rows(planes(before, 1, 2), planes(before, 1, 2), table, table, cu_dst, keep, cu_src)
        assert np.array_equal(planes(pool, 1, 2), want) and torch.equal(pool[0], before[0])


def test_moves_report_rows_and_pages_outside(ap):
    rng = np.random.default_rng(14)
    k, v = (normal(rng, (2, 6, 4, 2, 64), torch.bfloat16) for _ in range(2))
    ws = workspace(0)

    def compact(src_table, dst_table, keep, cu):
        kd, vd = torch.zeros_like(k), torch.zeros_like(v)
        a, b = ap.PagedCache(k, v, i32(src_table)), ap.PagedCache(kd, vd, i32(dst_table))
        ap.apack_paged_compact(a, b, i32(cu), len(keep), keep_idx=i32(keep), ws=ws)
        return kd, ap.apack_device_error(ws)

    kd, code = compact([[0, 1]], [[2, 3]], [0, 7], [0, 2])
    assert code == ap.APACK_OK and torch.equal(kd[:, 2, 1], k[:, 1, 3])
    for args in (([[0, 6]], [[2, 3]], [0, 7], [0, 2]), ([[0, -1]], [[2, 3]], [0, 7], [0, 2]),
                 ([[0, 1]], [[2, 3]], [0, 8], [0, 2]), ([[0, 1]], [[2, 3]], [0, -1], [0, 2])):
        kd, code = compact(*args)                       # row 0 is copied, the other is not
        assert code == ap.APACK_EDEVICE and torch.equal(kd[:, 2, 0], k[:, 0, 0]) and float(kd[:, 2, 1:].abs().sum()) == 0
    kd, code = compact([[0, 1]], [[2, 3]], list(range(8)) + [0], [0, 9])     # one row more than the table holds
    assert code == ap.APACK_EDEVICE and torch.equal(kd[:, 2:4], k[:, :2])
    cache = ap.PagedCache(k, v, i32([[0]]))
    k0 = k.clone()
    ap.apack_copy_pages(cache, i32([[0, 5], [6, 1], [2, -1]]), ws=ws)
    assert ap.apack_device_error(ws) == ap.APACK_EDEVICE
    k0[:, 5] = k0[:, 0]
    assert torch.equal(k, k0)


@pytest.mark.parametrize("layers,pages,tokens,heads,dim,order,n", [
    (28, 9, 16, 4, 128, "nhd", 1), (3, 200, 16, 2, 64, "hnd", 90), (2, 50, 5, 3, 64, "inside", 20), (1, 9, 1000, 1, 128, "nhd", 4),
])
def test_copy_pages(ap, layers, pages, tokens, heads, dim, order, n):
    rng = np.random.default_rng(pages)
    k, v = (make_pool(rng, layers, pages, tokens, heads, dim, torch.float16, order) for _ in range(2))
    pairs = rng.permutation(pages)[:2 * n].reshape(n, 2)
    if n > 3:
        pairs[3, 1] = pairs[3, 0]                       # a page with itself
    k0, v0 = k.clone(), v.clone()
    cache = ap.PagedCache(k, v, i32([[0]]))
    ap.apack_copy_pages(cache, i32(pairs))
    for pool, before in ((k, k0), (v, v0)):
        before[:, pairs[:, 1]] = before[:, pairs[:, 0]]
        assert torch.equal(pool, before)


# ---------------------------------------------------------------- streams, graphs, sizes


def test_pool_above_32_bit_offsets(ap):
    """Pages whose byte offsets pass 2^32: every operator at the far end of a pool of 5 GiB per tensor."""
    rng = np.random.default_rng(15)
    pages, tokens = 330000, 16
    k = torch.zeros(1, pages, tokens, 4, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    lens = [50]
    table = np.array([[pages - 1, 7, pages - 2, pages - 5]])
    cache = ap.PagedCache(k, v, i32(table))
    kv = normal(rng, (50, 8, 128), torch.bfloat16)
    ap.apack_rotary_append(None, cache, 0, None, kv[:, :4], kv[:, 4:], None, None, i32(np.arange(50)), seqs=i32(np.zeros(50)))
    q = normal(rng, (1, 28, 128), torch.bfloat16)
    out = torch.empty(1, 28, 128, device="cuda")
    ws = workspace(ap.apack_paged_decode_workspace_size(cache, 28))
    ap.apack_paged_decode_attention(cache, 0, i32(lens), q, out, ws)
    assert ap.apack_device_error(ws) == ap.APACK_OK
    small_k, small_v = (normal(rng, (1, 4, tokens, 4, 128), torch.bfloat16) for _ in range(2))
    small = ap.PagedCache(small_k, small_v, i32([[0, 1, 2, 3]]))
    ap.apack_paged_compact(cache, small, i32([0, 50]), 50)
    assert torch.equal(small_k[0].flatten(0, 1)[:50], kv[:, :4]) and torch.equal(small_v[0].flatten(0, 1)[:50], kv[:, 4:])
    want = torch.empty_like(out)
    ap.apack_paged_decode_attention(small, 0, i32(lens), q, want, ws)
    assert torch.equal(out, want)
    ap.apack_copy_pages(cache, i32([[pages - 1, pages - 3]]))
    assert torch.equal(k[0, pages - 3], k[0, pages - 1]) and float(k[0, pages - 4].abs().sum()) == 0


def test_decode_loop_captured_and_replayed(ap):
    """A decode step (rotary and append, then attention, then the lengths) captured once and replayed: the caches
    grow page by page, as eager calls make them."""
    rng = np.random.default_rng(16)
    hq, hkv, dim, tokens, layers, B = 28, 4, 128, 16, 2, 3
    lens0, steps = [14, 0, 200], 5
    table, pages = make_table(rng, [n + steps for n in lens0], tokens)
    k0, v0 = (make_pool(rng, layers, pages, tokens, hkv, dim, torch.bfloat16) for _ in range(2))
    new = normal(rng, (steps, layers, B, hq + 2 * hkv, dim), torch.bfloat16)
    pos = rng.integers(0, 100000, (steps, 3, B))
    rot = ap.Rotary(dim, base=1e6, sections=[16, 24, 24])

    class Run:
        def __init__(self):
            self.k, self.v = k0.clone(), v0.clone()
            self.cache = ap.PagedCache(self.k, self.v, i32(table))
            self.rows, self.lens = i32(lens0), i32(lens0) + 1
            self.qkv, self.pos = torch.empty_like(new[0]), i32(pos[0])
            self.q = torch.empty(layers, B, hq, dim, dtype=torch.bfloat16, device="cuda")
            self.out = torch.empty_like(self.q)
            self.ws = workspace(ap.apack_paged_decode_workspace_size(self.cache, hq))

        def step(self):
            for i in range(layers):
                x = self.qkv[i]
                ap.apack_rotary_append(rot, self.cache, i, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], self.q[i],
                                       self.pos, self.rows, ws=self.ws)
                ap.apack_paged_decode_attention(self.cache, i, self.lens, self.q[i], self.out[i], self.ws)
            self.rows += 1
            self.lens += 1

    a, b = Run(), Run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        b.qkv.copy_(new[0])
        b.step()                                            # warm-up; then the state is put back
        b.k.copy_(k0), b.v.copy_(v0), b.rows.copy_(i32(lens0)), b.lens.copy_(i32(lens0) + 1)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            b.step()
    for t in range(steps):
        for r in (a, b):
            r.qkv.copy_(new[t])
            r.pos.copy_(i32(pos[t]))
        a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.out, b.out) and torch.equal(a.k, b.k) and torch.equal(a.v, b.v)
    assert ap.apack_device_error(a.ws) == ap.APACK_OK and ap.apack_device_error(b.ws) == ap.APACK_OK
    ref, _, spread, size = po.paged_decode(f64(a.q[1]), f64(a.k[1]), f64(a.v[1]), table, [n + steps for n in lens0], dim ** -0.5)
    tol = 2.0 ** -8 * np.abs(ref) + spread * (2.0 ** -16 + 100 * 2.0 ** -23 + 2.0 ** -19 * size)[..., None]
    assert np.all(np.abs(f64(a.out[1]) - ref) <= tol)


def test_two_streams_with_their_own_workspaces(ap):
    rng = np.random.default_rng(17)
    lens = [3000, 1, 900]
    table, pages = make_table(rng, lens, 16)
    k, v = (make_pool(rng, 1, pages, 16, 4, 128, torch.bfloat16) for _ in range(2))
    cache = ap.PagedCache(k, v, i32(table))
    q = normal(rng, (2, 3, 28, 128), torch.bfloat16)
    n = ap.apack_paged_decode_workspace_size(cache, 28)
    l = i32(lens)
    want = torch.empty(2, 3, 28, 128, dtype=torch.bfloat16, device="cuda")
    ws = [workspace(n), workspace(n)]
    for i in range(2):
        ap.apack_paged_decode_attention(cache, 0, l, q[i], want[i], ws[i])
    got = torch.empty_like(want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            ap.apack_paged_decode_attention(cache, 0, l, q[i], got[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_prune_into_pages_and_decode(ap):
    """The operators together, as a program uses them: a prompt is rotated and written, scored and selected by the
    framework's own calls, its survivors move into pages, a sequence forks, and both decode."""
    import oracle
    rng = np.random.default_rng(18)
    hq, hkv, dim, T, nq = 28, 4, 128, 400, 4
    mod = np.zeros(T, np.uint8)
    mod[10:390] = 1 + (np.arange(380) % 3 > 0)
    x = normal(rng, (T, hq + 2 * hkv, dim), torch.bfloat16)
    pos = np.stack([np.arange(T), rng.integers(0, 50, T), rng.integers(0, 50, T)])
    rot = ap.Rotary(dim, base=1e6, sections=[16, 24, 24])
    slab_k, slab_v = (torch.zeros(1, 1, T, hkv, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slab = ap.PagedCache(slab_k, slab_v, i32([[0]]))
    q = torch.empty(T, hq, dim, dtype=torch.bfloat16, device="cuda")
    ap.apack_rotary_append(rot, slab, 0, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q, i32(pos), i32(np.arange(T)),
                           seqs=i32(np.zeros(T)))
    seqs = ap.Seqs([0, T], [0, nq], [int((mod == 1).sum())], [int((mod == 2).sum())], torch.from_numpy(mod).cuda(), hq, hkv)
    ws = workspace(ap.apack_workspace_size(seqs))
    scores = torch.empty(T, device="cuda")
    qrows = q[T - nq:].contiguous()
    ap.apack_score(seqs, qrows, slab_k, hkv * dim * 2, scores, ws)
    counts, cu = ap.apack_keep_counts(seqs, np.array([[0.3, 0.2]], np.float32))
    keep, cu_d = torch.empty(int(cu[-1]), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    ap.apack_select(seqs, scores, counts, keep, ws, new_cu_seqlens=cu_d)
    n = int(cu[-1])
    page = 16
    own = -(-n // page)
    k, v = (normal(rng, (1, 2 * own + 4, page, hkv, dim), torch.bfloat16) for _ in range(2))
    perm = rng.permutation(2 * own + 4)
    table = np.full((2, own + 1), -1)
    table[0, :own] = perm[:own]
    pool = ap.PagedCache(k, v, i32(table[:1]))
    ap.apack_paged_compact(slab, pool, cu_d, n, keep_idx=keep, ws=ws)
    # the fork shares the full pages and gets a last page of its own
    table[1, :own] = table[0, :own]
    table[1, own - 1] = perm[own]
    table[:, own] = perm[own + 1], perm[own + 2]
    both = ap.PagedCache(k, v, i32(table))
    ap.apack_copy_pages(both, i32([[table[0, own - 1], table[1, own - 1]]]), ws=ws)
    y = normal(rng, (2, hq + 2 * hkv, dim), torch.bfloat16)
    q1 = torch.empty(2, hq, dim, dtype=torch.bfloat16, device="cuda")
    newpos = np.full((3, 2), T)
    ap.apack_rotary_append(rot, both, 0, y[:, :hq], y[:, hq:hq + hkv], y[:, hq + hkv:], q1, i32(newpos), i32([n, n]), ws=ws)
    out = torch.empty(2, hq, dim, device="cuda")
    ws2 = workspace(ap.apack_paged_decode_workspace_size(both, hq))
    ap.apack_paged_decode_attention(both, 0, i32([n + 1, n + 1]), q1, out, ws2)
    for w in (ws, ws2):
        assert ap.apack_device_error(w) == ap.APACK_OK
    # the same in 64 bits from the kept rows
    idx = keep.cpu().numpy()
    ref_scores = oracle.relevance_scores(q[T - nq:].cpu().view(torch.int16).numpy().view(np.uint16),
                                         slab_k[0, 0].cpu().view(torch.int16).numpy().view(np.uint16),
                                         np.array([0, T]), np.array([0, nq]), mod, hq, hkv)
    assert np.all(np.abs(f64(scores) - ref_scores) <= oracle.score_tolerance(ref_scores))
    kk, vv = f64(slab_k[0, 0])[idx], f64(slab_v[0, 0])[idx]
    for b in range(2):
        kb = np.concatenate([kk, f64(k[0, table[b, n // page], n % page])[None]])
        vb = np.concatenate([vv, f64(v[0, table[b, n // page], n % page])[None]])
        ref, _, spread, size = po.paged_decode(f64(q1[b:b + 1]), kb[:, None], vb[:, None], np.arange(n + 1)[None], [n + 1], dim ** -0.5)
        tol = spread * (2.0 ** -16 + 200 * 2.0 ** -23 + 2.0 ** -19 * size)[..., None]
        assert np.all(np.abs(f64(out[b:b + 1]) - ref) <= tol)
    krot = po.rotary(f64(y[:, hq:hq + hkv]), newpos, rot.frequencies, [16, 24, 24])
    assert np.all(np.abs(np.stack([f64(k[0, table[b, n // page], n % page]) for b in range(2)]) - krot)
                  <= rotary_bound(f64(y[:, hq:hq + hkv]), rot.frequencies, newpos, [16, 24, 24], False, 1.0, krot, torch.bfloat16))


def test_tensors_elsewhere_are_refused(ap):
    x = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        ap.apack_rotary(ap.Rotary(64), x, pos, x)


def test_page_pool_prunes_forks_and_decodes(ap):
    """PagePool on the device: prefill caches taken with their kept rows, a fork, steps of both, a prune of one of them
    while it shares pages and of the other in place; every decode against the rows that the model keeps."""
    from paper_2608_08794_gb300.paged import PagePool
    rng = np.random.default_rng(19)
    hq, hkv, dim, layers, T = 8, 2, 128, 3, 300
    slab_k, slab_v = (normal(rng, (layers, 1, T, hkv, dim), torch.bfloat16) for _ in range(2))
    slab = ap.PagedCache(slab_k, slab_v, i32([[0]]))
    pool = PagePool(layers, 60, 16, hkv, dim, 4, max_pages=24)
    pool.k.fill_(math.nan)
    pool.v.fill_(math.nan)
    ws = workspace(ap.apack_paged_decode_workspace_size(pool.cache, hq))
    keep = np.sort(rng.permutation(T)[:201])
    a, = pool.take(slab, [201], keep_idx=i32(keep), ws=ws)
    rows = {a: [(f64(slab_k[:, 0, r]), f64(slab_v[:, 0, r])) for r in keep]}

    def step(seqs):
        first = pool.extend(seqs)
        kv = normal(rng, (layers, len(seqs), 2 * hkv, dim), torch.bfloat16)
        for i in range(layers):
            ap.apack_rotary_append(None, pool.cache, i, None, kv[i, :, :hkv], kv[i, :, hkv:], None, None, first, seqs=i32(seqs), ws=ws)
        for j, s in enumerate(seqs):
            rows[s] = rows[s] + [(f64(kv[:, j, :hkv]), f64(kv[:, j, hkv:]))]
        q, out = normal(rng, (4, hq, dim), torch.bfloat16), torch.empty(4, hq, dim, device="cuda")
        for i in range(layers):
            ap.apack_paged_decode_attention(pool.cache, i, pool.lengths, q, out, ws)
            for s in range(4):
                if s not in rows:
                    assert not out[s].any()
                    continue
                k, v = (np.stack([r[x][i] for r in rows[s]])[:, None] for x in (0, 1))
                ref, _, spread, size = po.paged_decode(f64(q[s:s + 1]), k, v, np.arange(len(k))[None], [len(k)], dim ** -0.5)
                tol = spread * (2.0 ** -16 + 120 * 2.0 ** -23 + 2.0 ** -19 * size)[..., None]
                assert np.all(np.abs(f64(out[s:s + 1]) - ref) <= tol)

    def prune(s, m, in_place=None):
        picks = np.sort(rng.permutation(len(rows[s]))[:m])
        pool.prune([s], i32(picks), [m], in_place=in_place, ws=ws)
        rows[s] = [rows[s][i] for i in picks]

    step([a])
    b = pool.fork(a)
    rows[b] = list(rows[a])
    step([b, a])
    prune(b, 90)                                   # shares pages with a: into new pages
    step([a, b])
    prune(b, 40, in_place=True)                    # its pages are its own now
    step([b])
    pool.free(a)
    del rows[a]
    step([b])
    assert ap.apack_device_error(ws) == ap.APACK_OK
    assert pool.free_pages == 60 - len(pool.pages(b))


FIRST_CALLS = r"""
import sys, threading
import torch
sys.path.insert(0, sys.argv[1])
import __graft_entry__
__graft_entry__.build()
import paper_2608_08794_gb300 as ap

torch.manual_seed(0)
n, hq, hkv = 300, 40, 4                                   # rings of two warps; the eager calls below take the same path
k, v = (torch.randn(1, 20, 16, hkv, 128, device="cuda").bfloat16() for _ in range(2))
table = torch.arange(19, -1, -1, dtype=torch.int32, device="cuda").view(1, 20)
cache = ap.PagedCache(k, v, table)
lens = torch.tensor([n], dtype=torch.int32, device="cuda")
row = lens - 1
x = torch.randn(1, hq + 2 * hkv, 128, device="cuda").bfloat16()
pos = torch.tensor([123456], dtype=torch.int32, device="cuda")
rot = ap.Rotary(128)
ws = torch.zeros(ap.apack_paged_decode_workspace_size(cache, hq) + 256, dtype=torch.uint8, device="cuda")
ws = ws[(-ws.data_ptr()) % 256:][:-256]
q, out = torch.empty(1, hq, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(1, hq, 128, device="cuda")
torch.cuda.synchronize()
assert ap.apack_launch_count() == 0
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):                             # the first calls of the process are captured
    ap.apack_rotary_append(rot, cache, 0, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q, pos, row)
    ap.apack_paged_decode_attention(cache, 0, lens, q, out, ws)
for _ in range(2):
    graph.replay()
torch.cuda.synchronize()
want = out.clone()

# then from two threads at once, each on a stream and with tensors of its own
go, errors, outs = threading.Barrier(2), [], {}
def work(i):
    try:
        torch.cuda.set_device(0)
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            w, o, qq = ws.clone(), torch.empty_like(out), torch.empty_like(q)
            off = (-w.data_ptr()) % 256
            assert off == 0
            s.synchronize()
            go.wait()
            for _ in range(50):
                ap.apack_rotary(rot, x[:, :hq], pos, qq)
                ap.apack_paged_decode_attention(cache, 0, lens, qq, o, w)
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


def test_first_calls_captured_and_calls_from_two_threads():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS, root], capture_output=True, text=True, cwd=root, timeout=600)
    assert r.returncode == 0 and "first calls ok" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]
