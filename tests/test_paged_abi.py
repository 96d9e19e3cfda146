"""The paged-cache entry points on the host: descriptors, refusals and frequencies (no device work)."""

import ctypes
import math

import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def cache(ap, layers=2, pages=6, tokens=16, heads=4, dim=128, dtype=torch.bfloat16, seqs=2, columns=3):
    k = torch.zeros(layers, pages, tokens, heads, dim, dtype=dtype)
    return ap.PagedCache(k, torch.zeros_like(k), torch.zeros(seqs, columns, dtype=torch.int32))


def status(ap, call):
    with pytest.raises(ap.ApackError) as e:
        call()
    return e.value.status


def test_frequencies(ap):
    i = np.arange(64)
    base = 1e6
    plain = base ** (-2.0 * i / 128)
    np.testing.assert_allclose(ap.Rotary(128, base).frequencies, plain, rtol=1e-14)
    np.testing.assert_allclose(ap.Rotary(128, base, scaling="linear", factor=4).frequencies, plain / 4, rtol=1e-14)
    np.testing.assert_allclose(ap.Rotary(128, base, scaling="ntk", factor=4).frequencies,
                               (base * 4 ** (128 / 126)) ** (-2.0 * i / 128), rtol=1e-13)
    y = ap.Rotary(128, base, scaling="yarn", factor=4, original_len=32768)
    turns = 32768 * plain / (2 * math.pi)
    np.testing.assert_allclose(y.frequencies[turns >= 32], plain[turns >= 32], rtol=1e-14)     # kept
    np.testing.assert_allclose(y.frequencies[turns <= 1], plain[turns <= 1] / 4, rtol=1e-14)   # stretched
    between = (turns > 1) & (turns < 32)
    g = (turns[between] - 1) / 31
    np.testing.assert_allclose(y.frequencies[between], plain[between] * g + plain[between] / 4 * (1 - g), rtol=1e-13)
    assert between.any() and y.magnitude == np.float32(0.1 * math.log(4) + 1)
    assert ap.Rotary(128, base, scaling="yarn", factor=1, original_len=10).magnitude == 1
    for bad in (dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=258), dict(rotary_dim=8, base=0.0),
                dict(rotary_dim=8, base=math.nan), dict(rotary_dim=2, scaling="ntk", factor=2),
                dict(rotary_dim=8, scaling="linear", factor=0.5), dict(rotary_dim=8, scaling="yarn", factor=2),
                dict(rotary_dim=8, scaling="yarn", factor=2, original_len=9, beta_fast=1.0, beta_slow=1.0)):
        assert status(ap, lambda: ap.Rotary(**bad)) == ap.APACK_EINVAL
    with pytest.raises(ValueError):
        ap.Rotary(8, scaling="other")
    with pytest.raises(ValueError):
        ap.Rotary(8, frequencies=[1.0, 2.0])
    with pytest.raises(ValueError):
        ap.Rotary(8, sections=[1, 1, 1, 1])


def test_descriptors(ap):
    c = cache(ap)
    assert ap.apack_paged_decode_workspace_size(c, 28) > 0
    for field, value, want in (("k", None, "EINVAL"), ("v", None, "EINVAL"), ("num_layers", 0, "EINVAL"),
                               ("num_pages", 0, "EINVAL"), ("page_tokens", 0, "EINVAL"), ("num_kv_heads", 0, "EINVAL"),
                               ("num_kv_heads", 257, "EINVAL"), ("head_dim", 96, "EUNSUPPORTED"),
                               ("dtype", ap.APACK_FP32, "EUNSUPPORTED"), ("token_stride", 1000, "EINVAL"),
                               ("token_stride", 512, "EINVAL"), ("head_stride", 128, "EINVAL"),
                               ("page_stride", 16 * 1024 - 16, "EINVAL"), ("page_stride", -16384, "EINVAL"),
                               ("layer_stride", 5 * 16384, "EINVAL"), ("page_table", None, "EINVAL"),
                               ("num_seqs", 0, "EINVAL"), ("num_seqs", 4097, "EINVAL"),
                               ("max_pages", 0, "EINVAL"), ("table_stride", 2, "EINVAL")):
        bad = cache(ap)
        setattr(bad.struct, field, value)
        assert status(ap, lambda: ap.apack_paged_decode_workspace_size(bad, 28)) == getattr(ap, "APACK_" + want), field
    assert status(ap, lambda: ap.apack_paged_decode_workspace_size(c, 30)) == ap.APACK_EINVAL
    assert status(ap, lambda: ap.apack_paged_decode_workspace_size(c, 4 * 33)) == ap.APACK_EUNSUPPORTED
    # heads outermost in a page, layers inside pages, and a single page without a stride are pools too
    k = torch.zeros(2, 6, 4, 16, 128, dtype=torch.float16)
    t = torch.zeros(2, 3, dtype=torch.int32)
    assert ap.apack_paged_decode_workspace_size(ap.PagedCache(k.permute(0, 1, 3, 2, 4), k.permute(0, 1, 3, 2, 4), t), 4) > 0
    inside = torch.zeros(6, 2, 16, 4, 128, dtype=torch.float16).transpose(0, 1)
    assert ap.apack_paged_decode_workspace_size(ap.PagedCache(inside, inside, t), 4) > 0
    one = torch.zeros(1, 1, 1000, 4, 64, dtype=torch.float16)
    assert ap.apack_paged_decode_workspace_size(ap.PagedCache(one, one, t), 4) > 0
    with pytest.raises(ValueError):
        ap.PagedCache(k, k[:1], t)
    with pytest.raises(ValueError):
        ap.PagedCache(k, k.permute(0, 1, 3, 2, 4), t)
    with pytest.raises(ValueError):
        ap.PagedCache(k, k, t.long())


def test_attention_refusals(ap):
    c = cache(ap)
    q = torch.zeros(2, 28, 128, dtype=torch.bfloat16)
    out, lens = torch.zeros_like(q), torch.zeros(2, dtype=torch.int32)
    n = ap.apack_paged_decode_workspace_size(c, 28)
    raw = torch.zeros(n + 256, dtype=torch.uint8)
    ws = raw[(-raw.data_ptr()) % 256:][:n]

    def call(**kw):
        a = dict(cache=c, layer=0, seqlens=lens, q=q, out=out, ws=ws, stream=0)
        a.update(kw)
        return lambda: ap.apack_paged_decode_attention(**a)

    assert status(ap, call(layer=2)) == ap.APACK_EINVAL
    assert status(ap, call(layer=-1)) == ap.APACK_EINVAL
    assert status(ap, call(scale=0.0)) == ap.APACK_EINVAL
    assert status(ap, call(scale=math.inf)) == ap.APACK_EINVAL
    assert status(ap, call(ws=ws[:-256])) == ap.APACK_EWORKSPACE
    assert status(ap, call(ws=raw[(-raw.data_ptr()) % 256 + 16:][:n])) in (ap.APACK_EINVAL, ap.APACK_EWORKSPACE)
    assert status(ap, call(out=out.half())) == ap.APACK_EINVAL          # neither the cache's type nor fp32
    assert status(ap, call()) == ap.APACK_EINVAL                        # host memory: nothing is launched
    for kw in (dict(q=q.half()), dict(q=q[:1]), dict(q=q[..., :64]), dict(q=q.transpose(0, 1)), dict(out=out[:1]),
               dict(seqlens=lens.long()), dict(seqlens=lens[:1]), dict(lse=torch.zeros(2, 28, dtype=torch.float64)),
               dict(lse=torch.zeros(28, 2))):
        with pytest.raises(ValueError):
            call(**kw)()


def test_rotary_refusals(ap):
    r = ap.Rotary(128, sections=[16, 24, 24])
    x = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    pos = torch.zeros(3, 3, dtype=torch.int32)
    for kw in (dict(positions=pos.long()), dict(positions=pos[:2]), dict(positions=pos[0]), dict(positions=pos[:, :2]),
               dict(out=x.half()), dict(out=x[:2]), dict(x=x.transpose(0, 1)), dict(x=x.double())):
        with pytest.raises(ValueError):
            ap.apack_rotary(**dict(dict(rotary=r, x=x, positions=pos, out=torch.zeros_like(x), stream=0), **kw))

    def raw(spec, dim=128, heads=4, n=3, dtype=ap.APACK_BF16, xp=x.data_ptr(), xs=1024, op=x.data_ptr(), os=1024, axis=3):
        return ap._lib.apack_rotary(ctypes.addressof(spec.struct), dtype, n, heads, dim, xp, xs, op, os, pos.data_ptr(), axis, 0, 0)

    assert raw(r, n=0) == ap.APACK_OK
    assert raw(r, n=-1) == ap.APACK_EINVAL and raw(r, heads=0) == ap.APACK_EINVAL
    assert raw(r, dim=64) == ap.APACK_EINVAL                            # rotary_dim above the head
    assert raw(r, dim=258) == ap.APACK_EUNSUPPORTED and raw(r, dtype=7) == ap.APACK_EUNSUPPORTED
    assert raw(r, xs=1022) == ap.APACK_EINVAL and raw(r, xs=1025) == ap.APACK_EINVAL
    assert raw(r, xp=x.data_ptr() + 1) == ap.APACK_EINVAL and raw(r, xp=None) == ap.APACK_EINVAL
    assert raw(r, os=2048) == ap.APACK_EINVAL                           # in place with another stride
    assert raw(r, axis=2) == ap.APACK_EINVAL
    for sections in ([16, 24, 25], [-1, 33, 32]):
        assert raw(ap.Rotary(128, sections=sections)) == ap.APACK_EINVAL
    assert raw(ap.Rotary(128, magnitude=math.inf)) == ap.APACK_EINVAL
    assert raw(ap.Rotary(128, frequencies=[math.nan] * 64)) == ap.APACK_EINVAL


def test_append_refusals(ap):
    c = cache(ap)
    r = ap.Rotary(128)
    qkv = torch.zeros(2, 36, 128, dtype=torch.bfloat16)
    q, k, v = qkv[:, :28], qkv[:, 28:32], qkv[:, 32:]
    rows, pos = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    base = dict(rotary=r, cache=c, layer=0, q=q, k=k, v=v, q_out=torch.zeros_like(q), positions=pos, rows=rows, stream=0)
    for kw in (dict(q_out=None), dict(q=None), dict(k=k[:1]), dict(v=v.half()), dict(rows=rows.long()),
               dict(rows=rows[:1]), dict(seqs=rows.long()), dict(positions=pos[:1]), dict(q=q[..., :64])):
        with pytest.raises(ValueError):
            ap.apack_rotary_append(**dict(base, **kw))
    assert status(ap, lambda: ap.apack_rotary_append(**dict(base, layer=2))) == ap.APACK_EINVAL
    big = torch.zeros(3, 36, 128, dtype=torch.bfloat16)                  # more tokens than sequences, and no seqs
    three = torch.zeros(3, dtype=torch.int32)
    assert status(ap, lambda: ap.apack_rotary_append(**dict(base, q=None, q_out=None, k=big[:, 28:32], v=big[:, 32:],
                                                            rows=three, positions=three))) == ap.APACK_EINVAL
    odd = torch.zeros(2 * 4 * 128 + 4, dtype=torch.bfloat16)[4:].view(2, 4, 128)   # 8 bytes off
    assert odd.data_ptr() % 16 == 8
    assert status(ap, lambda: ap.apack_rotary_append(**dict(base, k=odd))) == ap.APACK_EINVAL
    assert status(ap, lambda: ap.apack_rotary_append(**dict(base, rotary=ap.Rotary(64, frequencies=[math.inf] * 32)))) == ap.APACK_EINVAL


def test_move_refusals(ap):
    a, b = cache(ap), cache(ap, pages=9, tokens=32)
    cu, keep = torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)

    def call(src=a, dst=b, n_out=4, **kw):
        return lambda: ap.apack_paged_compact(src, dst, cu, n_out, **dict(dict(keep_idx=keep, stream=0), **kw))

    for kw in (dict(n_out=-1), dict(dst=cache(ap, heads=2)), dict(dst=cache(ap, dim=64)),
               dict(dst=cache(ap, dtype=torch.float16)),
               dict(num_layers=0), dict(num_layers=3), dict(src_layer=-1), dict(src_layer=2, num_layers=1),
               dict(dst_layer=1, num_layers=2), dict(keep_idx=None, cu_src=cu)):
        assert status(ap, call(**kw)) == ap.APACK_EINVAL, kw
    # one table on both sides: in place with an index, or layers apart
    assert status(ap, call(dst=a, keep_idx=None)) == ap.APACK_EINVAL
    assert status(ap, call(src=cache(ap, layers=3), dst_layer=1, num_layers=2)) == ap.APACK_EINVAL
    three = cache(ap, layers=3)
    assert status(ap, call(src=three, dst=three, dst_layer=1, num_layers=2)) == ap.APACK_EINVAL
    assert status(ap, call(src=three, dst=three, dst_layer=1, num_layers=1)) == ap.APACK_ECUDA      # goes on to the device
    assert status(ap, call(dst=ap.PagedCache(a.k, a.k, a.page_table))) == ap.APACK_EINVAL
    other = ap.PagedCache(a.k, a.v, torch.zeros(2, 3, dtype=torch.int32))                           # other pages of a pool
    assert status(ap, call(dst=other)) == ap.APACK_ECUDA
    for kw in (dict(n_out=5), dict(keep_idx=keep.long()), dict(cu_src=cu[:2])):
        with pytest.raises(ValueError):
            call(**kw)()
    call(n_out=0)()                                                      # nothing to do, nothing launched
    pairs = torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        ap.apack_copy_pages(a, pairs.long(), stream=0)
    with pytest.raises(ValueError):
        ap.apack_copy_pages(a, torch.zeros(2, 3, dtype=torch.int32), stream=0)
    ap.apack_copy_pages(a, pairs[:0], stream=0)
    assert ap._lib.apack_copy_pages(a._address, None, 2, None, 0) == ap.APACK_EINVAL
    assert ap._lib.apack_copy_pages(a._address, pairs.data_ptr(), -1, None, 0) == ap.APACK_EINVAL
    assert ap._lib.apack_copy_pages(a._address, pairs.data_ptr(), 1 << 40, None, 0) == ap.APACK_EINVAL
