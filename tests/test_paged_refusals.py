"""Refusals of the rotary calls (on the CPU: before anything is launched): outputs over rows that the call reads, and
missing positions."""

import numpy as np
import pytest
import torch


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


def test_rotary_over_other_rows_is_refused(ap):
    r = ap.Rotary(64)
    wide = torch.zeros(9, 6, 64, dtype=torch.bfloat16)
    pos = torch.zeros(9, dtype=torch.int32)

    def run(x, out):
        return status(ap, lambda: ap.apack_rotary(r, x, pos[:x.shape[0]], out, stream=0))

    flat = wide.view(-1)
    rows = wide[:, :2]
    for x, out in ((wide[:8], wide[1:]), (wide[1:], wide[:8]),                    # a token apart
                   (wide[:, :4], wide[:, 1:5]), (wide[:, 2:], wide[:, :4]),       # a head apart
                   (wide[:8, :3], wide[1:, 2:5]),                                 # both
                   (rows, flat[:9 * 2 * 64].view(9, 2, 64)),                      # other strides
                   (flat[64:64 + 9 * 2 * 64].view(9, 2, 64), rows),
                   (wide[0:9:2, :2], wide[:5, 1:3]),
                   (wide[:1], flat[8:8 + 6 * 64].view(1, 6, 64))):                # one token
        assert run(x, out) == ap.APACK_EINVAL


def test_append_over_rows_that_it_reads_is_refused(ap):
    cache = ap.PagedCache(*(torch.zeros(1, 4, 16, 2, 64, dtype=torch.bfloat16) for _ in range(2)),
                          torch.zeros(3, 2, dtype=torch.int32))
    qkv = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    other = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    n = torch.zeros(3, dtype=torch.int32)

    def run(q, k, v, q_out):
        return status(ap, lambda: ap.apack_rotary_append(ap.Rotary(64), cache, 0, q, k, v, q_out, n, n, stream=0))

    q, k, v = qkv[:, :4], qkv[:, 4:6], qkv[:, 6:]
    for q_out in (qkv[:, 1:5], qkv[:, 3:7], qkv[:, 4:]):                           # over q, k and v
        assert run(q, k, v, q_out) == ap.APACK_EINVAL
    assert run(other[:, :4], k, v, qkv[:, 4:]) == ap.APACK_EINVAL
    assert run(other[:, :4], k, other[:, 4:6], qkv[:, 1:5]) == ap.APACK_EINVAL      # k alone
    assert run(other[:, :4], other[:, 4:6], v, qkv.view(-1)[2 * 64:2 * 64 + 3 * 256].view(3, 4, 64)) == ap.APACK_EINVAL


def test_overlap_of_strided_rows_against_all_bytes(ap):
    """Random pairs of strided rows: refused exactly where they share a byte."""
    if torch.cuda.is_available():
        pytest.skip("what is not refused would go on to the device, with host memory")
    rng = np.random.default_rng(0)
    r = ap.Rotary(2)
    pos = torch.zeros(64, dtype=torch.int32)
    memory = torch.zeros(20000, dtype=torch.bfloat16)
    seen = [0, 0]
    for _ in range(200):
        n, heads, dim = int(rng.integers(1, 12)), int(rng.integers(1, 4)), int(rng.choice([2, 4, 16]))
        row = heads * dim
        sx = row + int(rng.integers(0, 40))
        so = sx if rng.random() < 0.5 else row + int(rng.integers(0, 40))
        x0, o0 = (int(v) for v in rng.integers(0, 300, 2))
        x = memory[x0:].as_strided((n, heads, dim), (sx, dim, 1))
        out = memory[o0:].as_strided((n, heads, dim), (so, dim, 1))
        in_x = {x0 + i * sx + e for i in range(n) for e in range(row)}
        in_out = {o0 + i * so + e for i in range(n) for e in range(row)}
        refused = bool(in_x & in_out) and not (x0 == o0 and (sx == so or n == 1))
        seen[refused] += 1
        code = ap._lib.apack_rotary(r._address, ap.APACK_BF16, n, heads, dim, x.data_ptr(), 2 * sx, out.data_ptr(), 2 * so,
                                    pos.data_ptr(), 64, 0, None)
        assert (code == ap.APACK_EINVAL) == refused, (n, heads, dim, x0, sx, o0, so)
    assert min(seen) > 30


def test_append_without_positions_is_a_value_error(ap):
    cache = ap.PagedCache(*(torch.zeros(1, 4, 16, 2, 64, dtype=torch.bfloat16) for _ in range(2)),
                          torch.zeros(3, 2, dtype=torch.int32))
    x, n = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="positions"):
        ap.apack_rotary_append(ap.Rotary(64), cache, 0, x, x, x, x.clone(), None, n, stream=0)


def test_handles_keep_what_they_were_made_with(ap):
    """The structures hold addresses of the arrays and tensors: nothing else can take their place."""
    rot = ap.Rotary(128, frequencies=np.arange(64.0))
    cache = ap.PagedCache(*(torch.zeros(1, 4, 16, 2, 64, dtype=torch.bfloat16) for _ in range(2)),
                          torch.zeros(3, 2, dtype=torch.int32))
    for handle, names in ((rot, ("frequencies", "rotary_dim", "magnitude", "num_axes")), (cache, ("k", "v", "page_table"))):
        for name in names:
            with pytest.raises(AttributeError):
                setattr(handle, name, getattr(handle, name))
    junk = [np.full(64, 7.5) for _ in range(300)]
    assert [rot.struct.freq_h[i] for i in range(64)] == list(range(64)) and len(junk) == 300
    assert (cache.struct.k, cache.struct.v, cache.struct.page_table) == (
        cache.k.data_ptr(), cache.v.data_ptr(), cache.page_table.data_ptr())
    assert (rot.rotary_dim, rot.magnitude, rot.num_axes) == (128, 1.0, 1)
    assert ap.Rotary(128, sections=[16, 24, 24], magnitude=1.1).num_axes == 3
