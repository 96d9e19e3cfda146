"""Attention over shared rows: outputs of rows of a single part, which are written without a merge."""

import math

import pytest
import torch

from test_gpu_group import Batch
from test_gpu_group_edges import near, slot

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


@pytest.mark.parametrize("heads,dim,dtype,page,groups", [
    ("28/4", 128, "bf16", 16, [(0, [(200 + 40 * i, 60 + 10 * i)]) for i in range(12)]),
    ("8/8", 64, "fp16", 32, [(0, [(300 + i, 290 + i % 9)]) for i in range(60)]),
    ("5/1", 128, "fp16", 7, [(0, [(260, 260)])] * 20),
])
def test_outputs_that_start_on_16_bytes(ap, heads, dim, dtype, page, groups):
    """A view into a larger buffer, 16 bytes behind a multiple of 32, and the lse 4 bytes behind one: the same bits."""
    b = Batch(ap, heads, dim, dtype, page, groups, seed=21, pad=2)
    b.plan()
    at = 1024 + (b.n_q * 16 + 255) // 256 * 256
    segs = b.ws[at:at + 32 * int(b.ws[256:336].view(torch.int32)[9])].view(torch.int32).view(-1, 8)
    assert (segs[:, 7] == -1).any()                                            # rows of a single part
    want = b.attend()
    near(b, *want)
    n = want[0].numel()
    room, room_lse = torch.full((n + 32,), 7.0, dtype=b.dt, device="cuda"), torch.full((want[1].numel() + 8,), 7.0, device="cuda")
    off = (-room.data_ptr() // 2) % 16 + 8
    out, lse = room[off:off + n].view(want[0].shape), room_lse[1:1 + want[1].numel()].view(want[1].shape)
    assert out.data_ptr() % 32 == 16
    b.ap.apack_paged_group_attention(b.cache, 0, b.q[0], out, b.ws, lse=lse)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert (room[:off] == 7).all() and (room[off + n:] == 7).all()
    assert (room_lse[:1] == 7).all() and (room_lse[1 + want[1].numel():] == 7).all()
    assert ap.apack_device_error(b.ws) == 0


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("heads,dim,dtype,page,count", [
    ("32/1", 128, "bf16", 16, 300), ("32/1", 64, "fp16", 16, 330), ("32/2", 128, "fp16", 7, 600),
    ("160/1", 128, "bf16", 16, 3), ("400/2", 64, "bf16", 32, 9),              # 129 to 256 query heads of a KV head
    ("28/4", 128, "bf16", 16, 40),                                            # (in parts)
])
def test_one_feature_that_is_no_number(ap, heads, dim, dtype, page, count, bad):
    """One token per sequence, so that every row sees all of its keys: a NaN or an infinity in one feature of one value reaches
    that feature of its KV head's rows and nothing else, and not the lse."""
    b = Batch(ap, heads, dim, dtype, page, [(0, [(1 + 31 * i % 200, 1)]) for i in range(count)], seed=22, pad=2)
    b.plan()
    want, want_lse = b.attend()
    near(b, want, want_lse)
    hit = torch.zeros_like(want, dtype=torch.bool)
    g = b.hq // b.hkv
    for i, feature in ((count - 1, 3), (count // 2, dim - 1)):
        row, head = int(b.seqlens[b.seqs[i]]) // 2, i % b.hkv
        p, s = slot(b, b.seqs[i], row)
        b.v[0, p, s, head, feature] = bad
        hit[i, head * g:(head + 1) * g, feature] = True
    out, lse = b.attend()
    assert torch.equal(lse, want_lse)
    assert torch.equal(out[~hit], want[~hit])
    assert torch.isnan(out[hit]).all() if math.isnan(bad) else not torch.isfinite(out[hit]).any()
    assert ap.apack_device_error(b.ws) == 0
