"""Attention over shared rows: outputs of rows of a single part, which are written without a merge."""

import pytest
import torch

from test_gpu_group import Batch
from test_gpu_group_edges import near

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
