"""Attention over shared rows with pages whose rows are copied by the lanes, in segments of several tiles whose tiles the two
accumulators take in turn: more tiles than the ring holds, and segments behind one another.  Tolerances: test_gpu_group.py."""

import pytest

from test_gpu_group import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


def in_turn(b):
    """Tiles of the planned segments whose tiles the accumulators take in turn."""
    head = b.ws[256:336].view(b.cu_q.dtype)
    at = 1024 + (b.n_q * 16 + 255) // 256 * 256
    segs = b.ws[at:at + 32 * int(head[9])].view(b.cu_q.dtype).view(-1, 8).tolist()
    return {-(-(key1 - key0) // 128) for _, _, _, _, key0, key1, _, step in segs if step > 0}


@pytest.mark.parametrize("heads,dim,dtype,page,groups,tiles", [
    ("28/4", 128, "bf16", 1, [(0, [(27000, 1)])], {6}),
    ("28/4", 128, "fp16", 7, [(0, [(14000, 2)])], {3}),
    ("28/4", 128, "fp16", 1, [(0, [(9000, 2)]), (0, [(8800, 1)]), (0, [(300, 1)])], {3, 4}),
    ("32/8", 128, "bf16", 12, [(0, [(1500 + 37 * i, 1 + i % 3)]) for i in range(20)], {3, 4, 5}),
    ("32/8", 128, "bf16", 7, [(0, [(1200, 1)])] * 4 + [(0, [(500, 1)])] * 20, {4, 10}),
    ("28/4", 64, "bf16", 1, [(0, [(27000, 1)])], {6}),
    ("32/8", 64, "fp16", 12, [(0, [(1500 + 37 * i, 1 + i % 3)]) for i in range(20)], {3, 4, 5}),
])
def test_tiles_in_turn(ap, heads, dim, dtype, page, groups, tiles):
    b = Batch(ap, heads, dim, dtype, page, groups, seed=page)
    b.plan()
    assert tiles <= in_turn(b)
    b.check(*b.attend())
    assert ap.apack_device_error(b.ws) == 0
