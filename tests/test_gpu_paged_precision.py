"""Precision of the paged attention's probabilities: fp32 outputs whose other errors are a few roundings."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ap():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    return ap


@pytest.mark.parametrize("hq,hkv,dim", [(28, 4, 128), (28, 4, 64), (32, 2, 128), (64, 2, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_probabilities_keep_32_bits(ap, dtype, hq, hkv, dim):
    """Two keys with logits 0 and -x, the first with the value 0 and the second with 1: out = p / (1 + p), p = e^-x.

    Errors relative to out, u = 2^-24, for 0 < x <= 1/2 (-x is a product of two 16-bit numbers, exact in fp32):
    x log2(e): its constant and the product in one rounding of less than 1, 2 u, which e turns into 2 ln 2 u;
    exp2 2^-22 = 4 u (twice, if both probabilities go through it); the sum, its reciprocal and the product 3 u; three
    terms of p that a matrix instruction may truncate 3 * 2 u; p itself as 16-bit terms: bf16 u / 2 or less with three,
    fp16 2^-22 = 4 u with two.  Below 24 u, taken as 2^-19.  Two terms of bf16 are off by up to 2^-17."""
    rng = np.random.default_rng(hq + dim)
    B = 40
    x = rng.uniform(0.01, 0.5, (B, hq))
    q = torch.zeros(B, hq, dim, dtype=dtype, device="cuda")
    q[:, :, 0] = torch.from_numpy(-x).to(dtype).cuda()
    k = torch.zeros(1, B, 16, hkv, dim, dtype=dtype, device="cuda")
    v = torch.zeros_like(k)
    k[:, :, 1, :, 0] = 1
    v[:, :, 1] = 1
    cache = ap.PagedCache(k, v, torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1))
    raw = torch.zeros(ap.apack_paged_decode_workspace_size(cache, hq) + 256, dtype=torch.uint8, device="cuda")
    ws = raw[(-raw.data_ptr()) % 256:][:-256]
    out = torch.empty(B, hq, dim, device="cuda")
    lens = torch.full((B,), 2, dtype=torch.int32, device="cuda")
    ap.apack_paged_decode_attention(cache, 0, lens, q, out, ws, scale=1.0)
    assert ap.apack_device_error(ws) == ap.APACK_OK
    p = np.exp(q[:, :, 0].double().cpu().numpy())
    want = (p / (1 + p))[..., None]
    worst = float((np.abs(out.double().cpu().numpy() - want) / want).max())
    assert worst <= 2.0 ** -19
