"""README's decode loop over a PagePool, run as written, against the fp64 oracle."""

import os
import re

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from test_gpu_paged import f64, i32, normal, rotary_bound

pytestmark = pytest.mark.gpu


def test_decode_loop_of_the_readme():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2608_08794_gb300 as ap
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "README.md")) as f:
        block, = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "PagePool" in b]
    rng = np.random.default_rng(21)
    T, n, m, layers, last = 300, 131, 40, 28, 27
    k, v = (torch.randn(layers, 1, T, 4, 128, device="cuda").bfloat16() for _ in range(2))
    keep = np.sort(rng.permutation(T)[:n])
    new = [normal(rng, (64, 36, 128), torch.bfloat16) for _ in range(layers)]
    pos = rng.integers(0, 100000, (3, 64))
    names = dict(ap=ap, torch=torch, k=k, v=v, table=i32([[0]]), n=n, keep_idx=i32(keep), m=m,
                 later_keep_idx=i32(np.sort(rng.permutation(n + 1)[:m])), positions=i32(pos),
                 project=lambda layer: (new[layer][:, :28], new[layer][:, 28:32], new[layer][:, 32:]),
                 q_rot=torch.empty(64, 28, 128, dtype=torch.bfloat16, device="cuda"),
                 out=torch.empty(64, 28, 128, device="cuda"))
    exec(block, names)
    pool, seq, out, q = names["pool"], names["seq"], names["out"], names["q_rot"]
    assert ap.apack_device_error(names["ws"]) == ap.APACK_OK
    assert pool.length(seq) == m and len(pool.pages(seq)) == -(-m // 16) == 4096 - pool.free_pages
    # the last layer's attention: the kept rows and the new one
    x = f64(new[last])
    freq = names["rotary"].frequencies
    turned = po.rotary(x[seq:seq + 1, :32], pos[:, seq:seq + 1], freq, [16, 24, 24])
    bound = rotary_bound(x[seq:seq + 1, :32], freq, pos[:, seq:seq + 1], [16, 24, 24], False, 1.0, turned, torch.bfloat16)
    assert np.all(np.abs(f64(q)[seq] - turned[0, :28]) <= bound[0, :28])
    rounded = torch.from_numpy(turned[:, 28:]).bfloat16().double().numpy()
    kk, vv = (np.concatenate([f64(t[last, 0])[keep], r])[:, None] for t, r in ((k, rounded), (v, x[seq:seq + 1, 32:])))
    ref, _, spread, size = po.paged_decode(f64(q)[seq:seq + 1], kk, vv, np.arange(n + 1)[None], [n + 1], 128 ** -0.5)
    # the new key's elements may round the other way than their fp64 values do: 2^-8 of its logit's terms, and so of its weight
    own = po.paged_decode(f64(q)[seq:seq + 1], kk[-1:], vv[-1:], np.zeros((1, 1), int), [1], 128 ** -0.5)[3] * 2.0 ** -8
    tol = spread * (2.0 ** -21 + 100 * 2.0 ** -23 + 2.0 ** -19 * size + 2 * own)[..., None]
    assert np.all(np.abs(f64(out)[seq:seq + 1] - ref) <= tol)
    others = [s for s in range(64) if s != seq]
    assert not out[others].any()
