"""Pins of the paged-cache oracle (CPU): hand values, invariants and the contiguous decode oracle."""

import numpy as np

import oracle
from oracle import paged_oracle as po
from synth.gen import f32_to_bf16_bits


def test_rotary_hand_values_and_invariants():
    x = np.zeros((1, 1, 6))
    x[0, 0] = [1, 2, 3, 4, 5, 6]
    f = np.array([np.pi / 2, np.pi])
    # halves: pairs (1, 3) by 90 degrees and (2, 4) by 180
    np.testing.assert_allclose(po.rotary(x, [[1]], f)[0, 0], [-3, -2, 1, -4, 5, 6], atol=1e-12)
    np.testing.assert_allclose(po.rotary(x, [[1]], f, interleaved=True)[0, 0], [-2, 1, -3, -4, 5, 6], atol=1e-12)
    # the second pair takes its position from the second axis
    np.testing.assert_allclose(po.rotary(x, [[1], [2]], f, sections=[1, 1])[0, 0], [-3, 2, 1, 4, 5, 6], atol=1e-12)
    rng = np.random.default_rng(0)
    x, y = rng.standard_normal((2, 5, 3, 16))
    f = 10000.0 ** (-np.arange(8) / 8)
    p = [[3, 9, 1000, 0, -4]]
    r = po.rotary(x, p, f, magnitude=1.5)
    np.testing.assert_allclose(np.linalg.norm(r, axis=-1), 1.5 * np.linalg.norm(x, axis=-1))
    # the transpose is the adjoint, and with magnitude 1 the inverse
    np.testing.assert_allclose((r * y).sum(), (x * po.rotary(y, p, f, magnitude=1.5, transpose=True)).sum())
    np.testing.assert_allclose(po.rotary(po.rotary(x, p, f), p, f, transpose=True), x, atol=1e-12)
    # scores depend on the distance alone
    a = (po.rotary(x, p, f) * po.rotary(y, [[v + 7 for v in p[0]]], f)).sum(-1)
    b = (x * po.rotary(y, [[7] * 5], f)).sum(-1)
    np.testing.assert_allclose(a, b, atol=1e-10)


def test_paged_decode_equals_the_contiguous_oracle():
    rng = np.random.default_rng(1)
    lens = [0, 1, 5, 13]
    cu = np.concatenate([[0], np.cumsum(lens)])
    k, v = (f32_to_bf16_bits(rng.standard_normal((cu[-1], 2, 128)).astype(np.float32)) for _ in range(2))
    q = f32_to_bf16_bits(rng.standard_normal((4, 6, 128)).astype(np.float32))
    k64, v64, q64 = (oracle.bf16_to_f64(x) for x in (k, v, q))
    table = np.array([[-1, -1, -1, -1], [7, -1, -1, -1], [0, 6, -1, -1], [2, 1, 5, 3]])
    kp, vp = np.full((2, 8, 4, 2, 128), np.nan)
    for b, n in enumerate(lens):
        for r in range(n):
            kp[table[b, r // 4], r % 4] = k64[cu[b] + r]
            vp[table[b, r // 4], r % 4] = v64[cu[b] + r]
    out, lse, spread, size = po.paged_decode(q64, kp, vp, table, lens, 128 ** -0.5)
    np.testing.assert_allclose(out, oracle.decode_attention(q, k, v, cu, 6, 2), rtol=1e-12, atol=1e-14)
    assert np.all(lse[0] == -np.inf) and np.all(out[0] == 0)
    x = k64[0] @ q64[1].T * 128 ** -0.5            # one row: its logit
    np.testing.assert_allclose(lse[1], [x[h // 3, h] for h in range(6)])
    assert np.all(spread >= np.abs(out) - 1e-15) and np.all(size[2] >= np.abs(lse[2]) - np.log(5))


def test_move_rows_by_hand():
    src = np.arange(6.).reshape(1, 3, 2, 1)                # pages (0, 1), (2, 3), (4, 5)
    dst = -np.ones((1, 2, 4, 1))
    got = po.move_rows(src, dst, [[2, 0], [1, -1]], [[1], [0]], [0, 2, 3], keep=[1, 2, 5], cu_src=[0, 4])
    assert got[0, 1, :, 0].tolist() == [5, 0, -1, -1] and got[0, 0, :, 0].tolist() == [3, -1, -1, -1]
