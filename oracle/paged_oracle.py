"""fp64 oracle of the paged-cache operators (test infrastructure): rotary positions, one-token
attention over pages, and the moves of rows and pages, from their definitions.

Arrays are float64 numpy; a pool is [pages, page_tokens, Hkv, D] of one layer."""

import numpy as np


def rotary(x, positions, freq, sections=None, interleaved=False, magnitude=1.0, transpose=False):
    """x [n, H, D], positions [axes, n], freq [r/2] radians per position."""
    n, _, _ = x.shape
    pairs = len(freq)
    sections = [pairs] if sections is None else list(sections)
    axis = np.repeat(np.arange(len(sections)), sections)
    out = np.array(x, np.float64)
    for t in range(n):
        for i in range(pairs):
            a = float(positions[axis[i]][t]) * freq[i]
            c, s = magnitude * np.cos(a), magnitude * np.sin(a)
            if transpose:
                s = -s
            lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
            u, w = np.array(out[t, :, lo]), np.array(out[t, :, hi])
            out[t, :, lo] = u * c - w * s
            out[t, :, hi] = w * c + u * s
    return out


def rows_of(pool, table_row, n):
    """The first n rows of a sequence, [n, Hkv, D]."""
    size = pool.shape[1]
    return np.stack([pool[table_row[r // size], r % size] for r in range(n)]) if n else pool[:0, 0]


def paged_decode(q, k_pool, v_pool, table, lens, scale):
    """Attention and ln-sum-exp; also, per query head, the two quantities that bound an fp32
    computation's error: sum_r p_r |v_r| and the largest scale * sum_i |q_i k_i|."""
    B, hq, D = q.shape
    hkv = k_pool.shape[2]
    out, lse = np.zeros((B, hq, D)), np.full((B, hq), -np.inf)
    spread, size = np.zeros((B, hq, D)), np.zeros((B, hq))
    for b in range(B):
        if lens[b] <= 0:
            continue
        k = rows_of(k_pool, table[b], lens[b])
        v = rows_of(v_pool, table[b], lens[b])
        for h in range(hq):
            g = h // (hq // hkv)
            x = scale * (k[:, g] @ q[b, h])
            m = x.max()
            p = np.exp(x - m)
            out[b, h] = p @ v[:, g] / p.sum()
            lse[b, h] = m + np.log(p.sum())
            spread[b, h] = p @ np.abs(v[:, g]) / p.sum()
            size[b, h] = scale * (np.abs(k[:, g]) @ np.abs(q[b, h])).max()
    return out, lse, spread, size


def move_rows(src, dst, src_table, dst_table, cu_dst, keep=None, cu_src=None):
    """Returns dst with the kept rows written (src and dst: [planes, pages, page_tokens, ...])."""
    out = np.array(dst)
    a, b = src.shape[1 + 1], dst.shape[1 + 1]
    source = np.array(src)
    for s in range(len(cu_dst) - 1):
        for j in range(cu_dst[s], cu_dst[s + 1]):
            to = j - cu_dst[s]
            frm = to if keep is None else keep[j] - (0 if cu_src is None else cu_src[s])
            out[:, dst_table[s][to // b], to % b] = source[:, src_table[s][frm // a], frm % a]
    return out


def group_attention(q, k_pool, v_pool, table, lens, seqs, new, scale):
    """Attention of each entry's new[e] last tokens (packed in q [n, Hq, D]) over the rows up to their own, every sequence
    by itself; also the lse and the two quantities of paged_decode that bound an fp32 computation's error."""
    n, hq, D = q.shape
    g = hq // k_pool.shape[2]
    out, lse = np.zeros((n, hq, D)), np.full((n, hq), -np.inf)
    spread, size = np.zeros((n, hq, D)), np.zeros((n, hq))
    at = 0
    for b, m in zip(seqs, new):
        k = rows_of(k_pool, table[b], lens[b])
        v = rows_of(v_pool, table[b], lens[b])
        for i in range(m):
            seen = lens[b] - m + i + 1
            if seen <= 0:
                continue
            for h in range(hq):
                kh, vh = k[:seen, h // g], v[:seen, h // g]
                x = scale * (kh @ q[at + i, h])
                top = x.max()
                p = np.exp(x - top)
                out[at + i, h] = p @ vh / p.sum()
                lse[at + i, h] = top + np.log(p.sum())
                spread[at + i, h] = p @ np.abs(vh) / p.sum()
                size[at + i, h] = scale * (np.abs(kh) @ np.abs(q[at + i, h])).max()
        at += m
    return out, lse, spread, size


class PageLists:
    """The bookkeeping of apack_pages_release, _fork and _extend with lists, one entry after the other."""

    def __init__(self, num_seqs, max_pages, num_pages, page_tokens):
        self.page, self.width = page_tokens, max_pages
        self.table = [[-1] * max_pages for _ in range(num_seqs)]
        self.lengths, self.refs = [0] * num_seqs, [0] * num_pages
        self.free = list(range(num_pages - 1, -1, -1))             # the last is on top

    def _count(self, rows):
        return -(-rows // self.page)

    def release(self, seqs, keep):
        given = []
        for b, n in zip(seqs, keep):
            for c in range(self._count(n), self._count(self.lengths[b])):
                given.append(self.table[b][c])
                self.table[b][c] = -1
            self.lengths[b] = n
        for p in given:
            self.refs[p] -= 1
        back = [p for i, p in enumerate(given) if self.refs[p] == 0 and p not in given[:i]]
        self.free += back[::-1]

    def fork(self, parents, seqs):
        for p, b in zip(parents, seqs):
            for c in range(self._count(self.lengths[p])):
                self.table[b][c] = self.table[p][c]
                self.refs[self.table[p][c]] += 1
            self.lengths[b] = self.lengths[p]

    def extend(self, seqs, grow):
        """Returns cu_new, rows, row_seqs, slots and pairs."""
        cu, rows, owners, slots, pairs = [0], [], [], [], []
        for b, m in zip(seqs, grow):
            n = self.lengths[b]
            pair = (0, 0)
            if m and n % self.page and self.refs[self.table[b][n // self.page]] > 1:
                pair = (self.table[b][n // self.page], self.free.pop())
                self.refs[pair[0]] -= 1
                self.refs[pair[1]] = 1
                self.table[b][n // self.page] = pair[1]
            for c in range(self._count(n), self._count(n + m)):
                self.table[b][c] = self.free.pop()
                self.refs[self.table[b][c]] = 1
            self.lengths[b] = n + m
            pairs.append(pair)
            cu.append(cu[-1] + m)
            rows += range(n, n + m)
            owners += [b] * m
            slots += [self.table[b][r // self.page] * self.page + r % self.page for r in range(n, n + m)]
        return cu, rows, owners, slots, pairs
