// group.cuh -- attention of a batch whose sequences share their first rows: what the plan (group_plan.cu) leaves in the
// workspace for the attention kernels (group_attention.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "paged.cuh"
#include "ptx.cuh"

namespace apack {

constexpr int kGTile = 128;          // keys of a tile
constexpr int kGSlot = 128;          // query rows of an accumulator
constexpr int kGRows = 2 * kGSlot;   // query rows of a segment
constexpr int32_t kGMagic = 0x47505631;

// Query rows are packed per KV head: row t * group + j is head h * group + j of token t, so that an item's rows are one
// run.  An item is a run of keys with the query rows that read it: the shared rows of a group with the new tokens of
// all its sequences, or the rest of one sequence with its own.  Its rows are cut into runs of 256, its keys into runs
// of `chunk` tiles; a segment is one of each, of one KV head.
struct GroupItem {
  int32_t seq;                       // row of the page table through which the keys are read
  int32_t key0, key1;                // keys [key0, key1)
  int32_t row0, rows;                // packed query rows; rows 0: nothing
  int32_t splits, chunk;             // runs of its keys, tiles of each
  int32_t sub;                       // 2: a segment of at most 128 rows writes two parts, of its even and odd tiles
  int32_t part;                      // first row of its parts: [split][sub][KV head][rows]
  int32_t causal;                    // rows see fewer keys than the item has
  int32_t pad[2];
};
struct GroupSeg {
  int32_t seq, head;
  int32_t row0, rows;                // packed query rows, of at most 256
  int32_t key0, key1;                // key0 >= key1: nothing to do
  int32_t part, step;                // its part's first row, and the second part's distance (0: one part; -1: one, and
                                     // its rows have no other: they are written out, and of the part (max, sum) alone)
};
struct GroupTok {
  int32_t limit;                     // keys that the token sees: those below it
  int32_t prefix, own;               // items, or -1
  int32_t real;                      // 0: behind the last sequence's tokens
};

struct GroupHead {
  int32_t magic, n_q, hq, hkv;
  int32_t head_dim, num_seqs, max_pages, page_tokens;
  int32_t num_pages, segs, causal_any, pad;
  int64_t item_off, ml_off, part_off, total;
};
constexpr size_t kGHeadOff = 256, kGClaimOff = 512, kGFixed = 1024;

// What the two calls agree on before anything is known of the lengths.
struct GroupShape {
  int group;
  int64_t cap_rows, cap_segs;
  size_t tok_off, item_off, seg_off, ml_off, part_off, total;
  bool halves;                       // segments of few rows may write two parts
};
apack_status group_shape(const apack_paged_cache *c, int32_t hq, int32_t n_seqs, int64_t n_q, GroupShape *s);

// Tokens of a TMA box (a tile is whole boxes, and a box lies in one page), or 0: rows are copied by the lanes.
inline int32_t group_box(int32_t page_tokens) {
  const int32_t low = page_tokens & -page_tokens;
  return low < 8 ? 0 : low < kGTile ? low : kGTile;
}

struct GroupArgs {
  PoolView pool;
  uint8_t *ws;
  int64_t ws_bytes;
  const uint8_t *q;
  int64_t q_stride;                  // bytes between tokens
  int32_t hq, hkv, group, n_q, head_dim;
  float scale2;                      // scale * log2(e)
  uint8_t *out;
  float *lse;
  int32_t box;                       // tokens of a TMA box, 0: rows are copied by the lanes
  int64_t seg_off;                   // of the segments in ws
  DeviceError *err;
};

// The plan's header, if it is one for this call.
__device__ __forceinline__ bool group_head(const GroupArgs &A, GroupHead &h) {
  const int4 *p = reinterpret_cast<const int4 *>(A.ws + kGHeadOff);
  int4 *d = reinterpret_cast<int4 *>(&h);
  static_assert(sizeof(GroupHead) == 80, "whole int4s");
#pragma unroll
  for (int i = 0; i < 5; ++i) d[i] = p[i];
  return h.magic == kGMagic && h.n_q == A.n_q && h.hq == A.hq && h.hkv == A.hkv && h.head_dim == A.head_dim &&
         h.num_seqs == A.pool.num_seqs && h.max_pages == A.pool.max_pages &&
         h.page_tokens == static_cast<int32_t>(A.pool.page_tokens.d) && h.num_pages == A.pool.num_pages &&
         h.total <= A.ws_bytes;
}

__device__ __forceinline__ float2 unpack16(uint32_t w, __nv_bfloat16) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ float2 unpack16(uint32_t w, __half) { return __half22float2(*reinterpret_cast<__half2 *>(&w)); }

// One query row by one warp, key by key: (max, sum, D / 32 values of the lane on from lane * D / 32) over keys
// [key0, key1) of `seq`, added to what the three hold.  fp32 throughout.
template <class T, int D>
__device__ void group_row(const GroupArgs &A, int seq, int head, int key0, int key1, const float *q, float &m, float &l,
                          float (&o)[D / 32]) {
  constexpr int kF = D / 32;
  const int lane = threadIdx.x & 31;
  for (int k0 = key0; k0 < key1; k0 += 32) {
    const int key = k0 + lane;
    int64_t off = -1;
    float x = -INFINITY;
    if (key < key1) {
      const int32_t page = A.pool.page_of(seq, key);
      off = A.pool.offset_in(page, key);
      if (off < 0) raise_device_error(A.err, APACK_EDEVICE, 140, seq, page);
      x = 0.f;                                                    // a page outside the pool is one of zeros
      if (off >= 0) {
        off += head * A.pool.head_stride;
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
          const uint4 w = *reinterpret_cast<const uint4 *>(A.pool.k + off + i * 16);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = unpack16(u[e], T());
            x = fmaf(f.x, q[i * 8 + 2 * e], x);
            x = fmaf(f.y, q[i * 8 + 2 * e + 1], x);
          }
        }
      }
      x *= A.scale2;
    }
    float top = x;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    top = fmaxf(top, m);
    const float f = m == top ? 1.f : ex2_approx(m - top);
    m = top;
    const float p = x == -INFINITY ? 0.f : ex2_approx(x - top);
    l *= f;
    float sum = p;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    l += sum;
#pragma unroll
    for (int e = 0; e < kF; ++e) o[e] *= f;
    const int n = min(32, key1 - k0);
    for (int j = 0; j < n; ++j) {
      const float pj = __shfl_sync(0xffffffffu, p, j);
      const int64_t oj = __shfl_sync(0xffffffffu, off, j);
      if (oj < 0) continue;
      const uint32_t *v = reinterpret_cast<const uint32_t *>(A.pool.v + oj + lane * kF * 2);
#pragma unroll
      for (int e = 0; e < kF / 2; ++e) {
        const float2 w = unpack16(v[e], T());
        o[2 * e] = fmaf(pj, w.x, o[2 * e]);
        o[2 * e + 1] = fmaf(pj, w.y, o[2 * e + 1]);
      }
    }
  }
}

}  // namespace apack
