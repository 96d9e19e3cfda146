// paged_decode.cu -- attention of one decode token per sequence over a paged key-value cache
// (the cost that Sec. 3.2's pruning shortens, over pages).
//
//   out[b, h] = sum_r softmax_r(scale q[b, h] . k[r, g(h)]) v[r, g(h)],  g(h) = h / (Hq / Hkv).
//
// Bound by HBM: K and V are read once, 4 D flop per query row and cached token.  With the G <= 8 query rows of a KV
// head as the N = 8 of a warp-level matrix instruction (keys, then features, as M) nothing is padded, the scores
// stay in registers from S^T = K Q^T over the softmax to O^T = V^T P^T, and no warp waits for another.
//
// Split over the cache's length.  The work is the list of all (sequence, head group, tile) in that order; every CTA
// takes an equal contiguous share of it and finds its start from the lengths on the device, so that the launch does
// not depend on them (a captured call follows growing caches).  Within a CTA a KV head has wph ring buffers of stages
// (filled by TMA from pages of a multiple of 8 or 16 tokens), each for every wph-th tile of the share; a ring is read by
// one warp of 8 or 16 query rows, or with more than 16 rows per KV head by 2 warps of 16.  Its first warp refills a
// stage as soon as it has been used.  At the end of a (sequence, head group) the warps of a head merge through shared
// memory; what a share holds whole is written out, what it holds in part goes to the workspace, and a second kernel
// merges those parts in order.
//
// Warp-level instructions, not tcgen05: that needs M = 128 keys, TMEM and a hand-over between warps for every tile of the
// same 8 rows, and the tensor work is far below what the read allows either way (on contiguous caches the tcgen05
// kernel of decode_tc.cu takes 50.6 us for the ten-minute cache).
//
// Measured (28/4 heads of 128, bf16, 16-token pages, calls in a row): 135,272 tokens (64-token pages) 50.4 us, 5.5 TB/s,
// 0.81 of the copy rate, of which the chunk kernel 45 us (0.9); 16 caches of 600 to 12,000 tokens 34.1 us; 473 tokens 8.3 us.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <numeric>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "paged.cuh"
#include "ptx.cuh"

namespace apack {
namespace {

// Tokens of a stage: 8 KB of K and V of one head.
constexpr int tile_tokens(int D) { return D == 64 ? 32 : 16; }
constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMergeFloats = 4096;              // shared-memory buffer of the warps' merge: 8 warps, 4 m-tiles
constexpr int kStageBytes = 16384 / 2;          // K and V of a tile
constexpr int kStageBytesCta = 196608;          // of all rings: three stages per warp
constexpr int kMaxStages = kStageBytesCta / kStageBytes;
constexpr int64_t kMaxUnits = INT32_MAX - 1024;   // of the work list

// What a (sequence, head group) costs a CTA beyond its tiles (its queries' latency, the merge, the write), as the
// bytes of K and V that it could have streamed meanwhile.  96 caches of 1 to 3,000 tokens (8/8 heads of 64): 24.2 us
// with 64 KB, 21.5 with 192; 32 of 50 to 4,000 (16/2 heads): 13.3 with 96 KB, 12.2 with 192; with 384 KB small
// batches lose (64 of 1 to 500: 10.1 -> 11.4 us).
constexpr int kSegBytes = 196608;

struct PdPlan {
  PoolView pool;
  const int32_t *seqlens;
  const uint8_t *q;
  int64_t q_stride;                  // bytes between sequences
  int32_t hq, group;                 // query heads, per KV head
  int32_t heads_cta, groups;         // KV heads of a CTA, head groups
  int32_t wph_log, rg_log;           // log2 of the rings per head, and of the groups of 8 query rows
  int32_t boxes;                     // TMA boxes of a tile: of 16 or 32 tokens, or (NG 1) of 8; 0: its rows are copied by the lanes
  int32_t max_rows;
  int32_t wide_lengths;              // seqlens can be read four at a time
  int32_t seg_cost;                  // what a segment costs beyond its tiles, in tiles
  float scale2;                      // scale * log2(e)
  float grow;                        // kGrow in units of q.k
  void *out;
  int32_t out_fp32;
  float *lse;
  int4 *info;                        // [grid]: (sequence, head group, parts, first slot) of a cut segment that starts here
  float2 *ml;                        // [slot][head][row group][8]
  float *part;                       // [slot][head][row group][D / 16][128]
  DeviceError *err;
};

// The 16-bit types of K, V and P.  A probability is exp2(logit - reference); the reference is kShift below the row's
// maximum when it was set, and set anew only when the maximum has grown by more than kGrow (log2 units), so that most
// tiles need one vote instead of a reduction and rescaled accumulators.  bf16 has the range of fp32.  fp16 ends at
// 2^16 and loses what lies below 2^-25: with probabilities of up to 2^15 (kShift + kGrow) the tail is kept down to
// 2^-36 of the maximum; up to 1, a hundred thousand keys 17 below the maximum would be lost, 2^-8 of the sum.
// kParts: a probability enters the value product as a sum of that many 16-bit numbers, so that it keeps the 24 bits that
// the row's sum is made of: three of bf16 (8 bits each: what is left out is below 2^-26), two of fp16 (11 bits and a sign
// each: 2^-23).  The third bf16 number costs 0.2 us of 50 or 34 (ten minutes, 16 caches), 0.5 of 31 with 16 query heads per
// KV head and 3.7 of 38 with 32, where a warp's chain of instructions is the bound (0.28 issued per clock and scheduler; the
// same call in fp16: 34.5); without it fp32 outputs were 2e-6 off.
template <class T>
struct Half16;
template <>
struct Half16<__nv_bfloat16> {
  static constexpr float kGrow = 8.f, kShift = 0.f;
  static constexpr int kParts = 3;
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&v);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <>
struct Half16<__half> {
  static constexpr float kGrow = 4.f, kShift = 11.f;
  static constexpr int kParts = 2;
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&v);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<__half2 *>(&w)); }
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
// Transposes an 8 x 8 matrix of 16-bit elements held by the warp (lane: row lane / 4, columns 2 (lane % 4) and + 1).
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int32_t c1, int32_t c2,
                                            int32_t c3, int32_t c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], "
      "[%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}

__device__ __forceinline__ void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

// The wph warps of head and row group `team`.
__device__ __forceinline__ void team_barrier(int team, int wph) {
  asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(32 * wph) : "memory");
}

__device__ __forceinline__ int clamped_length(const PdPlan &P, int b, bool report) {
  const int n = __ldg(P.seqlens + b);
  const int c = min(max(n, 0), P.max_rows);
  if (report && c != n) raise_device_error(P.err, APACK_EDEVICE, 81, b, n);
  return c;
}
// n / d in 32 bits where they do (a 64-bit division takes some 100 instructions).
__device__ __forceinline__ int quotient(int64_t n, int d) {
  return static_cast<int>((n >> 32) == 0 ? static_cast<uint32_t>(n) / static_cast<uint32_t>(d) : n / d);
}
template <int TILE>
__device__ __forceinline__ int tiles_of(int len) {
  return len / TILE + (len % TILE != 0);
}

// The clamped lengths of kWindow sequences from b0 on, in a warp's shared memory: a walk from sequence to sequence
// then costs no trip to L2 per step (a share of four short sequences reached its first loads 6 us late without).
constexpr int kWindow = 64;
struct LengthWindow {
  int b0;
  const int *v;
  __device__ __forceinline__ int at(const PdPlan &P, int b) const {
    return b - b0 < kWindow ? v[b - b0] : clamped_length(P, b, false);
  }
};

// A walk over the (sequence, head group) segments of a CTA's share, `n` units of the work list; positions are counted
// from the share's first unit.  A segment takes up seg_cost + nt units, the tiles behind the cost.
template <int TILE>
struct Walk {
  int b, g, len, nt;     // segment, its sequence's length and tiles
  int ts, te;            // the share's tiles of it
  int first;             // position of its first tile (below 0 where an earlier share starts it)
  __device__ __forceinline__ void span(int n) {
    ts = min(max(-first, 0), nt);
    te = min(max(n - first, 0), nt);
  }
  // The next segment with a tile in the share.
  __device__ __forceinline__ bool next(const PdPlan &P, const LengthWindow &lens, int n) {
    do {
      first += nt + P.seg_cost;
      if (first >= n) return false;
      if (++g >= P.groups) {
        g = 0;
        do {
          len = lens.at(P, ++b);
        } while (len == 0);
        nt = tiles_of<TILE>(len);
      }
      span(n);
    } while (ts >= te);
    return true;
  }
};

// NG: groups of 8 query rows of a warp, which share its reads of K and V from shared memory.  SHARED: a ring is read by 2
// warps; as templates, because the one-warp rings of most models are 1.5 % faster without the other case's registers and
// branches.  60,000 tokens of 4 KV heads of 128, bf16, 16-token pages: 28.5 us with 7 query heads each, 31.1 with 16, 38.1
// with 24 or 32.  With two 16-bit numbers per probability the last took 34.3, and 46.6 with 4 warps of one group per ring
// (every warp reads the whole tile, 4 times the traffic that fills it); 16 query heads as 2 warps of one group each the
// same as here, 29.6 against 30.2 on 64 caches of 100 to 2,000 tokens: one variant less.
template <class T, int D, int NG, bool SHARED>
__global__ void __launch_bounds__(kThreads, 1)
    paged_chunk_kernel(const __grid_constant__ PdPlan P, const __grid_constant__ CUtensorMap kmap,
                       const __grid_constant__ CUtensorMap vmap) {
  constexpr int KS = D / 16;                          // k-steps of S, m-tiles of O^T
  constexpr int kTile = tile_tokens(D), KM = kTile / 16;   // m-tiles of S, k-steps of O^T
  constexpr int kHalf = kTile * D * 2;                // bytes of a stage's K (and V)
  static_assert(2 * kHalf == kStageBytes, "8 KB stages");
  constexpr int kBlk = kTile * 128;                   // bytes of one 64-feature block of a stage
  extern __shared__ __align__(1024) uint8_t smem[];
  float *merge = reinterpret_cast<float *>(smem + kStageBytesCta);
  float2 *stat = reinterpret_cast<float2 *>(merge + kMergeFloats);        // [warp][8]
  uint64_t *bars = reinterpret_cast<uint64_t *>(stat + kWarps * 8);       // full, then empty, of all stages
  int *window = reinterpret_cast<int *>(bars + 2 * kMaxStages);           // [warp][kWindow]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // warp = (ring of the head, reader of the ring, head)
  constexpr int readers = SHARED ? 2 : 1;
  const int wph = 1 << P.wph_log;
  const int hw = warp % P.heads_cta, rd = SHARED ? (warp / P.heads_cta) & 1 : 0, sub = warp / P.heads_cta / readers;
  const int ring_id = sub * P.heads_cta + hw, stages = kMaxStages / kWarps * readers;
  uint64_t *full = bars + ring_id * stages, *empty = full + kMaxStages;
  const uint32_t ring = smem_u32(smem) + ring_id * stages * kStageBytes;
  if (sub < wph && rd == 0 && lane == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(&full[i], P.boxes ? 1 : 32);
      mbar_init(&empty[i], readers);
    }
    fence_mbar_init();
  }
  if (threadIdx.x == 32 && P.boxes) {
    tma_prefetch_desc(&kmap);
    tma_prefetch_desc(&vmap);
  }
  // lengths and page table on their way to L2 while the launch before this one ends (what that launch may still
  // write of them is read from L2 all the same)
  {
    const int line = blockIdx.x * kThreads + threadIdx.x, row_lines = (P.pool.max_pages + 31) / 32;
    if (line * 32 < P.pool.num_seqs) prefetch_l2(P.seqlens + line * 32);
    const int b = line / row_lines;
    if (b < P.pool.num_seqs) prefetch_l2(P.pool.table + b * P.pool.table_stride + (line - b * row_lines) * 32);
  }
  if (SHARED)
    __syncthreads();                                  // the ring's barriers, for its other warps
  else
    __syncwarp();
  pdl_wait_and_release();

  // ---- this CTA's share (every warp by itself: no barrier before the first load).  The list starts behind the first
  // segment's cost, which every CTA pays one of anyway.
  const int B = P.pool.num_seqs, grid = gridDim.x, cta = blockIdx.x, cost = P.seg_cost;
  const bool report = warp == 0 && cta == 0;
  if (threadIdx.x == 0) P.info[cta] = make_int4(0, 0, 0, 0);
  auto units64 = [&](int len) { return len > 0 ? static_cast<int64_t>(tiles_of<kTile>(len) + cost) * P.groups : 0; };
  auto units = [&](int len) { return static_cast<int>(units64(len)); };
  auto sum = [&](int64_t v) {                          // over the lanes
    const uint32_t low = static_cast<uint32_t>(v) & 0xFFFFFu, high = static_cast<uint32_t>(v >> 20);
    return (static_cast<int64_t>(__reduce_add_sync(0xffffffffu, high)) << 20) + __reduce_add_sync(0xffffffffu, low);
  };
  auto scan = [&](int v) {                             // inclusive, over the lanes
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += y;
    }
    return v;
  };
  LengthWindow lens;
  lens.v = window + warp * kWindow;
  int mine = 0, n0 = 0, n1 = 0;
  int64_t total = 0;
  const int per = ((B + 31) / 32 + 3) & ~3;            // consecutive sequences of a lane
  if (B <= kWindow) {
    // the window holds them all; lane and lane + 32 are its sequences
    if (lane < B) n0 = clamped_length(P, lane, report);
    if (lane + 32 < B) n1 = clamped_length(P, lane + 32, report);
    window[warp * kWindow + lane] = n0;
    window[warp * kWindow + lane + 32] = n1;
    lens.b0 = 0;
    mine = units(n0);
    total = units64(n0) + units64(n1);
  } else {
#pragma unroll 4
    for (int i = 0; i < per; i += 4) {
      const int b = lane * per + i;
      int len[4] = {0, 0, 0, 0};
      if (P.wide_lengths && b + 4 <= B) {
        const int4 v = __ldg(reinterpret_cast<const int4 *>(P.seqlens + b));
        len[0] = v.x;
        len[1] = v.y;
        len[2] = v.z;
        len[3] = v.w;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (b + k < B) len[k] = __ldg(P.seqlens + b + k);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = min(max(len[k], 0), P.max_rows);
        if (report && c != len[k]) raise_device_error(P.err, APACK_EDEVICE, 81, b + k, len[k]);
        total += units64(c);
      }
    }
    mine = static_cast<int>(total);
  }
  total = sum(total) - cost;
  // the list is counted in 32 bits from here on
  if (total > kMaxUnits) {
    if (report && lane == 0) raise_device_error(P.err, APACK_EDEVICE, 85);
    total = 0;
  }
  const int W = static_cast<int>(total);
  // A share has a tile per warp at least, or two where that leaves more parts than a warp of the merge loads at once and
  // a half (473 tokens: 7.8 us with one tile each, 8.3 with two; 1,000 tokens: 9.3 and 8.9).
  const int narrow = W >> P.wph_log;
  const int C = min(grid, max(narrow <= 16 ? narrow : narrow / 2, 1));
  if (W <= 0 || cta >= C || sub >= wph) return;
  const int u0 = cost + quotient(static_cast<int64_t>(W) * cta, C);
  const int n = cost + quotient(static_cast<int64_t>(W) * (cta + 1), C) - u0;
  Walk<kTile> seg;
  {
    int off = u0, b = 0, incl = scan(mine);
    const int half = __shfl_sync(0xffffffffu, incl, 31);
    if (B <= kWindow && u0 >= half) {                  // among the second 32
      mine = units(n1);
      incl = scan(mine) + half;
      b = 32;
    }
    const int src = __ffs(__ballot_sync(0xffffffffu, u0 >= incl - mine && u0 < incl)) - 1;
    off -= __shfl_sync(0xffffffffu, incl - mine, src);
    if (B <= kWindow) {
      b += src;
    } else {
      // among the lane's sequences, 32 at a time; they and the 32 behind them become the window
      for (b = src * per;; b += 32) {
        const int len = b + lane < B ? clamped_length(P, b + lane, false) : 0;
        mine = units(len);
        incl = scan(mine);
        const unsigned hit = __ballot_sync(0xffffffffu, off < incl);
        if (hit) {
          const int at = __ffs(hit) - 1;
          off -= __shfl_sync(0xffffffffu, incl - mine, at);
          lens.b0 = b;
          window[warp * kWindow + lane] = len;
          window[warp * kWindow + lane + 32] = b + lane + 32 < B ? clamped_length(P, b + lane + 32, false) : 0;
          b += at;
          break;
        }
        off -= __shfl_sync(0xffffffffu, incl, 31);
      }
    }
    __syncwarp();
    seg.b = b;
    seg.len = lens.at(P, b);
    seg.nt = tiles_of<kTile>(seg.len);
    seg.g = P.groups == 1 ? 0 : off / (seg.nt + cost);
    seg.first = cost - (off - seg.g * (seg.nt + cost));
    seg.span(n);
    if (seg.ts >= seg.te && !seg.next(P, lens, n)) return;      // the share holds no tile (for all warps alike)
  }

  // ---- producer (the ring's first warp): a queue of its next 32 tiles, one per lane; the lane of a tile issues its
  // loads
  Walk<kTile> head_w = seg;                                  // of the first tile behind the queue
  int head_t = seg.ts + sub;
  bool head_ok = true;
  while (head_ok && head_t >= head_w.te) {
    head_ok = head_w.next(P, lens, n);
    head_t = head_w.ts + sub;
  }
  int32_t q_page[KM], q_head = 0, q_b = 0, q_t = 0, q_len = 0;
  uint32_t q_in = 0;
  int queued = 0, issued = 0, used = 0;
  int issue_slot = 0, use_slot = 0, free_slot = 0;
  uint32_t use_phase = 0, free_phase = 0;
  auto refill = [&] {
    Walk<kTile> w = head_w;
    int t = head_t, skip = lane;
    bool ok = head_ok;
    while (ok) {
      const int here = t < w.te ? (w.te - t + wph - 1) >> P.wph_log : 0;
      if (skip < here) {
        t += skip << P.wph_log;
        break;
      }
      skip -= here;
      ok = w.next(P, lens, n);
      t = w.ts + sub;
    }
    if (ok) {
      q_b = w.b;
      q_t = t;
      q_len = w.len;
      q_head = w.g * P.heads_cta + hw;
      if (P.boxes && P.boxes <= KM) {
        const uint32_t p = P.pool.page_tokens.div(t * kTile);
        const int32_t *row = P.pool.table + w.b * P.pool.table_stride + p;
        q_in = t * kTile - p * P.pool.page_tokens.d;
        q_page[0] = __ldg(row);
        // pages of 16 (48, ...) tokens: the tile's second half may be the next page's
        if (KM > 1) q_page[KM - 1] = P.boxes > 1 && t * kTile + 16 < w.len && q_in + 16 >= P.pool.page_tokens.d ? __ldg(row + 1) : q_page[0];
      }
    }
    queued += __popc(__ballot_sync(0xffffffffu, ok));
    head_ok = __shfl_sync(0xffffffffu, static_cast<int>(ok), 31);
    head_w.b = __shfl_sync(0xffffffffu, w.b, 31);
    head_w.g = __shfl_sync(0xffffffffu, w.g, 31);
    head_w.len = __shfl_sync(0xffffffffu, w.len, 31);
    head_w.nt = __shfl_sync(0xffffffffu, w.nt, 31);
    head_w.first = __shfl_sync(0xffffffffu, w.first, 31);
    head_w.span(n);
    head_t = __shfl_sync(0xffffffffu, t, 31) + wph;
  };
  // One TMA box pair; a page outside the pool reads as zeros (the map ends there).
  auto load_box = [&](int slot, int32_t page, uint32_t in_page, int head, int b, int block, uint32_t offset) {
    if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(P.pool.num_pages)) {
      raise_device_error(P.err, APACK_EDEVICE, 82, b, page);
      page = P.pool.num_pages;
    }
    const uint32_t dst = ring + slot * kStageBytes + offset;
    tma_load_5d(dst, &kmap, &full[slot], in_page, block, head, page);
    tma_load_5d(dst + kHalf, &vmap, &full[slot], in_page, block, head, page);
  };
  // Tile number `issued` of the warp, if there is one.
  auto issue = [&] {
    if (issued == queued) {
      if (!head_ok) return;
      refill();
      if (issued == queued) return;
    }
    const int slot = issue_slot, owner = issued & 31;
    issue_slot = slot + 1 == stages ? 0 : slot + 1;
    if (P.boxes && P.boxes <= KM) {
      if (lane == owner) {
        const bool second = KM > 1 && P.boxes > 1 && q_t * kTile + 16 < q_len;
        mbar_arrive_expect_tx(&full[slot], KM > 1 && P.boxes > 1 && !second ? kHalf : 2 * kHalf);
        load_box(slot, q_page[0], q_in, q_head, q_b, 0, 0);
        if (second) load_box(slot, q_page[KM - 1], q_in + 16 >= P.pool.page_tokens.d ? 0 : q_in + 16, q_head, q_b, 0, 2048);
      }
      ++issued;
      return;
    }
    const int t = __shfl_sync(0xffffffffu, q_t, owner), b = __shfl_sync(0xffffffffu, q_b, owner);
    const int head = __shfl_sync(0xffffffffu, q_head, owner), len = __shfl_sync(0xffffffffu, q_len, owner);
    const int rows = min(kTile, len - t * kTile);
    if (NG == 1 && P.boxes) {
      // Pages of a multiple of 8 tokens: a box of 8 per lane (and 64-feature block), those that hold a row of the sequence.
      // Against copies by the lanes, 60,000 tokens of 4 heads of 128 in pages of 24 or 1,000: 28.9 and 29.7 us, of 8 29.5 and
      // 30.0; 120,000 of heads of 64: 28.6 and 29.3, in pages of 8 31.0 and 30.4 (96 short caches 22.6 and 23.9).
      // Not with two groups of rows per warp: 16-token pages would lose 1.5 to 2 % by the registers (31.1 -> 31.8, 38.3 ->
      // 39.1 us with 16 and 32 query heads per KV head), pages of 8 gain up to 6 % (46.5 -> 43.7).
      const int nbox = (rows + 7) / 8;
      if (lane == 0) mbar_arrive_expect_tx(&full[slot], nbox * 8 * D * 4);
      __syncwarp();
      if (lane < nbox) {
        const uint32_t row = t * kTile + lane * 8, p = P.pool.page_tokens.div(row);
        const int32_t page = __ldg(P.pool.table + b * P.pool.table_stride + p);
#pragma unroll
        for (int blk = 0; blk < D / 64; ++blk)
          load_box(slot, page, row - p * P.pool.page_tokens.d, head, b, blk, blk * kBlk + lane * 1024);
      }
    } else {
      // Other pages: rows copied by the lanes, 16 bytes at a time, to where a box would put them.  Smaller boxes are bound by
      // their number: 60,000 tokens of 4 heads of 128 in pages of 4 31.4 against 30.5 us, of 1 50.5 against 31.6.
      int64_t off = -1;
      if (lane < rows) {
        const int row = t * kTile + lane;
        const int32_t page = P.pool.page_of(b, row);
        off = P.pool.offset_in(page, row);
        if (off < 0) raise_device_error(P.err, APACK_EDEVICE, 82, b, page);
        off += off < 0 ? 0 : head * P.pool.head_stride;
      }
      constexpr int kChunks = D / 8, kAtOnce = 32 / kChunks;
      const int ch = lane % kChunks;
#pragma unroll
      for (int i = 0; i < kTile / kAtOnce; ++i) {
        const int r = i * kAtOnce + lane / kChunks;
        const int64_t o = __shfl_sync(0xffffffffu, off, r);
        if (r < rows) {
          const uint32_t dst = ring + slot * kStageBytes + (ch >> 3) * kBlk + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
          const int64_t src = (o < 0 ? 0 : o) + ch * 16;
          cp_async_16_or_zero(dst, P.pool.k + src, o >= 0);
          cp_async_16_or_zero(dst + kHalf, P.pool.v + src, o >= 0);
        }
      }
      cp_async_arrive(&full[slot]);
    }
    ++issued;
  };
  if (rd == 0)
    for (int i = 0; i < stages; ++i) issue();

  // ---- consumer
  const int t4 = lane & 3, g8 = lane >> 2;
  // ldmatrix rows of this lane: K fragments (keys x features) and, transposed, V fragments (features x keys)
  const uint32_t krow = (lane & 7) + ((lane >> 3) & 1) * 8, kchunk = lane >> 4;
  const uint32_t vrow = (lane & 7) + (lane >> 4) * 8, vchunk = (lane >> 3) & 1;
  bool dead = false;                                  // a wait gave up: no more loads are issued or waited for
  int first_seg = 1;
  // query fragments; the next segment's are loaded during this one
  using QFrag = uint32_t[NG][KS][2];
  auto load_q = [&](const Walk<kTile> &w, QFrag &f) {
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      const int r = (rd * NG + ng) * 8 + g8;
      const uint8_t *qb = P.q + w.b * P.q_stride + (static_cast<int64_t>(w.g * P.heads_cta + hw) * P.group + r) * D * 2;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          f[ng][ks][e] = r < P.group ? __ldg(reinterpret_cast<const uint32_t *>(qb + (ks * 16 + e * 8 + t4 * 2) * 2)) : 0u;
    }
  };
  QFrag qf, q_next;
  load_q(seg, qf);
  for (;;) {
    Walk<kTile> after = seg;
    const bool go_on = after.next(P, lens, n);
    if (go_on) load_q(after, q_next);
    const int head = seg.g * P.heads_cta + hw;
    // m: reference, log2 units; limit: of q.k, beyond which it grows; l and m of query rows 2 t4 and 2 t4 + 1
    // (of each group of 8)
    float o[NG][KS][4], m[NG][2], l[NG][2], limit[NG][2];
#pragma unroll
    for (int ng = 0; ng < NG; ++ng) {
      m[ng][0] = m[ng][1] = limit[ng][0] = limit[ng][1] = -INFINITY;
      l[ng][0] = l[ng][1] = 0.f;
#pragma unroll
      for (int i = 0; i < KS; ++i) o[ng][i][0] = o[ng][i][1] = o[ng][i][2] = o[ng][i][3] = 0.f;
    }
    for (int t = seg.ts + sub; t < seg.te && !dead; t += wph) {
      if (!__all_sync(0xffffffffu, mbar_wait(&full[use_slot], use_phase, kWaitLimitNs))) {
        if (lane == 0) raise_device_error(P.err, APACK_ETIMEOUT, 83, cta, warp);
        dead = true;
        break;
      }
      ++used;
      const int slot = use_slot;
      const uint32_t kb = ring + slot * kStageBytes, vb = kb + kHalf;
      if (++use_slot == stages) {
        use_slot = 0;
        use_phase ^= 1;
      }
      const int valid = seg.len - t * kTile;          // rows of the tile that belong to the sequence
      if (valid < kTile) {
        // what lies behind the last row takes no part: its logits become -infinity below, and its values
        // zeros here (0 times a stale infinity would be NaN; the warps of a ring all write the same zeros)
        for (int i = lane; i < (kTile - valid) * (D / 8); i += 32) {
          const int row = valid + i / (D / 8), ch = i % (D / 8);
          const uint32_t a = vb + (ch >> 3) * kBlk + row * 128 + (ch & 7) * 16;
          asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a), "r"(0) : "memory");
        }
        fence_proxy_async_smem();                     // before TMA writes the slot again
        __syncwarp();
      }
      float s[NG][KM][4];
#pragma unroll
      for (int ng = 0; ng < NG; ++ng)
#pragma unroll
        for (int km = 0; km < KM; ++km) s[ng][km][0] = s[ng][km][1] = s[ng][km][2] = s[ng][km][3] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int km = 0; km < KM; ++km) {
          uint32_t a[4];
          const uint32_t ch = ks * 2 + kchunk;
          ldmatrix4(kb + (ch >> 3) * kBlk + (km * 16 + krow) * 128 + (((ch & 7) ^ (krow & 7)) << 4), a);
#pragma unroll
          for (int ng = 0; ng < NG; ++ng) Half16<T>::mma(s[ng][km], a, qf[ng][ks][0], qf[ng][ks][1]);
        }
      // lane: keys g8 and g8 + 8 of 16, query rows 2 t4 and 2 t4 + 1
      if (valid < kTile)
#pragma unroll
        for (int km = 0; km < KM; ++km)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (km * 16 + g8 + (i >> 1) * 8 >= valid)
#pragma unroll
              for (int ng = 0; ng < NG; ++ng) s[ng][km][i] = -INFINITY;
      // (a NaN logit leaves the maximum to the others, and its probability NaN)
      float top[NG][2];
      bool grows = false;
#pragma unroll
      for (int ng = 0; ng < NG; ++ng)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          top[ng][e] = fmaxf(s[ng][0][e], s[ng][0][e + 2]);
          if (KM > 1) top[ng][e] = fmaxf(top[ng][e], fmaxf(s[ng][KM - 1][e], s[ng][KM - 1][e + 2]));
          grows |= !(top[ng][e] <= limit[ng][e]);
        }
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int ng = 0; ng < NG; ++ng)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = top[ng][e];
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            const float mn = fmaxf(m[ng][e], fmaf(x, P.scale2, -Half16<T>::kShift));
            const float f = mn == -INFINITY ? 1.f : ex2_approx(m[ng][e] - mn);
            m[ng][e] = mn;
            limit[ng][e] = fmaxf(limit[ng][e], x + P.grow);
            l[ng][e] *= f;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
              o[ng][i][e] *= f;
              o[ng][i][e + 2] *= f;
            }
          }
      }
      // P as the sum of kParts 16-bit numbers, each the rounding of what those before it leave, transposed into B fragments
      constexpr int kParts = Half16<T>::kParts;
      uint32_t pf[NG][KM][kParts][2];
#pragma unroll
      for (int ng = 0; ng < NG; ++ng)
#pragma unroll
        for (int km = 0; km < KM; ++km) {
          float p[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = ex2_approx(fmaf(s[ng][km][i], P.scale2, -m[ng][i & 1]));
          l[ng][0] += p[0] + p[2];
          l[ng][1] += p[1] + p[3];
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
              const uint32_t h = Half16<T>::pack(p[2 * e], p[2 * e + 1]);
              pf[ng][km][part][e] = transpose8x8(h);
              const float2 hf = Half16<T>::unpack(h);
              p[2 * e] -= hf.x;
              p[2 * e + 1] -= hf.y;
            }
        }
#pragma unroll
      for (int km = 0; km < KM; ++km)
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          uint32_t a[4];
          const uint32_t ch = i * 2 + vchunk;
          ldmatrix4_trans(vb + (ch >> 3) * kBlk + (km * 16 + vrow) * 128 + (((ch & 7) ^ (vrow & 7)) << 4), a);
#pragma unroll
          for (int ng = 0; ng < NG; ++ng)
#pragma unroll
            for (int part = 0; part < kParts; ++part) Half16<T>::mma(o[ng][i], a, pf[ng][km][part][0], pf[ng][km][part][1]);
        }
      __syncwarp();                                   // every lane has read the stage
      if (!SHARED) {
        issue();
      } else {
        if (lane == 0) mbar_arrive(&empty[slot]);
        // the stage before this one, which the ring's other warps have most likely left by now
        if (rd == 0 && used >= 2 && (issued < queued || head_ok)) {
          if (!__all_sync(0xffffffffu, mbar_wait(&empty[free_slot], free_phase, kWaitLimitNs))) {
            if (lane == 0) raise_device_error(P.err, APACK_ETIMEOUT, 84, cta, warp);
            dead = true;
            break;
          }
          if (++free_slot == stages) {
            free_slot = 0;
            free_phase ^= 1;
          }
          issue();
        }
      }
    }

    // ---- end of the segment: the warps of each head and reader number merge, one group of 8 query rows after the other
    const bool whole = seg.ts == 0 && seg.te == seg.nt;
    auto merge_and_write = [&](float(&o)[KS][4], float(&m)[2], float(&l)[2], int rg) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[e];
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        x += __shfl_xor_sync(0xffffffffu, x, 16);
        l[e] = x;
      }
      // Pairs of them exchange halves of their m-tiles until each holds its own of the sums, o[0] on from m-tile `base`
      const int hr = rd * P.heads_cta + hw, team = P.heads_cta * readers;   // warp = sub * team + hr
      int base = 0;
      bool mine_to_write = true;
      auto halve = [&](auto half, int bit) {
        constexpr int H = decltype(half)::value;        // 0: one m-tile each, which the lower of the two keeps
        constexpr int M = H ? H : 1;
        const bool upper = sub & bit;
        const int other = upper ? warp - bit * team : warp + bit * team;   // (team is no power of two for 3 heads)
        float4 *give = reinterpret_cast<float4 *>(merge) + warp * (KS / 2) * 32 + lane;
        const float4 *take = reinterpret_cast<float4 *>(merge) + other * (KS / 2) * 32 + lane;
        team_barrier(hr, wph);                          // the last exchange's halves have been read
#pragma unroll
        for (int i = 0; i < M; ++i) {
          float(&x)[4] = o[i], (&y)[4] = o[i + H];
          give[i * 32] = upper && H ? make_float4(x[0], x[1], x[2], x[3]) : make_float4(y[0], y[1], y[2], y[3]);
          if (H)
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = upper ? y[k] : x[k];
        }
        if (g8 == 0) {
          stat[warp * 8 + t4 * 2] = make_float2(m[0], l[0]);
          stat[warp * 8 + t4 * 2 + 1] = make_float2(m[1], l[1]);
        }
        team_barrier(hr, wph);
        float a[2], b[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 x = stat[other * 8 + t4 * 2 + e];
          const float top = fmaxf(m[e], x.x);
          a[e] = m[e] == top ? 1.f : ex2_approx(m[e] - top);
          b[e] = x.x == top ? 1.f : ex2_approx(x.x - top);
          l[e] = l[e] * a[e] + x.y * b[e];
          m[e] = top;
        }
#pragma unroll
        for (int i = 0; i < M; ++i) {
          const float4 x = take[i * 32];
          o[i][0] = o[i][0] * a[0] + x.x * b[0];
          o[i][1] = o[i][1] * a[1] + x.y * b[1];
          o[i][2] = o[i][2] * a[0] + x.z * b[0];
          o[i][3] = o[i][3] * a[1] + x.w * b[1];
        }
        if (upper) base += H;
        if (H == 0) mine_to_write = !upper;
      };
      auto write = [&](auto count) {
        constexpr int N = decltype(count)::value;
        if (whole) {                                    // the whole segment: its output
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = rg * 8 + t4 * 2 + e;
            if (r >= P.group) continue;
            const int64_t row = static_cast<int64_t>(seg.b) * P.hq + head * P.group + r;
            const float inv = l[e] == 0.f ? 0.f : 1.f / l[e];
            if (P.lse && g8 == 0 && base == 0) P.lse[row] = (m[e] + log2f(l[e])) * 0.6931471805599453f;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const int64_t at = row * D + (base + i) * 16 + h * 8 + g8;
                const float x = o[i][e + 2 * h] * inv;
                if (P.out_fp32)
                  static_cast<float *>(P.out)[at] = x;
                else
                  static_cast<T *>(P.out)[at] = static_cast<T>(x);
              }
          }
        } else {
          const int slot = 2 * cta + (first_seg ? 0 : 1);
          const int64_t at = ((static_cast<int64_t>(slot) * P.heads_cta + hw) << P.rg_log) + rg;
          if (g8 == 0 && base == 0) {
            P.ml[at * 8 + t4 * 2] = make_float2(m[0], l[0]);
            P.ml[at * 8 + t4 * 2 + 1] = make_float2(m[1], l[1]);
          }
          float4 *pp = reinterpret_cast<float4 *>(P.part) + (at * KS + base) * 32 + lane;
#pragma unroll
          for (int i = 0; i < N; ++i) pp[i * 32] = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
        }
      };
      if (wph == 1) {
        write(std::integral_constant<int, KS>());
      } else {
        halve(std::integral_constant<int, KS / 2>(), wph / 2);
        if (wph == 2) {
          write(std::integral_constant<int, KS / 2>());
        } else {
          halve(std::integral_constant<int, KS / 4>(), wph / 4);
          if (wph == 8) halve(std::integral_constant<int, KS / 8>(), 1);
          // (D = 64: one m-tile each from here on)
          if (wph == 4)
            write(std::integral_constant<int, KS / 4>());
          else if (mine_to_write)
            write(std::integral_constant<int, KS / 8 ? KS / 8 : 1>());
        }
      }
    };
#pragma unroll
    for (int ng = 0; ng < NG; ++ng)
      if ((rd * NG + ng) * 8 < P.group) merge_and_write(o[ng], m[ng], l[ng], rd * NG + ng);
    if (threadIdx.x == 0 && seg.ts == 0 && !whole) {
      // this share starts the segment; the one that holds its last tile ends it
      const int64_t end = u0 - cost + seg.first + seg.nt;      // unit behind the last tile, without the list's first cost
      const int c_end = quotient(end * C + W - 1, W) - 1;
      P.info[cta] = make_int4(seg.b, seg.g, c_end - cta + 1, 2 * cta + (first_seg ? 0 : 1));
    }
    first_seg = 0;
    if (!go_on) break;
    seg = after;
#pragma unroll
    for (int ng = 0; ng < NG; ++ng)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ng][ks][0] = q_next[ng][ks][0];
        qf[ng][ks][1] = q_next[ng][ks][1];
      }
  }
  if (dead)   // loads of the stages that were issued and not used may still be in flight
    for (int k = used; k < issued; ++k) mbar_wait(&full[k % stages], (k / stages) & 1u, kWaitLimitNs / 4);
}

// Merges the parts of the cut segments.  A unit is (segment, head, 8 query rows, 16 features).  Every CTA lists the
// shares that start a cut segment (info), then the units of segments of many parts are merged by a CTA each, a run
// of the parts per warp, and those of few parts by a warp each.  Bound by latency: the launch boundary (1.0 to 1.7 us),
// the list, one round of loads from L2, the write: 3 us of a call of 473 tokens, 5 us of one of ten minutes.  All of a
// segment's parts by the last share to arrive, inside the chunk kernel, took 13.5 us against 9.3 (473 tokens).
constexpr int kCombineWarps = 16;
constexpr int kCombineBatch = 10;      // parts whose loads a warp has in flight
constexpr int kCombineFew = 30;        // parts that one warp merges
constexpr int kMaxGrid = 512;

// (max, sum, o) of two query rows (2 t4 and + 1) and two features (g8 and + 8), in log2 units.
struct PartState {
  float m0, m1, l0, l1;
  float4 o;                            // row 0 feature g8, row 1 g8, row 0 g8 + 8, row 1 g8 + 8
};
// Merges N parts into a: maxima first, then the factors, which do not wait for one another.  Equal maxima (both
// -infinity among them) give the factor 1.
template <int N>
__device__ __forceinline__ void merge_parts(PartState &a, const float4 (&ml)[N], const float4 (&x)[N]) {
  float n0 = a.m0, n1 = a.m1;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    n0 = fmaxf(n0, ml[k].x);
    n1 = fmaxf(n1, ml[k].z);
  }
  const float a0 = a.m0 == n0 ? 1.f : ex2_approx(a.m0 - n0), a1 = a.m1 == n1 ? 1.f : ex2_approx(a.m1 - n1);
  a.l0 *= a0;
  a.l1 *= a1;
  a.o = make_float4(a.o.x * a0, a.o.y * a1, a.o.z * a0, a.o.w * a1);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float b0 = ml[k].x == n0 ? 1.f : ex2_approx(ml[k].x - n0), b1 = ml[k].z == n1 ? 1.f : ex2_approx(ml[k].z - n1);
    a.l0 += ml[k].y * b0;
    a.l1 += ml[k].w * b1;
    a.o.x += x[k].x * b0;
    a.o.y += x[k].y * b1;
    a.o.z += x[k].z * b0;
    a.o.w += x[k].w * b1;
  }
  a.m0 = n0;
  a.m1 = n1;
}

template <class T, int D>
__device__ __forceinline__ PartState merge_run(const PdPlan &P, const int4 &inf, int hn, int i, int p0, int p1, int lane) {
  PartState a = {-INFINITY, -INFINITY, 0.f, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
  for (int p = p0; p < p1; p += kCombineBatch) {
    float4 ml[kCombineBatch], x[kCombineBatch];
#pragma unroll
    for (int k = 0; k < kCombineBatch; ++k) {
      // the first part lies where its share put it, the others are their shares' first
      const int q = min(p + k, p1 - 1);
      const int slot = q == 0 ? inf.w : 2 * ((inf.w >> 1) + q);
      const int64_t at = (static_cast<int64_t>(slot) * P.heads_cta << P.rg_log) + hn;
      ml[k] = *reinterpret_cast<const float4 *>(P.ml + at * 8 + (lane & 3) * 2);
      x[k] = reinterpret_cast<const float4 *>(P.part)[(at * (D / 16) + i) * 32 + lane];
    }
#pragma unroll
    for (int k = 0; k < kCombineBatch; ++k)
      if (p + k >= p1) {                        // behind the run: nothing
        ml[k] = make_float4(-INFINITY, 0.f, -INFINITY, 0.f);
        x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    merge_parts(a, ml, x);
  }
  return a;
}

template <class T, int D>
__device__ __forceinline__ void write_unit(const PdPlan &P, const int4 &inf, int hn, int i, const PartState &a, int lane) {
  const int t4 = lane & 3, g8 = lane >> 2;
  const int head = inf.y * P.heads_cta + (hn >> P.rg_log);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = (hn & ((1 << P.rg_log) - 1)) * 8 + t4 * 2 + e;
    if (r >= P.group) continue;
    const int64_t row = static_cast<int64_t>(inf.x) * P.hq + head * P.group + r;
    const float L = e ? a.l1 : a.l0, inv = L == 0.f ? 0.f : 1.f / L;
    if (P.lse && i == 0 && g8 == 0) P.lse[row] = ((e ? a.m1 : a.m0) + log2f(L)) * 0.6931471805599453f;
    const float x0 = (e ? a.o.y : a.o.x) * inv, x1 = (e ? a.o.w : a.o.z) * inv;
    const int64_t at = row * D + i * 16 + g8;
    if (P.out_fp32) {
      static_cast<float *>(P.out)[at] = x0;
      static_cast<float *>(P.out)[at + 8] = x1;
    } else {
      static_cast<T *>(P.out)[at] = static_cast<T>(x0);
      static_cast<T *>(P.out)[at + 8] = static_cast<T>(x1);
    }
  }
}

template <class T, int D>
__global__ void __launch_bounds__(32 * kCombineWarps)
    paged_combine_kernel(const __grid_constant__ PdPlan P, int grid) {
  constexpr int KS = D / 16;
  __shared__ int4 seg[kMaxGrid];
  __shared__ uint16_t list[kMaxGrid];          // segments of few parts from the front, of many from the back
  __shared__ int n_few, n_many;
  __shared__ float4 so[kCombineWarps][32];
  __shared__ float4 sml[kCombineWarps][4];     // (m, l) of query rows 2 t, 2 t + 1
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait_and_release();
  for (int c = threadIdx.x; c < grid; c += 32 * kCombineWarps) seg[c] = P.info[c];
  __syncthreads();
  if (warp == 0) {                             // in one order, the same in every CTA
    int few = 0, many = 0;
    for (int c = lane; c - lane < grid; c += 32) {
      const int parts = c < grid ? seg[c].z : 0;
      const bool is_few = parts > 0 && parts <= kCombineFew, is_many = parts > kCombineFew;
      const unsigned f = __ballot_sync(0xffffffffu, is_few), m = __ballot_sync(0xffffffffu, is_many), below = (1u << lane) - 1;
      if (is_few) list[few + __popc(f & below)] = c;
      if (is_many) list[kMaxGrid - 1 - many - __popc(m & below)] = c;
      few += __popc(f);
      many += __popc(m);
    }
    if (lane == 0) {
      n_few = few;
      n_many = many;
    }
  }
  __syncthreads();
  const int per_seg = (P.heads_cta << P.rg_log) * KS;
  for (int u = blockIdx.x; u < n_many * per_seg; u += gridDim.x) {
    const int4 inf = seg[list[kMaxGrid - 1 - u / per_seg]];
    const int hn = u % per_seg / KS, i = u % KS;
    const PartState a = merge_run<T, D>(P, inf, hn, i, inf.z * warp / kCombineWarps, inf.z * (warp + 1) / kCombineWarps, lane);
    so[warp][lane] = a.o;
    if (lane < 4) sml[warp][lane] = make_float4(a.m0, a.l0, a.m1, a.l1);
    __syncthreads();
    if (warp == 0) {
      PartState t = {-INFINITY, -INFINITY, 0.f, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
      float4 ml[kCombineWarps], x[kCombineWarps];
#pragma unroll
      for (int w = 0; w < kCombineWarps; ++w) {
        ml[w] = sml[w][lane & 3];
        x[w] = so[w][lane];
      }
      merge_parts(t, ml, x);
      write_unit<T, D>(P, inf, hn, i, t, lane);
    }
    __syncthreads();
  }
  // empty sequences: zeros and -infinity
  for (int b = blockIdx.x; b < P.pool.num_seqs; b += gridDim.x) {
    if (clamped_length(P, b, false) > 0) continue;
    for (int i = threadIdx.x; i < P.hq * D; i += 32 * kCombineWarps) {
      const int64_t o = static_cast<int64_t>(b) * P.hq * D + i;
      if (P.out_fp32)
        static_cast<float *>(P.out)[o] = 0.f;
      else
        static_cast<uint16_t *>(P.out)[o] = 0;
    }
    if (P.lse)
      for (int i = threadIdx.x; i < P.hq; i += 32 * kCombineWarps) P.lse[static_cast<int64_t>(b) * P.hq + i] = -INFINITY;
  }
  for (int u = warp * gridDim.x + blockIdx.x; u < n_few * per_seg; u += gridDim.x * kCombineWarps) {
    const int4 inf = seg[list[u / per_seg]];
    const int hn = u % per_seg / KS, i = u % KS;
    write_unit<T, D>(P, inf, hn, i, merge_run<T, D>(P, inf, hn, i, 0, inf.z, lane), lane);
  }
}

// ------------------------------------------------------------------ host side
struct PdShape {
  int group, rg_log, heads_cta, wph_log, groups, grid;
  size_t info_off, ml_off, part_off, total;
};

apack_status plan_shape(const apack_paged_cache *c, int32_t hq, PdShape *s) {
  if (hq < 1 || hq > 1024 || hq % c->num_kv_heads != 0) return APACK_EINVAL;
  s->group = hq / c->num_kv_heads;
  if (s->group > 32) return APACK_EUNSUPPORTED;
  s->rg_log = s->group > 16 ? 2 : s->group > 8 ? 1 : 0;
  const int readers_log = s->rg_log > 1;
  // KV heads of a CTA: the largest divisor of their number that its warps cover; the other warps split the tiles
  s->heads_cta = 1;
  for (int h = 1; h <= kWarps >> readers_log; ++h)
    if (c->num_kv_heads % h == 0) s->heads_cta = h;
  s->wph_log = 0;
  while ((s->heads_cta << (readers_log + s->wph_log + 1)) <= kWarps) ++s->wph_log;
  s->groups = c->num_kv_heads / s->heads_cta;
  s->grid = std::min(device_sm_count(), kMaxGrid);
  auto up = [](size_t x) { return (x + 255) & ~static_cast<size_t>(255); };
  const size_t rows = (static_cast<size_t>(2 * s->grid) * s->heads_cta << s->rg_log) * 8;
  s->info_off = 256;
  s->ml_off = up(s->info_off + s->grid * sizeof(int4));
  s->part_off = up(s->ml_off + rows * sizeof(float2));
  s->total = up(s->part_off + rows * c->head_dim * sizeof(float));
  return APACK_OK;
}

constexpr size_t kSmem = kStageBytesCta + kMergeFloats * sizeof(float) + kWarps * 8 * sizeof(float2) +
                         2 * kMaxStages * sizeof(uint64_t) + kWarps * kWindow * sizeof(int);

template <class T, int D, int NG, bool SHARED>
cudaError_t launch_chunk(const PdPlan &P, const CUtensorMap &kmap, const CUtensorMap &vmap, int grid, cudaStream_t stream) {
  static std::atomic<uint64_t> attr{0};
  const cudaError_t e = once_per_device(attr, [] {
    return cudaFuncSetAttribute(paged_chunk_kernel<T, D, NG, SHARED>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(kSmem));
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(paged_chunk_kernel<T, D, NG, SHARED>, dim3(grid), dim3(kThreads), kSmem, stream, P, kmap, vmap);
}

template <class T, int D>
cudaError_t launch_paged(const PdPlan &P, const CUtensorMap &kmap, const CUtensorMap &vmap, int grid,
                         cudaStream_t stream) {
  cudaError_t e = P.rg_log == 0   ? launch_chunk<T, D, 1, false>(P, kmap, vmap, grid, stream)
                  : P.rg_log == 1 ? launch_chunk<T, D, 2, false>(P, kmap, vmap, grid, stream)
                                  : launch_chunk<T, D, 2, true>(P, kmap, vmap, grid, stream);
  if (e != cudaSuccess) return e;
  count_launches(1);
  e = launch_pdl(paged_combine_kernel<T, D>, dim3(grid), dim3(32 * kCombineWarps), 0, stream, P, grid);
  if (e == cudaSuccess) count_launches(1);
  return e;
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

apack_status apack_paged_decode_workspace_size(const apack_paged_cache *cache, int32_t num_q_heads, size_t *bytes) {
  if (!bytes) return APACK_EINVAL;
  apack_status st = validate_pool(cache, true);
  if (st != APACK_OK) return st;
  PdShape s;
  st = plan_shape(cache, num_q_heads, &s);
  if (st == APACK_OK) *bytes = s.total;
  return st;
}

apack_status apack_paged_decode_attention(const apack_paged_cache *cache, int32_t layer, const int32_t *seqlens,
                                          const void *q, int64_t q_token_stride, int32_t num_q_heads, float scale,
                                          void *out, int32_t out_dtype, float *lse, void *ws, size_t ws_bytes,
                                          void *stream) {
  apack_status st = validate_pool(cache, true);
  if (st != APACK_OK) return st;
  PdShape s;
  st = plan_shape(cache, num_q_heads, &s);
  if (st != APACK_OK) return st;
  if (layer < 0 || layer >= cache->num_layers || !seqlens || !q || !out || !ws || !(scale > 0.f) ||
      !std::isfinite(scale * 1.4426950408889634f))
    return APACK_EINVAL;
  if (out_dtype != cache->dtype && out_dtype != APACK_FP32) return APACK_EINVAL;
  const int64_t row = static_cast<int64_t>(num_q_heads) * cache->head_dim * 2;
  if ((reinterpret_cast<uintptr_t>(q) & 15) || (q_token_stride & 15) || (cache->num_seqs > 1 && q_token_stride < row) ||
      (reinterpret_cast<uintptr_t>(out) & 15) || (reinterpret_cast<uintptr_t>(ws) & 255) ||
      ((reinterpret_cast<uintptr_t>(seqlens) | reinterpret_cast<uintptr_t>(lse)) & 3))
    return APACK_EINVAL;
  const int64_t out_row = row * (out_dtype == APACK_FP32 ? 2 : 1);
  if (rows_overlap(cache->num_seqs, static_cast<int64_t>(reinterpret_cast<uintptr_t>(q)), q_token_stride, row,
                   static_cast<int64_t>(reinterpret_cast<uintptr_t>(out)), out_row, out_row))
    return APACK_EINVAL;
  if (ws_bytes < s.total) return APACK_EWORKSPACE;
  if (!on_current_device(cache->k) || !on_current_device(cache->v)) return APACK_EINVAL;   // read by TMA
  PdPlan P;
  std::memset(&P, 0, sizeof(P));
  P.pool = pool_view(cache, layer);
  P.seqlens = seqlens;
  P.wide_lengths = (reinterpret_cast<uintptr_t>(seqlens) & 15) == 0;
  P.q = static_cast<const uint8_t *>(q);
  P.q_stride = q_token_stride;
  P.hq = num_q_heads;
  P.group = s.group;
  P.heads_cta = s.heads_cta;
  P.wph_log = s.wph_log;
  P.rg_log = s.rg_log;
  P.groups = s.groups;
  const int tile = tile_tokens(cache->head_dim);
  const int box_tokens = std::gcd(cache->page_tokens, tile);
  P.boxes = box_tokens < (s.rg_log > 0 ? 16 : 8) ? 0 : tile / box_tokens;
  P.max_rows = static_cast<int32_t>(
      std::min<int64_t>(INT32_MAX - tile, static_cast<int64_t>(cache->max_pages) * cache->page_tokens));
  P.seg_cost = std::max(1, kSegBytes / (tile * s.heads_cta * cache->head_dim * 4));
  P.scale2 = scale * 1.4426950408889634f;
  P.grow = (cache->dtype == APACK_BF16 ? Half16<__nv_bfloat16>::kGrow : Half16<__half>::kGrow) / P.scale2;
  P.out = out;
  P.out_fp32 = out_dtype == APACK_FP32;
  P.lse = lse;
  uint8_t *w = static_cast<uint8_t *>(ws);
  P.info = reinterpret_cast<int4 *>(w + s.info_off);
  P.ml = reinterpret_cast<float2 *>(w + s.ml_off);
  P.part = reinterpret_cast<float *>(w + s.part_off);
  P.err = static_cast<DeviceError *>(ws);
  CUtensorMap kmap, vmap;
  std::memset(&kmap, 0, sizeof(kmap));
  std::memset(&vmap, 0, sizeof(vmap));
  const uint32_t blocks = box_tokens < 16 ? 1 : cache->head_dim / 64;   // tiles keep their blocks apart
  if (P.boxes && (!make_page_map(&kmap, cache, P.pool.k, box_tokens, blocks) ||
                  !make_page_map(&vmap, cache, P.pool.v, box_tokens, blocks)))
    return APACK_ECUDA;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  if (cache->dtype == APACK_BF16)
    return check_cuda(cache->head_dim == 128 ? launch_paged<__nv_bfloat16, 128>(P, kmap, vmap, s.grid, cs)
                                             : launch_paged<__nv_bfloat16, 64>(P, kmap, vmap, s.grid, cs));
  return check_cuda(cache->head_dim == 128 ? launch_paged<__half, 128>(P, kmap, vmap, s.grid, cs)
                                           : launch_paged<__half, 64>(P, kmap, vmap, s.grid, cs));
}

}  // extern "C"
