// paged_copy.cu -- rows and pages of paged caches moved: the compaction of Sec. 3.2 ("slice their KV-cache
// entries") between pools (apack_paged_compact), and whole pages (apack_copy_pages).
//
// Bound by HBM: every byte is read once and written once.  A plane is K or V of one layer (of one head, where a
// token's heads are not back to back).  A CTA resolves the page of each row of its run once and then moves those
// rows in several planes.  Measured: 24 layers of a contiguous cache, 27,144 rows to 11,844 in pages, 172.6 us, 6.7
// TB/s, 0.99 of the copy rate; 257 pages of 28 layers 71.2 us (0.98); 13 caches of 512-byte rows, pages to pages,
// 42.6 us (0.91); one page of 28 layers 2.3 us.
#include <algorithm>
#include <cstdlib>
#include <cstring>

#include "paged.cuh"
#include "ptx.cuh"

namespace apack {
namespace {

// A CTA moves the same rows, about 32 KB of a plane, in several planes: with half of that, the time of 13 caches of
// 512-byte rows was 46 us, with this 43 (their rows' addresses take two rounds of loads to find).
constexpr int kChunkBytes = 32768;
constexpr int kRows = 128;             // rows whose addresses a CTA holds at most
constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 8;         // 16-byte pieces a thread has in flight

struct MovePlan {
  PoolView src, dst;
  int64_t n_rows;
  int32_t num_seqs;
  const int32_t *keep_idx, *cu_src, *cu_dst;
  const int32_t *pairs;                // apack_copy_pages
  int32_t layers, heads;               // planes = 2 * layers * heads
  int32_t pieces;                      // 16-byte pieces of a row
  FastDiv piece_div;
  int32_t planes_cta, planes;
  int32_t rows_cta;
  DeviceError *err;
};

// Offsets of up to this many sequences are brought to shared memory in one round of loads before they are searched
// (a search in L2 takes a round trip per step).
constexpr int kStagedSeqs = 1024;

// Sequence of output row j: the last b with cu[b] <= j.
__device__ __forceinline__ int find_seq(const int32_t *cu, int n, int64_t j) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= j) lo = mid; else hi = mid;
  }
  return lo;
}

// Source and destination byte offsets of output row j within a layer's planes (src -1: not copied).
// cu: cu_dst, staged or not.
__device__ __forceinline__ void resolve(const MovePlan &P, const int32_t *cu, int32_t keep, int64_t j, int64_t *src, int64_t *dst) {
  *src = -1;
  *dst = -1;
  if (j >= P.n_rows) return;
  if (P.pairs) {
    const uint32_t i = P.src.page_tokens.div(static_cast<uint32_t>(j)), r = static_cast<uint32_t>(j) - i * P.src.page_tokens.d;
    const int32_t a = __ldg(P.pairs + 2 * static_cast<int64_t>(i)), b = __ldg(P.pairs + 2 * static_cast<int64_t>(i) + 1);
    if (static_cast<uint32_t>(a) >= static_cast<uint32_t>(P.src.num_pages) ||
        static_cast<uint32_t>(b) >= static_cast<uint32_t>(P.src.num_pages)) {
      if (P.err) raise_device_error(P.err, APACK_EDEVICE, 92, a, b);
      return;
    }
    if (a == b) return;                // padding: not even written back, so that it may stand beside a pair that writes the page
    *src = a * P.src.page_stride + r * P.src.token_stride;
    *dst = b * P.src.page_stride + r * P.src.token_stride;
    return;
  }
  if (j >= cu[P.num_seqs]) return;
  const int b = find_seq(cu, P.num_seqs, j);
  const int32_t to = static_cast<int32_t>(j - cu[b]);
  const int32_t from = P.keep_idx ? keep - (P.cu_src ? __ldg(P.cu_src + b) : 0) : to;
  const int64_t s = P.src.row_offset(b, from), d = P.dst.row_offset(b, to);
  if (s < 0 || d < 0) {
    if (P.err) raise_device_error(P.err, APACK_EDEVICE, 91, b, static_cast<int32_t>(j));
    return;
  }
  *src = s;
  *dst = d;
}

__device__ __forceinline__ void plane_bases(const MovePlan &P, int plane, const uint8_t **src, uint8_t **dst) {
  const int head = plane % P.heads, lp = plane / P.heads;
  const int layer = lp >> 1;
  const bool v = lp & 1;
  *src = (v ? P.src.v : P.src.k) + layer * P.src.layer_stride + head * P.src.head_stride;
  *dst = (v ? P.dst.v : P.dst.k) + layer * P.dst.layer_stride + head * P.dst.head_stride;
}

__global__ void __launch_bounds__(kMoveThreads, 4) move_rows_kernel(const __grid_constant__ MovePlan P) {
  __shared__ int64_t so[kRows], to[kRows];
  __shared__ int32_t cu_s[kStagedSeqs + 1];
  pdl_wait_and_release();
  const int64_t j = static_cast<int64_t>(blockIdx.x) * P.rows_cta + threadIdx.x;
  const int32_t *cu = P.cu_dst;
  int32_t keep = 0;
  // n_rows may be more than cu_dst[B]; keep_idx ends there
  if (P.keep_idx && threadIdx.x < P.rows_cta && j < min(P.n_rows, static_cast<int64_t>(__ldg(P.cu_dst + P.num_seqs))))
    keep = __ldg(P.keep_idx + j);
  if (!P.pairs && P.num_seqs <= kStagedSeqs) {
    for (int b = threadIdx.x; b <= P.num_seqs; b += kMoveThreads) cu_s[b] = __ldg(P.cu_dst + b);
    __syncthreads();
    cu = cu_s;
  }
  if (threadIdx.x < P.rows_cta) resolve(P, cu, keep, j, &so[threadIdx.x], &to[threadIdx.x]);
  __syncthreads();
  const int total = P.rows_cta * P.pieces;
  const int p1 = min(P.planes, static_cast<int>(blockIdx.y + 1) * P.planes_cta);
  for (int plane = blockIdx.y * P.planes_cta; plane < p1; ++plane) {
    const uint8_t *src;
    uint8_t *dst;
    plane_bases(P, plane, &src, &dst);
    for (int e0 = threadIdx.x; e0 < total; e0 += kMoveThreads * kMoveUnroll) {
      uint4 x[kMoveUnroll];
#pragma unroll
      for (int u = 0; u < kMoveUnroll; ++u) {
        const int e = e0 + u * kMoveThreads;
        if (e < total) {
          const int r = P.piece_div.div(e), c = e - r * P.pieces;
          if (so[r] >= 0) x[u] = *reinterpret_cast<const uint4 *>(src + so[r] + c * 16);
        }
      }
#pragma unroll
      for (int u = 0; u < kMoveUnroll; ++u) {
        const int e = e0 + u * kMoveThreads;
        if (e < total) {
          const int r = P.piece_div.div(e), c = e - r * P.pieces;
          if (so[r] >= 0) *reinterpret_cast<uint4 *>(dst + to[r] + c * 16) = x[u];
        }
      }
    }
  }
}

// In place: output row j of a sequence reads row from(j) >= j of the same sequence, from ascending.  A warp owns
// W 16-byte pieces of every row of one plane of one sequence and walks the rows upwards, kStep at a time; the rows that a
// step reads have all arrived before it writes, and no later step reads a row below those this step writes.  So no
// warp waits for another, and the loads of kDepth steps are in flight (into the warp's ring in shared memory); addresses
// are found a step before their loads, from page numbers read two and indices read three steps before.  A step costs
// about one trip to L2 for those.  24 layers of 27,144 rows to 11,844, 4 heads of 128, calls in a row: 266 us in pages of
// 16 tokens (4.4 TB/s), 260 of 64, 221 in one page, 368 of 1; 8 caches of 9,000 rows, half of them kept, 16-token pages: 582
// us, 6.1 TB/s.  When it was chosen (266 was 275, 582 was 589): 514 and 989 with the loads of one step of 64 rows in
// registers, 306 and 632 or less with steps of 64 in the ring, 267 and 706 with 3 steps of 128.
constexpr int kStep = 128, kDepth = 2, kPlaceWarps = 2;
constexpr int place_bytes(int w) { return kPlaceWarps * kDepth * kStep * (w * 16 + 8); }
template <int W>
__global__ void __launch_bounds__(32 * kPlaceWarps)
    move_in_place_kernel(const __grid_constant__ MovePlan P, int segs, int64_t units) {
  extern __shared__ __align__(16) uint8_t place_smem[];
  pdl_wait_and_release();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t unit = static_cast<int64_t>(blockIdx.x) * kPlaceWarps + warp;
  if (unit >= units) return;
  const int seg = static_cast<int>(unit % segs);
  const int64_t rest = unit / segs;
  const int plane = static_cast<int>(rest % P.planes), b = static_cast<int>(rest / P.planes);
  const int64_t j0 = max(__ldg(P.cu_dst + b), 0), j1 = min(static_cast<int64_t>(__ldg(P.cu_dst + b + 1)), P.n_rows);
  const uint8_t *src;
  uint8_t *dst;
  plane_bases(P, plane, &src, &dst);
  constexpr int kRowsAtOnce = 32 / W, kLoads = kStep / kRowsAtOnce, kRows = kStep / 32;
  const int c = seg * W + lane % W;
  const bool mine = c < P.pieces;
  const int32_t base = P.cu_src ? __ldg(P.cu_src + b) : 0;
  uint4 *ring = reinterpret_cast<uint4 *>(place_smem) + warp * kDepth * kStep * W;
  int64_t *ring_to = reinterpret_cast<int64_t *>(place_smem + kPlaceWarps * kDepth * kStep * W * 16) + warp * kDepth * kStep;
  // lane i finds the addresses of rows i, i + 32, ... of a step: its index, the pages of both rows, the offsets
  int32_t keep[kRows], row[kRows], from_page[kRows], to_page[kRows];
  int64_t from[kRows], to[kRows];
  auto read_keep = [&](int64_t j) {
#pragma unroll
    for (int h = 0; h < kRows; ++h)
      if (j + h * 32 + lane < j1) keep[h] = __ldg(P.keep_idx + j + h * 32 + lane);
  };
  auto read_pages = [&](int64_t j) {
#pragma unroll
    for (int h = 0; h < kRows; ++h) {
      const int64_t r = j + h * 32 + lane;
      if (r >= j1) continue;
      row[h] = keep[h] - base;
      from_page[h] = P.src.page_of(b, row[h]);
      to_page[h] = P.dst.page_of(b, static_cast<int32_t>(r - j0));
    }
  };
  auto find = [&](int64_t j) {
#pragma unroll
    for (int h = 0; h < kRows; ++h) {
      const int64_t r = j + h * 32 + lane;
      from[h] = to[h] = -1;
      if (r >= j1) continue;
      const int64_t s = P.src.offset_in(from_page[h], row[h]), d = P.dst.offset_in(to_page[h], static_cast<int32_t>(r - j0));
      if (s >= 0 && d >= 0) {
        from[h] = s;
        to[h] = d;
      } else if (P.err) {
        raise_device_error(P.err, APACK_EDEVICE, 93, b, static_cast<int32_t>(r - j0));
      }
    }
  };
  // a lane writes what it has loaded itself
  auto load = [&](int slot) {
#pragma unroll
    for (int h = 0; h < kRows; ++h) ring_to[slot * kStep + h * 32 + lane] = to[h];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int64_t s = __shfl_sync(0xffffffffu, from[u / W], u % W * kRowsAtOnce + lane / W);
      if (s >= 0 && mine) cp_async_16(smem_u32(ring + (slot * kLoads + u) * 32 + lane), src + s + c * 16);
    }
    cp_async_commit();
  };
  int64_t ahead = j0;                                  // the step that is loaded next
  read_keep(ahead);
  read_pages(ahead);
  read_keep(ahead + kStep);
  find(ahead);
  read_pages(ahead + kStep);
  read_keep(ahead + 2 * kStep);
  auto advance = [&](int slot) {
    load(slot);
    ahead += kStep;
    find(ahead);
    read_pages(ahead + kStep);
    read_keep(ahead + 2 * kStep);
  };
#pragma unroll
  for (int slot = 0; slot < kDepth; ++slot) advance(slot);
  int slot = 0;
  for (int64_t j = j0; j < j1; j += kStep) {
    cp_async_wait<kDepth - 1>();
    __syncwarp();                                      // every row of the step has been read
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int64_t d = ring_to[slot * kStep + u * kRowsAtOnce + lane / W];
      if (d >= 0 && mine) *reinterpret_cast<uint4 *>(dst + d + c * 16) = ring[(slot * kLoads + u) * 32 + lane];
    }
    __syncwarp();
    advance(slot);
    slot = slot + 1 == kDepth ? 0 : slot + 1;
  }
  cp_async_wait<0>();
}

template <int W>
cudaError_t launch_in_place(const MovePlan &P, int segs, int64_t units, unsigned grid, cudaStream_t stream) {
  static std::atomic<uint64_t> attr{0};
  const cudaError_t e = once_per_device(attr, [] {
    return cudaFuncSetAttribute(move_in_place_kernel<W>, cudaFuncAttributeMaxDynamicSharedMemorySize, place_bytes(W));
  });
  if (e != cudaSuccess) return e;
  return launch_pdl(move_in_place_kernel<W>, dim3(grid), dim3(32 * kPlaceWarps), place_bytes(W), stream, P, segs, units);
}

// Heads of a token back to back: one plane per layer and tensor.
bool fused_heads(const apack_paged_cache *c) { return c->num_kv_heads == 1 || c->head_stride == c->head_dim * 2; }

apack_status launch_move(MovePlan &P, const apack_paged_cache *a, const apack_paged_cache *b, int32_t layers,
                         bool in_place, cudaStream_t stream) {
  const bool fused = fused_heads(a) && fused_heads(b);
  P.layers = layers;
  P.heads = fused ? 1 : a->num_kv_heads;
  P.pieces = a->head_dim / 8 * (fused ? a->num_kv_heads : 1);
  P.piece_div = fast_div(P.pieces);
  P.planes = 2 * layers * P.heads;
  if (in_place) {
    // 128 bytes of a row per warp; fewer where that leaves SMs with less than 4 warps (the prompt's prune 292 us with 2,
    // 278 with 4; with 8, and so 32 bytes, no more)
    int w = 8;
    auto segs = [&](int width) { return (P.pieces + width - 1) / width; };
    auto units_of = [&](int width) { return static_cast<int64_t>(P.num_seqs) * P.planes * segs(width); };
    while (w > 2 && units_of(w) < 4 * static_cast<int64_t>(device_sm_count())) w /= 2;
    const int64_t units = units_of(w), grid = (units + kPlaceWarps - 1) / kPlaceWarps;
    if (grid > INT32_MAX) return APACK_EUNSUPPORTED;
    const unsigned g = static_cast<unsigned>(grid);
    if (check_cuda(w == 8   ? launch_in_place<8>(P, segs(8), units, g, stream)
                   : w == 4 ? launch_in_place<4>(P, segs(4), units, g, stream)
                            : launch_in_place<2>(P, segs(2), units, g, stream)) != APACK_OK)
      return APACK_ECUDA;
    count_launches(1);
    return APACK_OK;
  }
  P.rows_cta = static_cast<int32_t>(std::min<int64_t>(P.n_rows, std::min(kRows, std::max(1, kChunkBytes / (P.pieces * 16)))));
  const int64_t chunks = (P.n_rows + P.rows_cta - 1) / P.rows_cta;
  // planes of a CTA: as many as leave 32 CTAs per SM (the two-minute prompt: 172.8 us; with 8 per SM 181.3)
  const int64_t want = 32 * static_cast<int64_t>(device_sm_count());
  int64_t splits = std::min<int64_t>(P.planes, std::max<int64_t>(1, (want + chunks - 1) / chunks));
  splits = std::max<int64_t>(splits, (P.planes + 65534) / 65535);
  P.planes_cta = static_cast<int32_t>((P.planes + splits - 1) / splits);
  splits = (P.planes + P.planes_cta - 1) / P.planes_cta;
  if (check_cuda(launch_pdl(move_rows_kernel, dim3(static_cast<unsigned>(chunks), static_cast<unsigned>(splits)),
                            dim3(kMoveThreads), 0, stream, P)) != APACK_OK)
    return APACK_ECUDA;
  count_launches(1);
  return APACK_OK;
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

apack_status apack_paged_compact(const apack_paged_cache *src, const apack_paged_cache *dst, int32_t src_layer,
                                 int32_t dst_layer, int32_t num_layers, const int32_t *keep_idx,
                                 const int32_t *cu_src, const int32_t *cu_dst, int64_t n_out, void *ws, void *stream) {
  apack_status st = validate_pool(src, true);
  if (st == APACK_OK) st = validate_pool(dst, true);
  if (st != APACK_OK) return st;
  if (src->num_kv_heads != dst->num_kv_heads || src->head_dim != dst->head_dim || src->dtype != dst->dtype ||
      src->num_seqs != dst->num_seqs)
    return APACK_EINVAL;
  if (num_layers < 1 || src_layer < 0 || dst_layer < 0 || num_layers > src->num_layers - src_layer ||
      num_layers > dst->num_layers - dst_layer || n_out < 0 || n_out > INT32_MAX || !cu_dst || (cu_src && !keep_idx))
    return APACK_EINVAL;
  if ((reinterpret_cast<uintptr_t>(keep_idx) | reinterpret_cast<uintptr_t>(cu_src) | reinterpret_cast<uintptr_t>(cu_dst) |
       reinterpret_cast<uintptr_t>(ws)) & 3)
    return APACK_EINVAL;
  // one page table on both sides: in place, in the same layers of the same pool with an index, or in layers apart
  bool in_place = false;
  if ((src->k == dst->k || src->v == dst->v) && src->page_table == dst->page_table) {
    if (src->k != dst->k || src->v != dst->v || src->table_stride != dst->table_stride || src->max_pages != dst->max_pages ||
        src->num_pages != dst->num_pages || src->page_tokens != dst->page_tokens || src->page_stride != dst->page_stride ||
        src->token_stride != dst->token_stride || src->head_stride != dst->head_stride || src->layer_stride != dst->layer_stride)
      return APACK_EINVAL;
    in_place = src_layer == dst_layer;
    if (in_place ? !keep_idx : std::abs(src_layer - dst_layer) < num_layers) return APACK_EINVAL;
  }
  if (n_out == 0) return APACK_OK;
  MovePlan P;
  std::memset(&P, 0, sizeof(P));
  P.src = pool_view(src, src_layer);
  P.dst = pool_view(dst, dst_layer);
  P.n_rows = n_out;
  P.num_seqs = src->num_seqs;
  P.keep_idx = keep_idx;
  P.cu_src = cu_src;
  P.cu_dst = cu_dst;
  P.err = static_cast<DeviceError *>(ws);
  return launch_move(P, src, dst, num_layers, in_place, static_cast<cudaStream_t>(stream));
}

apack_status apack_copy_pages(const apack_paged_cache *cache, const int32_t *pairs, int64_t n_pairs, void *ws,
                              void *stream) {
  const apack_status st = validate_pool(cache, false);
  if (st != APACK_OK) return st;
  if (n_pairs < 0 || n_pairs > INT32_MAX / cache->page_tokens) return APACK_EINVAL;
  if (n_pairs == 0) return APACK_OK;
  if (!pairs || ((reinterpret_cast<uintptr_t>(pairs) | reinterpret_cast<uintptr_t>(ws)) & 3)) return APACK_EINVAL;
  MovePlan P;
  std::memset(&P, 0, sizeof(P));
  P.src = pool_view(cache, 0);
  P.dst = P.src;
  P.n_rows = n_pairs * cache->page_tokens;
  P.num_seqs = 1;
  P.pairs = pairs;
  P.err = static_cast<DeviceError *>(ws);
  return launch_move(P, cache, cache, cache->num_layers, false, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
