// paged.cuh -- the paged key-value cache on the device, shared by its operators (rotary.cu,
// paged_decode.cu, paged_copy.cu).
#pragma once
#include "internal.cuh"

namespace apack {

// Division of 0 <= n < 2^31 by a constant of the launch: (hi(n * mul) + n) >> shift, with
// shift = ceil(log2 d) and mul = floor(2^32 (2^shift - d) / d) + 1 (round-up reciprocal).
struct FastDiv {
  uint32_t d, mul, shift;
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};
inline FastDiv fast_div(uint32_t d) {
  FastDiv f{d, 0, 0};
  while ((uint64_t{1} << f.shift) < d) ++f.shift;
  f.mul = static_cast<uint32_t>(((uint64_t{1} << 32) * ((uint64_t{1} << f.shift) - d)) / d + 1);
  return f;
}

// One pool as a kernel sees it.  k and v already point at the first layer of the call.
struct PoolView {
  uint8_t *k, *v;
  int64_t layer_stride, page_stride, token_stride, head_stride;
  const int32_t *table;
  int64_t table_stride;
  int32_t num_pages, num_seqs, max_pages;
  FastDiv page_tokens;

  // The page of row `row` of sequence `seq`, or -1: a negative row, or one behind the table.
  __device__ __forceinline__ int32_t page_of(uint32_t seq, int32_t row) const {
    if (row < 0) return -1;
    const uint32_t p = page_tokens.div(static_cast<uint32_t>(row));
    return p < static_cast<uint32_t>(max_pages) ? __ldg(table + static_cast<int64_t>(seq) * table_stride + p) : -1;
  }
  // Byte offset of the row in that page within a layer (head 0), or -1: a page outside the pool.
  __device__ __forceinline__ int64_t offset_in(int32_t page, int32_t row) const {
    if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(num_pages)) return -1;
    const uint32_t r = static_cast<uint32_t>(row);
    return page * page_stride + static_cast<int64_t>(r - page_tokens.div(r) * page_tokens.d) * token_stride;
  }
  // Both in one (with one division), or -1.
  __device__ __forceinline__ int64_t row_offset(uint32_t seq, int32_t row) const {
    if (row < 0) return -1;
    const uint32_t p = page_tokens.div(static_cast<uint32_t>(row));
    if (p >= static_cast<uint32_t>(max_pages)) return -1;
    const int32_t page = __ldg(table + static_cast<int64_t>(seq) * table_stride + p);
    if (static_cast<uint32_t>(page) >= static_cast<uint32_t>(num_pages)) return -1;
    return page * page_stride + static_cast<int64_t>(static_cast<uint32_t>(row) - p * page_tokens.d) * token_stride;
  }
};

// Checks a descriptor (null pointers, sizes, alignment, overlap of its slots); `table`: the call reads the
// page table.
apack_status validate_pool(const apack_paged_cache *c, bool table);
PoolView pool_view(const apack_paged_cache *c, int32_t layer);
// Whether any of n rows of `row_a` bytes, stride_a apart from a on, shares a byte with any of n rows at b.
bool rows_overlap(int64_t n, int64_t a, int64_t stride_a, int64_t row_a, int64_t b, int64_t stride_b, int64_t row_b);
// Whether p is device memory of the current device (or managed memory).
bool on_current_device(const void *p);

// 5-D TMA map of one layer's K (or V): {64 features, token in page, 64-feature block, head, page}, boxes of
// box_tokens tokens and box_blocks blocks of one head, 128-byte swizzle; pages outside the pool read as zeros.
bool make_page_map(CUtensorMap *map, const apack_paged_cache *c, const void *layer_base, uint32_t box_tokens,
                   uint32_t box_blocks);

}  // namespace apack
