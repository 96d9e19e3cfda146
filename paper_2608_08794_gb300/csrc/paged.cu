// paged.cu -- host side of the paged key-value cache: descriptor checks and TMA maps.
#include <algorithm>

#include "paged.cuh"

namespace apack {

namespace {

// Two nested extents: `n` items of `inner` bytes, `stride` apart.  Returns their span, or -1 on overlap.
int64_t span_of(int64_t n, int64_t stride, int64_t inner) {
  if (n <= 1) return inner;
  if (stride < inner || stride > INT64_MAX / n) return -1;
  return (n - 1) * stride + inner;
}

// Items of two indices that may be nested either way.
bool nested(int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t inner, int64_t *span) {
  const int64_t a = span_of(n1, s1, inner), ab = a < 0 ? -1 : span_of(n2, s2, a);
  const int64_t b = span_of(n2, s2, inner), ba = b < 0 ? -1 : span_of(n1, s1, b);
  *span = ab >= 0 ? ab : ba;
  return *span >= 0;
}

}  // namespace

bool on_current_device(const void *p) {
  cudaPointerAttributes at{};
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaPointerGetAttributes(&at, p) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return at.type == cudaMemoryTypeManaged || (at.type == cudaMemoryTypeDevice && at.device == dev);
}

bool rows_overlap(int64_t n, int64_t a, int64_t stride_a, int64_t row_a, int64_t b, int64_t stride_b, int64_t row_b) {
  if (n == 1) stride_a = stride_b = 0;
  if (a + (n - 1) * stride_a + row_a <= b || b + (n - 1) * stride_b + row_b <= a) return false;
  if (n == 1) return true;
  if (stride_a == stride_b) {            // rows i and j: -row_b < b - a + (j - i) stride < row_a
    const int64_t d = b - a + row_b;     // the least j - i above -d / stride
    const int64_t least = d >= 0 ? -((d - 1 + stride_a) / stride_a) + 1 : -d / stride_a + 1;
    const int64_t m = std::max(least, 1 - n);
    return m < n && b - a + m * stride_a < row_a;
  }
  for (int64_t i = std::max<int64_t>(0, (b - a - row_a) / stride_a); i < n && a + i * stride_a < b + (n - 1) * stride_b + row_b; ++i) {
    const int64_t at = a + i * stride_a, d = at - b - row_b;   // the first row of b that ends behind `at`
    const int64_t j = d < 0 ? 0 : d / stride_b + 1;
    if (j < n && b + j * stride_b < at + row_a) return true;
  }
  return false;
}

apack_status validate_pool(const apack_paged_cache *c, bool table) {
  if (!c || !c->k || !c->v) return APACK_EINVAL;
  if (c->dtype != APACK_BF16 && c->dtype != APACK_FP16) return APACK_EUNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return APACK_EUNSUPPORTED;
  if (c->num_layers < 1 || c->num_pages < 1 || c->page_tokens < 1 || c->page_tokens > (1 << 30) ||
      c->num_kv_heads < 1 || c->num_kv_heads > 256)
    return APACK_EINVAL;
  if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v) | c->layer_stride | c->page_stride |
       c->token_stride | c->head_stride) & 15)
    return APACK_EINVAL;
  int64_t page = 0, all = 0;
  if (!nested(c->num_kv_heads, c->head_stride, c->page_tokens, c->token_stride, 2 * c->head_dim, &page) ||
      !nested(c->num_pages, c->page_stride, c->num_layers, c->layer_stride, page, &all))
    return APACK_EINVAL;
  if (table) {
    if (!c->page_table || (reinterpret_cast<uintptr_t>(c->page_table) & 3)) return APACK_EINVAL;
    if (c->num_seqs < 1 || c->num_seqs > APACK_MAX_SEQS || c->max_pages < 1 || c->table_stride < c->max_pages)
      return APACK_EINVAL;
  }
  return APACK_OK;
}

PoolView pool_view(const apack_paged_cache *c, int32_t layer) {
  PoolView p{};
  p.k = static_cast<uint8_t *>(c->k) + static_cast<int64_t>(layer) * c->layer_stride;
  p.v = static_cast<uint8_t *>(c->v) + static_cast<int64_t>(layer) * c->layer_stride;
  p.layer_stride = c->layer_stride;
  p.page_stride = c->page_stride;
  p.token_stride = c->token_stride;
  p.head_stride = c->head_stride;
  p.table = c->page_table;
  p.table_stride = c->table_stride;
  p.num_pages = c->num_pages;
  p.num_seqs = c->num_seqs;
  p.max_pages = c->max_pages;
  p.page_tokens = fast_div(static_cast<uint32_t>(c->page_tokens));
  return p;
}

bool make_page_map(CUtensorMap *map, const apack_paged_cache *c, const void *layer_base, uint32_t box_tokens,
                   uint32_t box_blocks) {
  const EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[5] = {64, static_cast<cuuint64_t>(c->page_tokens), static_cast<cuuint64_t>(c->head_dim / 64),
                              static_cast<cuuint64_t>(c->num_kv_heads), static_cast<cuuint64_t>(c->num_pages)};
  // a dimension of one element takes any valid stride
  const cuuint64_t strides[4] = {static_cast<cuuint64_t>(c->page_tokens > 1 ? c->token_stride : 128), 128,
                                 static_cast<cuuint64_t>(c->num_kv_heads > 1 ? c->head_stride : 128),
                                 static_cast<cuuint64_t>(c->num_pages > 1 ? c->page_stride : 128)};
  const cuuint32_t box[5] = {64, box_tokens, box_blocks, 1, 1};
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 5, const_cast<void *>(layer_base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace apack
