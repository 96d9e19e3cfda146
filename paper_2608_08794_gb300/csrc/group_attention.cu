// group_attention.cu -- attention of new tokens over paged caches, the shared rows of a group of sequences read once.
#include <cmath>
#include <cstring>

#include "group.cuh"

namespace apack {
namespace {

// A warp per query row.
template <class T, int D>
__global__ void __launch_bounds__(256) group_rows_kernel(const __grid_constant__ GroupArgs A) {
  constexpr int kF = D / 32;
  __shared__ float qs[8][D];
  pdl_wait_and_release();
  GroupHead h;
  if (!group_head(A, h)) {
    if (threadIdx.x == 0 && blockIdx.x == 0) raise_device_error(A.err, APACK_EDEVICE, 150);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t u = blockIdx.x * 8ll + warp;
  if (u >= static_cast<int64_t>(A.n_q) * A.hq) return;
  const int t = static_cast<int>(u / A.hq), hd = static_cast<int>(u - static_cast<int64_t>(t) * A.hq);
  const GroupTok tok = reinterpret_cast<const GroupTok *>(A.ws + h.tok_off)[t];
  if (!tok.real) return;
  const T *q = reinterpret_cast<const T *>(A.q + t * A.q_stride) + hd * D;
  for (int i = lane; i < D; i += 32) qs[warp][i] = static_cast<float>(q[i]);
  __syncwarp();
  float m = -INFINITY, l = 0.f, o[kF] = {};
  const GroupItem *items = reinterpret_cast<const GroupItem *>(A.ws + h.item_off);
#pragma unroll 1
  for (int part = 0; part < 2; ++part) {
    const int i = part ? tok.own : tok.prefix;
    if (i < 0) continue;
    group_row<T, D>(A, items[i].seq, hd / A.group, items[i].key0, min(items[i].key1, tok.limit), qs[warp], m, l, o);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < kF; ++e) reinterpret_cast<T *>(A.out)[u * D + lane * kF + e] = static_cast<T>(o[e] * inv);
  if (A.lse && lane == 0) A.lse[u] = (m + log2f(l)) * 0.6931471805599453f;
}

template <class T, int D>
cudaError_t launch_rows(const GroupArgs &A, cudaStream_t stream) {
  const int64_t rows = static_cast<int64_t>(A.n_q) * A.hq;
  const cudaError_t e = launch_pdl(group_rows_kernel<T, D>, dim3(static_cast<unsigned>((rows + 7) / 8)), dim3(256), 0, stream, A);
  if (e == cudaSuccess) count_launches(1);
  return e;
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" apack_status apack_paged_group_attention(const apack_paged_cache *cache, int32_t layer, int64_t n_q,
                                                    const void *q, int64_t q_token_stride, int32_t num_q_heads,
                                                    float scale, void *out, float *lse, void *ws, size_t ws_bytes,
                                                    void *stream) {
  apack_status st = validate_pool(cache, true);
  if (st != APACK_OK) return st;
  GroupShape s;
  st = group_shape(cache, num_q_heads, 1, n_q, &s);
  if (st != APACK_OK) return st;
  if (layer < 0 || layer >= cache->num_layers || !ws || !(scale > 0.f) || !std::isfinite(scale * 1.4426950408889634f))
    return APACK_EINVAL;
  if ((reinterpret_cast<uintptr_t>(ws) & 255)) return APACK_EINVAL;
  if (ws_bytes < s.total) return APACK_EWORKSPACE;
  if (n_q == 0) return APACK_OK;
  const int64_t row = static_cast<int64_t>(num_q_heads) * cache->head_dim * 2;
  if (!q || !out || (reinterpret_cast<uintptr_t>(q) & 15) || (q_token_stride & 15) || (n_q > 1 && q_token_stride < row) ||
      (reinterpret_cast<uintptr_t>(out) & 15) || (reinterpret_cast<uintptr_t>(lse) & 3))
    return APACK_EINVAL;
  if (rows_overlap(n_q, static_cast<int64_t>(reinterpret_cast<uintptr_t>(q)), q_token_stride, row,
                   static_cast<int64_t>(reinterpret_cast<uintptr_t>(out)), row, row))
    return APACK_EINVAL;
  if (!on_current_device(cache->k) || !on_current_device(cache->v)) return APACK_EINVAL;   // read by TMA
  GroupArgs A;
  std::memset(&A, 0, sizeof(A));
  A.pool = pool_view(cache, layer);
  A.ws = static_cast<uint8_t *>(ws);
  A.ws_bytes = static_cast<int64_t>(ws_bytes);
  A.q = static_cast<const uint8_t *>(q);
  A.q_stride = q_token_stride;
  A.hq = num_q_heads;
  A.hkv = cache->num_kv_heads;
  A.group = s.group;
  A.n_q = static_cast<int32_t>(n_q);
  A.head_dim = cache->head_dim;
  A.scale2 = scale * 1.4426950408889634f;
  A.out = static_cast<uint8_t *>(out);
  A.lse = lse;
  A.box = group_box(cache->page_tokens);
  A.err = static_cast<DeviceError *>(ws);
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  if (cache->dtype == APACK_BF16)
    return check_cuda(cache->head_dim == 128 ? launch_rows<__nv_bfloat16, 128>(A, cs) : launch_rows<__nv_bfloat16, 64>(A, cs));
  return check_cuda(cache->head_dim == 128 ? launch_rows<__half, 128>(A, cs) : launch_rows<__half, 64>(A, cs));
}
