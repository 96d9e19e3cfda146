// rotary.cu -- rotary positions of packed token rows, alone (apack_rotary) or with the write of new
// tokens into the pages of a cache (apack_rotary_append).
//
// Pair i of a head turns by t = position * freq[i]; (a, b) -> m (a cos t - b sin t, b cos t + a sin t).
// The transposed map (the gradient) turns by -t.
//
// Angles: in 32 bits position * freq loses the angle of far positions (at 10^6 radians one ulp is 0.06).
// The host turns each frequency into 64-bit fixed point, in turns; position * freq mod 2^64 is then the
// phase with whole turns dropped, exactly, in one integer multiplication, for negative positions too.  Its top
// 32 bits as a signed fraction of a half turn go to sincospif.
//
// Bound by HBM with many tokens: a row is read once and written once, the angles are shared by all heads of a token.
// Behind it comes instruction issue (2 loads, 2 stores and about 60 instructions per 16 elements), so a lane owns
// one 16-byte chunk position of a head (both halves of its pairs) and keeps its (cos, sin) in registers over the
// heads it walks through.  Few tokens are bound by latency: position -> angle -> product.
// Measured: 27,144 tokens of 28/4 heads of 128 with append 80.8 us, 6.2 TB/s, 0.91 of the copy rate; 27,144 rows of 32
// heads 78.1 us (0.84), fp32 144.4 (0.91); 8,780 rows of 18 heads 17.8 us (0.67), fp32 29.3 (0.82); 61 tokens 3.4 us.
// Narrow accesses (rows or halves that are no whole 16-byte pieces) are bound by issue: the 8,780 rows 30.4 us, 27,144 of 32
// heads with 36 of 128 elements rotated 243.
#include <algorithm>
#include <cmath>
#include <cstring>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "paged.cuh"

namespace apack {
namespace {

constexpr int kRotThreads = 256;
constexpr int kMaxPairs = 128;          // head_dim <= 256
constexpr int kRotUnroll = 3;           // heads whose loads a lane has in flight
constexpr int kRotCtas = 3;             // CTAs per SM

struct RotPlan {
  uint64_t freq[kMaxPairs];             // 2^-64 turns per position
  float magnitude;
  int32_t pairs, axis1, axis2;          // pairs from axis1 on take axis 1, from axis2 on axis 2
  int32_t n1, n2;                       // chunk positions of a head: rotated, passed through
  int32_t half_off;                     // elements from a chunk to its partner (HALF)
  int32_t head_slots;                   // a warp's lanes: chunk positions x head_slots
  int64_t whole, units;                 // tokens that a warp takes whole, and units of work in all
  int32_t splits, unit_heads;           // parts of the other tokens' heads, and heads of a part
  int32_t heads, rot_heads, q_heads;    // heads in all; the first rot_heads are rotated; q_heads of them are q
  int32_t head_dim;
  int64_t n_tokens;
  const uint8_t *x, *k, *v;
  uint8_t *out;
  int64_t xs, ks, vs, outs;             // token strides in bytes
  const int32_t *positions;
  int64_t pos_axis_stride;
  const int32_t *rows, *seqs;
  PoolView pool;
  DeviceError *err;
};

template <class T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
  static __device__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
  static __device__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  static __device__ float to(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __nv_bfloat16 from(float v) { return __float2bfloat16_rn(v); }
};
template <>
struct Elem<__half> {
  static __device__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
  static __device__ uint32_t pack(float a, float b) {
    const __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
  }
  static __device__ float to(__half v) { return __half2float(v); }
  static __device__ __half from(float v) { return __float2half_rn(v); }
};
template <>
struct Elem<float> {
  static __device__ float to(float v) { return v; }
  static __device__ float from(float v) { return v; }
};

// V consecutive elements, moved in one access (V = 1, or 16 bytes).
template <class T, int V>
struct __align__(sizeof(T) * V) Chunk {
  T e[V];
};

// Turns the pairs of a chunk: element j of lo with element j of hi (SPLIT), or neighbours of lo.
template <class T, int V, bool SPLIT, int N>
__device__ __forceinline__ void turn(Chunk<T, V> &lo, Chunk<T, V> &hi, const float2 (&a)[N]) {
  if constexpr (sizeof(T) == 2 && V > 1) {         // a word holds two elements
    uint32_t(&l)[V / 2] = *reinterpret_cast<uint32_t(*)[V / 2]>(&lo), (&h)[V / 2] = *reinterpret_cast<uint32_t(*)[V / 2]>(&hi);
#pragma unroll
    for (int k = 0; k < V / 2; ++k) {
      if constexpr (SPLIT) {
        const float2 x = Elem<T>::unpack(l[k]), y = Elem<T>::unpack(h[k]);
        const float2 p = a[2 * k], q = a[2 * k + 1];
        l[k] = Elem<T>::pack(x.x * p.x - y.x * p.y, x.y * q.x - y.y * q.y);
        h[k] = Elem<T>::pack(y.x * p.x + x.x * p.y, y.y * q.x + x.y * q.y);
      } else {
        const float2 x = Elem<T>::unpack(l[k]);
        l[k] = Elem<T>::pack(x.x * a[k].x - x.y * a[k].y, x.y * a[k].x + x.x * a[k].y);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      T &pa = SPLIT ? lo.e[j] : lo.e[(2 * j) % V], &pb = SPLIT ? hi.e[j] : lo.e[(2 * j + 1) % V];
      const float x = Elem<T>::to(pa), y = Elem<T>::to(pb);
      pa = Elem<T>::from(x * a[j].x - y * a[j].y);
      pb = Elem<T>::from(y * a[j].x + x * a[j].y);
    }
  }
}

// (m cos, sign m sin) of a pair's angle.
__device__ __forceinline__ float2 angle(const RotPlan &P, int32_t pos, uint64_t freq, float sign) {
  const uint64_t phase = static_cast<uint64_t>(static_cast<int64_t>(pos)) * freq;
  float s, c;
  sincospif(static_cast<float>(static_cast<int32_t>(phase >> 32)) * 4.656612873077393e-10f, &s, &c);   // 2^-31
  return make_float2(P.magnitude * c, sign * P.magnitude * s);
}

// V: elements of an access.  PAIRS: neighbouring elements form a pair; a chunk then holds its pairs whole (V = 1:
// two accesses, as in the HALF layout with the partner one element on).  APPEND: k and v go to pages.
//
// A warp takes a token, or with few tokens a part of its heads, and never waits for another.  Its lanes are chunk
// positions x head_slots; the first heads' loads are under way while the angles are computed (shared by the lanes
// through shared memory) and the slot is looked up, from a position and row that were read one token ahead.
template <class T, int V, bool PAIRS, bool APPEND>
__global__ void __launch_bounds__(kRotThreads, kRotCtas) rotary_kernel(const __grid_constant__ RotPlan P, float sign) {
  using C = Chunk<T, V>;
  constexpr bool kSplit = !PAIRS || V == 1;            // a rotated chunk has a partner chunk
  constexpr int kAngles = kSplit ? V : V / 2;          // pairs of a chunk position
  constexpr int kAhead = kMaxPairs / 32;
  __shared__ __align__(16) float2 cs_all[kRotThreads / 32][kMaxPairs];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float2 *cs = cs_all[warp];
  const int pairs = P.pairs, hd = P.head_dim;
  // chunk positions beyond 32 are walked through, `positions` at a time
  const int n = P.n1 + P.n2, width = min(n, 32);
  const int c0 = lane % width, hs = lane / width;
  const int64_t stride = static_cast<int64_t>(gridDim.x) * (kRotThreads / 32);
  int64_t u = static_cast<int64_t>(blockIdx.x) * (kRotThreads / 32) + warp;
  uint64_t freq[kAhead];                               // of this lane's pairs (parameters are slow to index by lane)
#pragma unroll
  for (int k = 0; k < kAhead; ++k) freq[k] = lane + 32 * k < pairs ? P.freq[lane + 32 * k] : 0;
  pdl_wait_and_release();
  int32_t pos[kAhead], row = -1, seq = 0;
  auto read_ahead = [&](int64_t t) {
    if (t >= P.n_tokens) return;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = lane + 32 * k;
      if (i < pairs) pos[k] = __ldg(P.positions + ((i >= P.axis1) + (i >= P.axis2)) * P.pos_axis_stride + t);
    }
    if (APPEND) {
      row = __ldg(P.rows + t);
      seq = P.seqs ? __ldg(P.seqs + t) : static_cast<int32_t>(t);
    }
  };
  auto token_of = [&](int64_t unit) {
    return unit < P.whole ? unit : P.whole + static_cast<uint32_t>(unit - P.whole) / static_cast<uint32_t>(P.splits);
  };
  read_ahead(token_of(u));
  for (; u < P.units; u += stride) {
    const int64_t t = token_of(u);
    int h_begin = 0, h_end = P.heads;
    if (u >= P.whole) {
      h_begin = static_cast<int>(u - P.whole - (t - P.whole) * P.splits) * P.unit_heads;
      h_end = min(P.heads, h_begin + P.unit_heads);
    }
    int64_t off = -1;
    for (int c = c0;; c += 32) {
      const bool here = hs < P.head_slots && c < n, turns = c < P.n1;
      // this lane's elements of a head: first .. first + V, and the partner's
      const int first = turns ? (PAIRS && V == 1 ? 2 * c : c * V) : 2 * pairs + (c - P.n1) * V;
      const int partner = first + (PAIRS ? 1 : P.half_off);
      C lo[kRotUnroll], hi[kRotUnroll];
      auto load = [&](int hb) {
#pragma unroll
        for (int k = 0; k < kRotUnroll; ++k) {
          const int h = hb + k * P.head_slots;
          if (h >= h_end) continue;
          const uint8_t *src;
          if (!APPEND || h < P.q_heads) {
            src = P.x + t * P.xs + h * hd * static_cast<int>(sizeof(T));
          } else {
            const bool is_v = h >= P.rot_heads;
            src = (is_v ? P.v + t * P.vs : P.k + t * P.ks) + (h - (is_v ? P.rot_heads : P.q_heads)) * hd * static_cast<int>(sizeof(T));
          }
          const T *s = reinterpret_cast<const T *>(src);
          lo[k] = *reinterpret_cast<const C *>(s + first);
          if (kSplit && turns) hi[k] = *reinterpret_cast<const C *>(s + partner);
        }
      };
      int hb = h_begin + hs;
      if (here) load(hb);
      if (c == c0) {                                   // angles and slot of the token, once
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (lane + 32 * k < pairs) cs[lane + 32 * k] = angle(P, pos[k], freq[k], sign);
        if (APPEND && row >= 0) {
          if (static_cast<uint32_t>(seq) < static_cast<uint32_t>(P.pool.num_seqs)) off = P.pool.row_offset(seq, row);
          if (off < 0 && P.err && lane == 0) raise_device_error(P.err, APACK_EDEVICE, 71, seq, row);
        }
        read_ahead(token_of(u + stride));
        __syncwarp();
      }
      if (here) {
        float2 a[kAngles];
        if (turns) {
#pragma unroll
          for (int j = 0; j < kAngles; ++j) a[j] = cs[c * kAngles + j];
        }
        for (;;) {
#pragma unroll
          for (int k = 0; k < kRotUnroll; ++k) {
            const int h = hb + k * P.head_slots;
            if (h >= h_end) continue;
            uint8_t *dst;
            if (!APPEND || h < P.q_heads) {
              dst = P.out + t * P.outs + h * hd * static_cast<int>(sizeof(T));
            } else {
              const bool is_v = h >= P.rot_heads;
              if (off < 0) continue;
              dst = (is_v ? P.pool.v : P.pool.k) + off + (h - (is_v ? P.rot_heads : P.q_heads)) * P.pool.head_stride;
            }
            if (turns && h < P.rot_heads) turn<T, V, kSplit>(lo[k], hi[k], a);
            T *d = reinterpret_cast<T *>(dst);
            *reinterpret_cast<C *>(d + first) = lo[k];
            if (kSplit && turns) *reinterpret_cast<C *>(d + partner) = hi[k];
          }
          hb += kRotUnroll * P.head_slots;
          if (hb >= h_end) break;
          load(hb);
        }
      }
      if (c - c0 + 32 >= n) break;
    }
    __syncwarp();                                      // the angles are read
  }
}

template <class T, bool APPEND>
cudaError_t launch_rotary(RotPlan &P, bool pairs_layout, bool wide, float sign, cudaStream_t stream) {
  constexpr int W = 16 / sizeof(T);
  const int D = P.head_dim, r = 2 * P.pairs;
  const int V = wide ? W : 1;
  P.n1 = (pairs_layout && V > 1) ? r / V : r / 2 / V;
  P.n2 = (D - r) / V;
  P.half_off = r / 2;
  P.head_slots = 32 / std::min(P.n1 + P.n2, 32);
  // A warp per token as long as there is one for every warp of the grid; the tokens that are left over (or few) in
  // parts of their heads, down to those whose loads a lane has in flight at once.
  const int64_t warps = static_cast<int64_t>(kRotCtas) * (kRotThreads / 32) * device_sm_count();
  const int batch = P.head_slots * kRotUnroll, batches = (P.heads + batch - 1) / batch;
  P.whole = static_cast<int64_t>(P.n_tokens / warps) * warps;
  const int64_t rest = P.n_tokens - P.whole;
  P.splits = rest > 0 ? static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(batches, warps / rest))) : 1;
  P.unit_heads = ((P.heads + P.head_slots - 1) / P.head_slots + P.splits - 1) / P.splits * P.head_slots;
  P.splits = (P.heads + P.unit_heads - 1) / P.unit_heads;
  P.units = P.whole + rest * P.splits;
  const int64_t per = kRotThreads / 32;
  const int64_t grid = std::min<int64_t>((P.units + per - 1) / per, static_cast<int64_t>(kRotCtas) * device_sm_count());
  void (*fn)(RotPlan, float);
  if (wide)
    fn = pairs_layout ? rotary_kernel<T, W, true, APPEND> : rotary_kernel<T, W, false, APPEND>;
  else
    fn = pairs_layout ? rotary_kernel<T, 1, true, APPEND> : rotary_kernel<T, 1, false, APPEND>;
  const cudaError_t e = launch_pdl(fn, dim3(static_cast<unsigned>(grid)), dim3(kRotThreads), 0, stream, P, sign);
  if (e == cudaSuccess) count_launches(1);
  return e;
}

// f radians in turns, modulo one turn, in units of 2^-64.  A position multiplies its error by up to 2^31, so 53 bits are
// too few: 1/(2 pi) is taken as a sum of two doubles and the product with the first one whole (its rounding from an fma).
// Off by at most 2 units for |f| up to 2^40; a negative frequency is the two's complement of its opposite.
uint64_t turns_of(double f) {
  constexpr double kHigh = 0.15915494309189535, kLow = -9.839338337591243e-18;
  const double a = std::fabs(f), high = a * kHigh;
  double low = std::fma(a, kLow, std::fma(a, kHigh, -high));
  low -= std::floor(low + 0.5);
  constexpr double kUnit = 18446744073709551616.0;                       // 2^64
  double whole;                                                          // (modf: no difference that could become an fma)
  const uint64_t turns = static_cast<uint64_t>(std::modf(high, &whole) * kUnit) + static_cast<uint64_t>(std::llrint(low * kUnit));
  return f < 0 ? ~turns + 1 : turns;
}

apack_status plan_spec(const apack_rotary_spec *s, int32_t head_dim, RotPlan &P) {
  if (s->layout != APACK_ROTARY_HALF && s->layout != APACK_ROTARY_PAIRS) return APACK_EINVAL;
  if (s->rotary_dim < 2 || s->rotary_dim > head_dim || (s->rotary_dim & 1) || !s->freq_h) return APACK_EINVAL;
  if (s->num_axes < 1 || s->num_axes > 3 || !std::isfinite(s->magnitude)) return APACK_EINVAL;
  P.pairs = s->rotary_dim / 2;
  P.axis1 = P.axis2 = P.pairs;
  if (s->num_axes > 1) {
    int64_t sum = 0;
    for (int a = 0; a < s->num_axes; ++a) {
      if (s->section[a] < 0) return APACK_EINVAL;
      sum += s->section[a];
    }
    if (sum != P.pairs) return APACK_EINVAL;
    P.axis1 = s->section[0];
    if (s->num_axes > 2) P.axis2 = s->section[0] + s->section[1];
  }
  P.magnitude = s->magnitude;
  for (int i = 0; i < P.pairs; ++i) {
    if (!std::isfinite(s->freq_h[i])) return APACK_EINVAL;
    P.freq[i] = turns_of(s->freq_h[i]);
  }
  return APACK_OK;
}

bool aligned16(std::initializer_list<int64_t> v) {
  int64_t all = 0;
  for (int64_t x : v) all |= x;
  return (all & 15) == 0;
}
int64_t addr(const void *p) { return static_cast<int64_t>(reinterpret_cast<uintptr_t>(p)); }

// Chunks of 16 bytes fit the rotated part, its halves and the rest of the head.
bool wide_heads(int32_t rotary_dim, int32_t head_dim, int size) {
  const int w = 16 / size;
  return head_dim % w == 0 && rotary_dim % (2 * w) == 0;
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

apack_status apack_rotary_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor,
                                      int64_t original_len, double beta_fast, double beta_slow, double *freq_h,
                                      float *magnitude_h) {
  if (rotary_dim < 2 || rotary_dim > 2 * kMaxPairs || (rotary_dim & 1) || !freq_h || !magnitude_h) return APACK_EINVAL;
  if (!(base > 0) || !std::isfinite(base)) return APACK_EINVAL;
  if (scaling < APACK_ROTARY_NONE || scaling > APACK_ROTARY_YARN) return APACK_EINVAL;
  if (scaling != APACK_ROTARY_NONE && (!(factor >= 1) || !std::isfinite(factor))) return APACK_EINVAL;
  if (scaling == APACK_ROTARY_NTK && rotary_dim < 4) return APACK_EINVAL;
  if (scaling == APACK_ROTARY_YARN &&
      (original_len < 1 || !std::isfinite(beta_fast) || !(beta_slow >= 0) || !(beta_fast > beta_slow)))
    return APACK_EINVAL;
  const double r = rotary_dim;
  const double b = scaling == APACK_ROTARY_NTK ? base * std::pow(factor, r / (r - 2)) : base;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double f = std::pow(b, -2.0 * i / r);
    if (scaling == APACK_ROTARY_LINEAR) f /= factor;
    if (scaling == APACK_ROTARY_YARN) {
      const double turns = static_cast<double>(original_len) * f / 6.283185307179586476925286766559;
      const double g = std::min(1.0, std::max(0.0, (turns - beta_slow) / (beta_fast - beta_slow)));
      f = f * g + f / factor * (1 - g);
    }
    if (!std::isfinite(f)) return APACK_EINVAL;
    freq_h[i] = f;
  }
  *magnitude_h = scaling == APACK_ROTARY_YARN ? static_cast<float>(0.1 * std::log(factor) + 1.0) : 1.f;
  return APACK_OK;
}

apack_status apack_rotary(const apack_rotary_spec *spec, int32_t dtype, int64_t n_tokens, int32_t num_heads,
                          int32_t head_dim, const void *x, int64_t x_token_stride, void *out, int64_t out_token_stride,
                          const int32_t *positions, int64_t pos_axis_stride, int32_t transpose, void *stream) {
  if (!spec || n_tokens < 0 || n_tokens > INT32_MAX || num_heads < 1 || num_heads > (1 << 16)) return APACK_EINVAL;
  if (head_dim < 2 || head_dim > 2 * kMaxPairs || (head_dim & 1)) return APACK_EUNSUPPORTED;
  if (dtype != APACK_BF16 && dtype != APACK_FP16 && dtype != APACK_FP32) return APACK_EUNSUPPORTED;
  RotPlan P;
  std::memset(&P, 0, sizeof(P));
  const apack_status st = plan_spec(spec, head_dim, P);
  if (st != APACK_OK) return st;
  const int size = dtype == APACK_FP32 ? 4 : 2;
  const int64_t row = static_cast<int64_t>(num_heads) * head_dim * size;
  if (x_token_stride % size || out_token_stride % size || (n_tokens > 1 && (x_token_stride < row || out_token_stride < row)))
    return APACK_EINVAL;
  if (n_tokens == 0) return APACK_OK;
  if (!x || !out || !positions || addr(x) % size || addr(out) % size || (addr(positions) & 3)) return APACK_EINVAL;
  if (spec->num_axes > 1 && pos_axis_stride != 0 && pos_axis_stride < n_tokens) return APACK_EINVAL;
  if (!(x == out && (n_tokens == 1 || x_token_stride == out_token_stride)) &&
      rows_overlap(n_tokens, addr(x), x_token_stride, row, addr(out), out_token_stride, row))
    return APACK_EINVAL;
  P.heads = P.rot_heads = P.q_heads = num_heads;
  P.head_dim = head_dim;
  P.n_tokens = n_tokens;
  P.x = static_cast<const uint8_t *>(x);
  P.out = static_cast<uint8_t *>(out);
  P.xs = x_token_stride;
  P.outs = out_token_stride;
  P.positions = positions;
  P.pos_axis_stride = pos_axis_stride;
  const bool wide = wide_heads(spec->rotary_dim, head_dim, size) &&
                    aligned16({addr(x), addr(out), x_token_stride, out_token_stride});
  const bool pairs = spec->layout == APACK_ROTARY_PAIRS;
  const float sign = transpose ? -1.f : 1.f;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case APACK_BF16: return check_cuda(launch_rotary<__nv_bfloat16, false>(P, pairs, wide, sign, s));
    case APACK_FP16: return check_cuda(launch_rotary<__half, false>(P, pairs, wide, sign, s));
    default: return check_cuda(launch_rotary<float, false>(P, pairs, wide, sign, s));
  }
}

apack_status apack_rotary_append(const apack_rotary_spec *spec, const apack_paged_cache *cache, int32_t layer,
                                 int64_t n_tokens, const void *q, int64_t q_token_stride, void *q_out,
                                 int64_t q_out_token_stride, int32_t num_q_heads, const void *k,
                                 int64_t k_token_stride, const void *v, int64_t v_token_stride,
                                 const int32_t *positions, int64_t pos_axis_stride, const int32_t *rows,
                                 const int32_t *seqs, void *ws, void *stream) {
  apack_status st = validate_pool(cache, true);
  if (st != APACK_OK) return st;
  if (layer < 0 || layer >= cache->num_layers || n_tokens < 0 || n_tokens > INT32_MAX) return APACK_EINVAL;
  if (num_q_heads < 0 || num_q_heads > 1024 || (num_q_heads == 0) != (q == nullptr) || (!q) != (!q_out))
    return APACK_EINVAL;
  if (!seqs && n_tokens > cache->num_seqs) return APACK_EINVAL;
  RotPlan P;
  std::memset(&P, 0, sizeof(P));
  if (spec) {
    st = plan_spec(spec, cache->head_dim, P);
    if (st != APACK_OK) return st;
  }
  const int64_t head = cache->head_dim * 2;
  const int64_t qrow = num_q_heads * head, kvrow = cache->num_kv_heads * head;
  if (n_tokens == 0) return APACK_OK;
  if (!k || !v || !rows || (spec && !positions) ||
      !aligned16({addr(q), addr(q_out), addr(k), addr(v), q ? q_token_stride : 0, q ? q_out_token_stride : 0,
                  k_token_stride, v_token_stride}) ||
      ((addr(rows) | addr(seqs) | addr(positions) | addr(ws)) & 3))
    return APACK_EINVAL;
  if (n_tokens > 1 && ((q && (q_token_stride < qrow || q_out_token_stride < qrow)) || k_token_stride < kvrow ||
                       v_token_stride < kvrow))
    return APACK_EINVAL;
  auto q_out_over = [&](const void *p, int64_t stride, int64_t bytes) {
    return rows_overlap(n_tokens, addr(q_out), q_out_token_stride, qrow, addr(p), stride, bytes);
  };
  if (q && ((!(q == q_out && (n_tokens == 1 || q_token_stride == q_out_token_stride)) && q_out_over(q, q_token_stride, qrow)) ||
            q_out_over(k, k_token_stride, kvrow) || q_out_over(v, v_token_stride, kvrow)))
    return APACK_EINVAL;
  if (spec && spec->num_axes > 1 && pos_axis_stride != 0 && pos_axis_stride < n_tokens) return APACK_EINVAL;
  P.q_heads = num_q_heads;
  P.heads = num_q_heads + 2 * cache->num_kv_heads;
  P.rot_heads = num_q_heads + cache->num_kv_heads;
  P.head_dim = cache->head_dim;
  P.n_tokens = n_tokens;
  P.x = static_cast<const uint8_t *>(q);
  P.out = static_cast<uint8_t *>(q_out);
  P.k = static_cast<const uint8_t *>(k);
  P.v = static_cast<const uint8_t *>(v);
  P.xs = q_token_stride;
  P.outs = q_out_token_stride;
  P.ks = k_token_stride;
  P.vs = v_token_stride;
  P.positions = positions;
  P.pos_axis_stride = pos_axis_stride;
  P.rows = rows;
  P.seqs = seqs;
  P.pool = pool_view(cache, layer);
  P.err = static_cast<DeviceError *>(ws);
  const bool pairs = spec && spec->layout == APACK_ROTARY_PAIRS;
  const bool wide = wide_heads(2 * P.pairs, cache->head_dim, 2);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return check_cuda(cache->dtype == APACK_BF16 ? launch_rotary<__nv_bfloat16, true>(P, pairs, wide, 1.f, s)
                                               : launch_rotary<__half, true>(P, pairs, wide, 1.f, s));
}

}  // extern "C"
