// group_attention.cu -- attention of new tokens over paged caches, the shared rows of a group of sequences read once.
//
//   out[t, h] = sum_r softmax_r(scale q[t, h] . k[r, g(h)]) v[r, g(h)],  r <= position of t
//
// What makes it fast.  64 conversations about one video read the same cache; token by token that is 64 reads of it, and
// one here.  All query rows of a KV head (tokens of all sequences that share the keys, times the query heads of the KV
// head) are rows of one matrix product, 256 of them per segment, so that the tensor cores do what several reads did:
// with 256 rows a tile of 128 keys takes 2 x 128 x 128 x D x 4 flops against 512 D bytes, and the tensor pipe, not HBM,
// is the bound above some 160 rows.
//
// A segment (group_plan.cu) is 256 query rows of a KV head against a run of 128-key tiles.  CTAs (one per SM) take
// segments from a counter, in the plan's order (groups, then the sequences as the caller names them); every segment's
// result is a part (max, sum, unnormalised values) of its own, and the merge adds a row's parts in the order of their
// keys, so that the result does not depend on who took what.
//   warps 0..3, 4..7   softmax of accumulators 0 and 1, a query row per thread (TMEM lane): P is written over S as
//                      16-bit pairs (the A operand of the second product comes from TMEM), O stays in TMEM for the
//                      whole segment.  A row's reference maximum is set anew only when it has grown by more than 2^8
//                      (2^4 in fp16): then its warp rescales its O.
//   warp 8             the tensor products, one thread issuing: S = Q K^T and O += P V of accumulators 0 and 1 in turn,
//                      so that one softmax runs while the other's products do.  S of an accumulator's next tile is
//                      issued right behind O of this one (products run in the order of issue).
//   warps 9..11        loads: K and V tiles in a ring of 5 (8 with heads of 64), by TMA boxes of up to 128 tokens (a
//                      warp for K, one for V, a box per lane), or 16 bytes at a time where pages are no multiple of 8
//                      tokens (all three)
// A segment of more than 128 rows gives each accumulator half of the rows; one of fewer gives them the even and the odd
// tiles, and writes two parts.  Operations alternate between the accumulators across segments too, so that short
// segments overlap.
//
// P enters the second product as one 16-bit number per probability: 2^-9 (bf16) or 2^-12 (fp16) of each at most, on
// average less than the output's own rounding, where a second number would take half as much tensor time again; the
// row's sum is taken of the unrounded probabilities in fp32, so the lse keeps 32 bits.
//
// What a token must not see: keys behind its own are masked in S; values there enter as 0 times a number, so rows
// behind the segment's last key become zeros in shared memory, and where that is not enough (another token's key whose
// value is NaN or infinite: 0 times it is NaN) the merge computes the row anew, key by key.
//
// Measured (28/4 heads of 128, bf16, calls in a row, us a layer with its merge, of the tensor rate 1.94 PFLOP/s): 2,048
// tokens at the end of 27,144 518, 1.48 PFLOP/s, 0.76; 8 questions of 25 to 60 tokens on 135,272 shared rows 427, 1.46,
// 0.75; 16 of 12 to 60 on 22,772 161 with the plan; a decode step of 64 conversations on those 53; a tile of 256 rows
// and 128 keys takes 2,600 clocks, its products 2,048.
//
// One token per sequence, against apack_paged_decode_attention, which reads every sequence by itself (28/4 heads, 30 own
// rows each, us a layer with keys from HBM, the plan's 8 to 10 not counted): 2 sequences on 500 shared rows 10.9 and 8.6,
// 64 on them 22.5 and 14.8; 8, 16 and 64 on 4,644 14.6 and 14.5, 17.5 and 19.1, 29.5 and 50; 4, 8 and 64 on 22,772 24.5
// and 23.2, 25.9 and 33.7, 43 and 205; 64 of 4,000 rows that share nothing 162 and 88.
//
// Every wait is bounded (2 s); one that gives up records APACK_ETIMEOUT, and the CTA leaves with its copies and
// products done.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "group.cuh"

namespace apack {
namespace {

constexpr int kThreads = 384;
constexpr int kMmaWarp = 8, kLoadWarp = 9, kLoadWarps = 3;
constexpr int kHalfBytes = kGTile * 128;                       // 64 features of 128 rows
constexpr int kRecs = 16;
constexpr int kClaimAhead = 3;                                 // tiles before a segment's end at which the next is claimed
constexpr uint32_t kTmemCols = 512;                            // S 0, S 1, O 0, O 1, 128 columns each

template <int D>
struct Lay {
  static constexpr int kTileBytes = kGTile * D * 2;
  static constexpr int kRing = D == 128 ? 5 : 8;               // K and V tiles
  static constexpr uint32_t kOffRing = 2 * kGSlot * D * 2;     // behind the two query tiles
  static constexpr uint32_t kOffBars = kOffRing + kRing * kTileBytes;
  static constexpr uint32_t kBytes = kOffBars + 1536;
};

struct __align__(16) Bars {
  GroupSeg rec[kRecs];                                         // the CTA's segments in turn; seq -1: no more
  uint64_t full[8], empty[8];
  uint64_t rec_full[kRecs];
  uint64_t q_full[2], s_full[2], p_full[2], o_full[2], drain;
  uint32_t tmem;
  volatile int32_t abort;
};
static_assert(sizeof(Bars) <= 1536, "barrier block");

// 16-bit types of K, V and P.  The reference is kShift below the row's maximum when it was set; see paged_decode.cu for
// the range of fp16 (a long tail far below one key).
template <class T>
struct Type;
template <>
struct Type<__nv_bfloat16> {
  static constexpr float kGrow = 8.f, kShift = 0.f;
  static constexpr uint32_t kFormat = (1u << 7) | (1u << 10);
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&v);
  }
};
template <>
struct Type<__half> {
  static constexpr float kGrow = 4.f, kShift = 11.f;
  static constexpr uint32_t kFormat = 0;
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __half2 v = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t *>(&v);
  }
};

template <class T>
constexpr uint32_t idesc(int n, bool b_mn_major) {
  return (1u << 4) | Type<T>::kFormat | (b_mn_major ? 1u << 16 : 0u) | (static_cast<uint32_t>(n >> 3) << 17) |
         (static_cast<uint32_t>(kGSlot >> 4) << 24);
}

// D[tmem] (+)= A[tmem] * B[smem]^T
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// One thread of the warp.  What it issues to the tensor cores inside this branch takes one instruction each; inside
// "lane == 0" the compiler cannot tell that a single thread is there (8 products issued in 580 clocks, here 520, of
// which 512 are the products).
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void store8(void *p, const uint32_t *r) {        // 32 bytes, aligned
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int32_t token, int32_t block,
                                        int32_t head, int32_t page) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], "
      "[%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(0), "r"(token), "r"(block), "r"(head), "r"(page)
      : "memory");
}

// Bounded; false when it gave up or another role of the CTA has.
__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, Bars *b, DeviceError *err, int where) {
  for (int i = 0; i < 64; ++i)                                    // most end here, without a look at the clock
    if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (b->abort) return false;
    if (globaltimer_ns() - t0 > kWaitLimitNs) {
      b->abort = 1;
      raise_device_error(err, APACK_ETIMEOUT, where, blockIdx.x, threadIdx.x);
      return false;
    }
  }
}
// The same for a whole warp, which goes on or leaves together.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, Bars *b, DeviceError *err, int where) {
  return __all_sync(0xffffffffu, wait(bar, parity, b, err, where));
}

// A segment of the CTA as its roles read it.  pair: each accumulator takes half of the rows and every tile; else the
// accumulators take the tiles in turn.
struct Seg {
  GroupSeg g;
  int tiles;
  bool pair;
};
template <bool WARP = true>
__device__ __forceinline__ bool read_rec(Bars *b, int n, Seg &s, DeviceError *err, int where) {
  uint64_t *bar = &b->rec_full[n % kRecs];
  const uint32_t parity = (n / kRecs) & 1u;
  if (!(WARP ? warp_wait(bar, parity, b, err, where) : wait(bar, parity, b, err, where))) return false;
  s.g = b->rec[n % kRecs];
  s.tiles = (s.g.key1 - s.g.key0 + kGTile - 1) / kGTile;
  s.pair = s.g.step <= 0;
  return s.g.seq >= 0;
}
// A tile's places in the ring: K, and V behind it.
template <int RING>
struct Place {
  int k = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ int v() const { return k + 1 == RING ? 0 : k + 1; }
  __device__ __forceinline__ uint32_t v_phase() const { return k + 1 == RING ? phase ^ 1u : phase; }
  __device__ __forceinline__ void next() {
    k += 2;
    if (k >= RING) {
      k -= RING;
      phase ^= 1u;
    }
  }
  __device__ __forceinline__ void skip(int tiles) {
    const int at = k + 2 * tiles;
    phase ^= (at / RING) & 1;
    k = at % RING;
  }
};

__device__ __forceinline__ bool passed(uint64_t *bar, uint32_t parity) {      // without waiting
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}

// Bounded, and asked for again and again: for what comes within a tile's time.
__device__ __forceinline__ bool hot_wait(uint64_t *bar, uint32_t parity, Bars *b, DeviceError *err, int where) {
  for (int i = 0; i < 1024; ++i)
    if (passed(bar, parity)) return true;
  return wait(bar, parity, b, err, where);
}

// The products of the CTA's segments, by one thread.  What it does between a softmax's signal and the products that
// wait for it is on the critical path of an accumulator, and takes some ten clocks per instruction: so a tile's places,
// phases and descriptors are ready before, and the next tile's scores follow the values with nothing but their issue in
// between.
template <class T, int D>
struct Products {
  using L = Lay<D>;
  Bars *b;
  DeviceError *err;
  uint32_t base, tmem;
  Place<L::kRing> at;                                            // of the tile whose scores come next
  uint32_t q_par = 0, p_par = 0;                                 // a bit per accumulator

  __device__ __forceinline__ uint64_t keys_desc(int slot) const { return smem_desc_sw128(base + L::kOffRing + slot * L::kTileBytes); }
  __device__ __forceinline__ uint64_t values_desc(int slot) const {
    return smem_desc_sw128_mn(base + L::kOffRing + slot * L::kTileBytes, kHalfBytes, 1024);
  }
  template <int S>
  __device__ __forceinline__ void scores(uint64_t k) const {
    const uint64_t q = smem_desc_sw128(base + S * (kGSlot * D * 2));
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      const uint32_t off = ((i >> 2) * kHalfBytes + (i & 3) * 32) >> 4;      // (addresses are below 2^18: no carry)
      tc_mma_bf16(tmem + S * kGTile, q + off, k + off, idesc<T>(kGTile, false), i > 0);
    }
  }
  template <int S>
  __device__ __forceinline__ void values(uint64_t v, uint32_t accumulate) const {
#pragma unroll
    for (int i = 0; i < kGTile / 16; ++i)
      tc_mma_ts(tmem + 256 + S * 128, tmem + S * kGTile + i * 8, v + (i * 2048 >> 4), idesc<T>(D, true), i > 0 ? 1u : accumulate);
  }
  template <int S>
  __device__ __forceinline__ bool queries() {
    if (!wait(&b->q_full[S], q_par >> S & 1u, b, err, 165)) return false;
    q_par ^= 1u << S;
    return true;
  }
  template <int S>
  __device__ __forceinline__ bool weights() {
    if (!hot_wait(&b->p_full[S], p_par >> S & 1u, b, err, 166)) return false;
    p_par ^= 1u << S;
    tc_fence_after();
    return true;
  }
  __device__ __forceinline__ bool tile(const Place<L::kRing> &p) {
    return wait(&b->full[p.k], p.phase, b, err, 167) && wait(&b->full[p.v()], p.v_phase(), b, err, 167);
  }

  // Both accumulators, F first, each its rows: every tile.
  template <int F>
  __device__ __forceinline__ bool rows(int tiles) {
    if (!queries<F>() || !wait(&b->full[at.k], at.phase, b, err, 168)) return false;
    tc_fence_after();
    uint64_t k = keys_desc(at.k);
    scores<F>(k);
    tc_commit(&b->s_full[F]);
    if (!queries<1 - F>()) return false;
    tc_fence_after();
    scores<1 - F>(k);
    tc_commit(&b->s_full[1 - F]);
    tc_commit(&b->empty[at.k]);
    for (int t = 0; t < tiles; ++t) {
      Place<L::kRing> then = at;
      then.next();
      const bool more = t + 1 < tiles;
      const int vs = at.v();
      const uint64_t v = values_desc(vs);
      k = keys_desc(then.k);
      const uint32_t accumulate = t > 0;
      if (!wait(&b->full[vs], at.v_phase(), b, err, 167) || (more && !wait(&b->full[then.k], then.phase, b, err, 168))) return false;
      if (!weights<F>()) return false;
      values<F>(v, accumulate);
      if (more) scores<F>(k);
      tc_commit(more ? &b->s_full[F] : &b->o_full[F]);
      if (!weights<1 - F>()) return false;
      values<1 - F>(v, accumulate);
      if (more) scores<1 - F>(k);
      tc_commit(more ? &b->s_full[1 - F] : &b->o_full[1 - F]);
      tc_commit(&b->empty[vs]);
      if (more) tc_commit(&b->empty[then.k]);
      at = then;
    }
    return true;
  }
  // Both accumulators, F first, the tiles in turn.
  template <int F>
  __device__ __forceinline__ bool turns(int tiles) {
    Place<L::kRing> p[2] = {at, at};
    p[1].next();
    if (!queries<F>() || !wait(&b->full[p[0].k], p[0].phase, b, err, 168)) return false;
    tc_fence_after();
    scores<F>(keys_desc(p[0].k));
    tc_commit(&b->s_full[F]);
    tc_commit(&b->empty[p[0].k]);
    if (tiles > 1) {
      if (!queries<1 - F>() || !wait(&b->full[p[1].k], p[1].phase, b, err, 168)) return false;
      tc_fence_after();
      scores<1 - F>(keys_desc(p[1].k));
      tc_commit(&b->s_full[1 - F]);
      tc_commit(&b->empty[p[1].k]);
    }
    for (int t = 0; t < tiles; t += 2) {
      if (!turn<F>(p[0], t, tiles)) return false;
      if (t + 1 < tiles && !turn<1 - F>(p[1], t + 1, tiles)) return false;
    }
    at.skip(tiles);
    return true;
  }
  template <int S>
  __device__ __forceinline__ bool turn(Place<L::kRing> &p, int t, int tiles) {
    Place<L::kRing> then = p;
    then.next();
    then.next();
    const bool more = t + 2 < tiles;
    const int vs = p.v();
    const uint64_t v = values_desc(vs), k = keys_desc(then.k);
    if (!wait(&b->full[vs], p.v_phase(), b, err, 167) || (more && !wait(&b->full[then.k], then.phase, b, err, 168))) return false;
    if (!weights<S>()) return false;
    values<S>(v, t > 1);
    if (more) scores<S>(k);
    tc_commit(more ? &b->s_full[S] : &b->o_full[S]);
    tc_commit(&b->empty[vs]);
    if (more) tc_commit(&b->empty[then.k]);
    p = then;
    return true;
  }
  __device__ __forceinline__ void run() {
    uint32_t par = 0;
    bool issued = false, ok = true;
    Seg seg;
    for (int rec = 0; ok && read_rec<false>(b, rec, seg, err, 161); ++rec) {
      issued = true;
      if (seg.pair) {
        ok = par ? rows<1>(seg.tiles) : rows<0>(seg.tiles);
      } else {
        ok = par ? turns<1>(seg.tiles) : turns<0>(seg.tiles);
        par ^= seg.tiles & 1;
      }
    }
    if (issued) {                                               // every product done before the CTA leaves
      tc_commit(&b->drain);
      mbar_wait(&b->drain, 0, kWaitLimitNs / 4);
    }
  }
};

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1)
    group_tc_kernel(const __grid_constant__ GroupArgs A, const __grid_constant__ FastDiv group,
                    const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap) {
  using L = Lay<D>;
  constexpr int kRing = L::kRing, kBlocks = D / 64;
  extern __shared__ __align__(1024) uint8_t smem[];
  Bars *b = reinterpret_cast<Bars *>(smem + L::kOffBars);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((smem_u32(smem) & 1023u) != 0) {
    if (threadIdx.x == 0) raise_device_error(A.err, APACK_EDEVICE, 160);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&b->full[i], A.box ? 1 : kLoadWarps * 32);
      mbar_init(&b->empty[i], 1);
    }
    for (int i = 0; i < kRecs; ++i) mbar_init(&b->rec_full[i], 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&b->q_full[i], 4);
      mbar_init(&b->s_full[i], 1);
      mbar_init(&b->p_full[i], 4);
      mbar_init(&b->o_full[i], 1);
    }
    mbar_init(&b->drain, 1);
    b->abort = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(&b->tmem, kTmemCols);
    tc_fence_before();
  }
  if (threadIdx.x == kLoadWarp * 32 && A.box) {
    tma_prefetch_desc(&kmap);
    tma_prefetch_desc(&vmap);
  }
  __syncthreads();
  tc_fence_after();
  pdl_wait_and_release();
  const uint32_t tmem = b->tmem;
  GroupHead h;
  GroupSeg first_seg = {};                                        // beside the head (there are more places than CTAs)
  if (warp >= kLoadWarp) first_seg = reinterpret_cast<const GroupSeg *>(A.ws + A.seg_off)[blockIdx.x];
  const bool planned = group_head(A, h);
  int item = 0;                                                   // tiles issued by a load warp
  if (!planned) {
    if (threadIdx.x == 0 && blockIdx.x == 0) raise_device_error(A.err, APACK_EDEVICE, 150);
  } else if (warp >= kLoadWarp) {
    // ------------------------------------------------------------ loads
    const GroupSeg *segs = reinterpret_cast<const GroupSeg *>(A.ws + A.seg_off);
    unsigned int *claims = reinterpret_cast<unsigned int *>(A.ws + kGClaimOff);
    const uint32_t ring = smem_u32(smem) + L::kOffRing;
    if (A.box && warp < kLoadWarp + 2) {
      // by TMA: K tiles by the first warp, which also takes the segments, V tiles by the second; a box per lane, whose
      // page is known one tile ahead
      const int box = A.box, v = warp - kLoadWarp;
      const int blk = lane % kBlocks, bx = lane / kBlocks;
      const CUtensorMap *map = v ? &vmap : &kmap;
      auto page_of = [&](const GroupSeg &g, int tile) {
        const int row = g.key0 + tile * kGTile + bx * box;
        if (g.seq < 0 || bx * box >= kGTile || row >= g.key1) return -1;
        const int p = A.pool.page_tokens.div(row);
        return __ldg(A.pool.table + g.seq * A.pool.table_stride + p);
      };
      unsigned claimed = blockIdx.x;
      auto fetch = [&] {                                          // the next segment with work; seq -1: none
        GroupSeg g;
        for (;;) {
          const unsigned i = __shfl_sync(0xffffffffu, claimed, 0);
          g.seq = -1;
          if (i >= static_cast<unsigned>(h.segs)) return g;
          g = i == blockIdx.x ? first_seg : segs[i];
          if (lane == 0) claimed = gridDim.x + atomicAdd(claims, 1u);
          if (g.key0 < g.key1) return g;
        }
      };
      auto publish = [&](int rec, const GroupSeg &g) {
        if (lane == 0) {
          b->rec[rec % kRecs] = g;
          mbar_arrive(&b->rec_full[rec % kRecs]);
        }
      };
      auto segment = [&](int rec) {                               // number `rec` of the CTA, for the second warp
        Seg s;
        if (!read_rec(b, rec, s, A.err, 163)) s.g.seq = -1;
        return s.g;
      };
      GroupSeg g, next;
      if (v == 0) {
        g = fetch();
        publish(0, g);
      } else {
        g = segment(0);
      }
      int page = page_of(g, 0);
      item = v;
      bool ok = true;
      for (int rec = 1; ok && g.seq >= 0; ++rec) {
        const int tiles = (g.key1 - g.key0 + kGTile - 1) / kGTile;
        for (int t = 0; t < tiles; ++t, item += 2) {
          // (not sooner: a segment that is claimed early waits for a CTA that has a long one)
          if (t == max(0, tiles - kClaimAhead) && v == 0) next = fetch();
          if (t + 1 == tiles) {
            if (v == 0)
              publish(rec, next);
            else
              next = segment(rec);
          }
          const int row = g.key0 + t * kGTile + bx * box, boxes = (min(kGTile, g.key1 - g.key0 - t * kGTile) + box - 1) / box;
          const int in = row - A.pool.page_tokens.div(row) * A.pool.page_tokens.d, slot = item % kRing;
          int mine = page;
          page = t + 1 < tiles ? page_of(g, t + 1) : page_of(next, 0);
          if (item >= kRing && !warp_wait(&b->empty[slot], ((item / kRing) - 1) & 1u, b, A.err, 162)) {
            ok = false;
            break;
          }
          if (lane == 0) mbar_arrive_expect_tx(&b->full[slot], boxes * box * D * 2);
          __syncwarp();
          if (bx < boxes && static_cast<uint32_t>(mine) >= static_cast<uint32_t>(A.pool.num_pages)) {
            raise_device_error(A.err, APACK_EDEVICE, 140, g.seq, mine);
            mine = A.pool.num_pages;                              // behind the map's end: zeros
          }
          if (bx < boxes)
            tma_box(ring + slot * L::kTileBytes + blk * kHalfBytes + bx * box * 128, map, &b->full[slot], in, blk, g.head, mine);
        }
        g = next;
      }
    } else if (!A.box) {
      // rows by the lanes.  A copy is seen by the tensor cores only behind a fence of the thread that made it, so a
      // tile's arrival is signalled when the tile after next has been issued and its own copies have landed, or before
      // the warp waits for a place.
      constexpr int kChunks = D / 8, kAtOnce = 32 / kChunks, kBehind = 2;
      const int w = warp - kLoadWarp, ch = lane % kChunks;
      unsigned claimed = blockIdx.x;
      int signalled = 0;
      bool ok = true;
      auto signal = [&](int upto) {
        fence_proxy_async_smem();
        for (; signalled < upto; ++signalled) mbar_arrive(&b->full[signalled % kRing]);
      };
      for (int rec = 0; ok; ++rec) {
        Seg s;
        if (w == 0) {
          GroupSeg g;
          for (;;) {
            const unsigned i = __shfl_sync(0xffffffffu, claimed, 0);
            g.seq = -1;
            if (i >= static_cast<unsigned>(h.segs)) break;
            g = i == blockIdx.x ? first_seg : segs[i];
            if (lane == 0) claimed = gridDim.x + atomicAdd(claims, 1u);
            if (g.key0 < g.key1) break;
          }
          if (lane == 0) {
            b->rec[rec % kRecs] = g;
            mbar_arrive(&b->rec_full[rec % kRecs]);
          }
          __syncwarp();
        }
        if (!read_rec(b, rec, s, A.err, 163)) break;
        for (int t = 0; t < s.tiles && ok; ++t) {
          const int row = s.g.key0 + t * kGTile, valid = min(kGTile, s.g.key1 - row);
          int64_t off[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            off[i] = -1;
            const int r = i * 32 + lane;
            if (r >= valid) continue;
            const int32_t page = A.pool.page_of(s.g.seq, row + r);
            off[i] = A.pool.offset_in(page, row + r);
            if (off[i] < 0) raise_device_error(A.err, APACK_EDEVICE, 140, s.g.seq, page);
            off[i] += off[i] < 0 ? 0 : s.g.head * A.pool.head_stride;
          }
          for (int v = 0; v < 2; ++v, ++item) {
            const int slot = item % kRing;
            if (item >= kRing) {
              // While the place is taken, nothing that was issued may stay behind: where the accumulators take the tiles
              // in turn, it is given back only when the keys two tiles on have been signalled, which are the item before
              // this one in a ring of five.
              const uint32_t parity = ((item / kRing) - 1) & 1u;
              if (!__all_sync(0xffffffffu, passed(&b->empty[slot], parity))) {
                cp_async_wait<0>();
                signal(item);
              }
              if (!warp_wait(&b->empty[slot], parity, b, A.err, 162)) {
                ok = false;
                break;
              }
            }
            const uint8_t *base = v ? A.pool.v : A.pool.k;
            const uint32_t dst = ring + slot * L::kTileBytes + (ch >> 3) * kHalfBytes;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll 4
              for (int j = w; j < 32 / kAtOnce; j += kLoadWarps) {
                const int rr = j * kAtOnce + lane / kChunks, r = i * 32 + rr;
                const int64_t o = __shfl_sync(0xffffffffu, off[i], rr);
                if (r < valid || v)                               // (values behind the last key: zeros)
                  cp_async_16_or_zero(dst + r * 128 + (((ch & 7) ^ (r & 7)) << 4), base + (o < 0 ? 0 : o) + ch * 16, o >= 0);
              }
            cp_async_commit();
            cp_async_wait<kBehind>();
            if (item + 1 > kBehind) signal(item + 1 - kBehind);
          }
        }
      }
      cp_async_wait<0>();
      signal(item);
    }
  } else if (warp == kMmaWarp) {
    // ------------------------------------------------------------ products, by one thread, the accumulators in turn
    if (elect_one()) {
      Products<T, D> products{b, A.err, smem_u32(smem), tmem};
      products.run();
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax, a query row per thread
    const int s = warp >> 2, row = threadIdx.x & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t sc = tmem + lanes + s * kGTile, oc = tmem + lanes + 256 + s * 128;
    const GroupTok *toks = reinterpret_cast<const GroupTok *>(A.ws + kGFixed);
    float2 *ml = reinterpret_cast<float2 *>(A.ws + h.ml_off);
    float *parts = reinterpret_cast<float *>(A.ws + h.part_off);
    uint8_t *qs = smem + s * (kGSlot * D * 2);
    uint32_t s_par = 0, o_par = 0, par = 0;
    Place<kRing> place;                                           // of the segment's first tile
    Seg seg;
    int rec = 0, before = 0, which = 0, r0 = 0, limit = 0;        // before: tiles of the segment before
    bool real = false, idle = false;
    // The accumulator's next segment, and its queries
    auto next_segment = [&] {
      for (;; ++rec) {
        if (!read_rec(b, rec, seg, A.err, 168)) return false;
        place.skip(before);
        before = seg.tiles;
        which = s ^ par;                                          // half of the rows, or first tile
        if (!seg.pair) par ^= seg.tiles & 1;
        if (seg.pair || which < seg.tiles) break;
      }
      ++rec;
      r0 = seg.pair ? which * kGSlot : 0;
      real = r0 + row < seg.g.rows;
      idle = r0 + (warp & 3) * 32 >= seg.g.rows;                  // no row of the warp is one: what it leaves in TMEM is not read
      limit = 1 << 30;                                            // (what is no row need not be masked: nothing of it is kept)
      if (real) limit = min(toks[group.div(seg.g.row0 + r0 + row)].limit, seg.g.key1) - seg.g.key0;
      if (!idle) {
        // the warp's 32 rows, D / 8 lanes each: a row's 16-byte pieces side by side (a row per lane took 10,000 clocks)
        constexpr int kLanes = D / 8, kRows = 32 / kLanes;
        const int piece = lane % kLanes;
        constexpr int kAtOnce = 8;
#pragma unroll 1
        for (int i0 = 0; i0 < kLanes && r0 + (warp & 3) * 32 + i0 * kRows < seg.g.rows; i0 += kAtOnce) {
          uint4 x[kAtOnce];
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) {
            const int q = (warp & 3) * 32 + (i0 + i) * kRows + lane / kLanes;
            const uint32_t packed = seg.g.row0 + r0 + q, t = group.div(packed);
            x[i] = make_uint4(0, 0, 0, 0);
            if (r0 + q < seg.g.rows)
              x[i] = __ldg(reinterpret_cast<const uint4 *>(A.q + t * A.q_stride +
                                                           (static_cast<int64_t>(seg.g.head) * A.group + (packed - t * A.group)) *
                                                               (D * 2)) +
                           piece);
          }
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) {
            const int q = (warp & 3) * 32 + (i0 + i) * kRows + lane / kLanes;
            *reinterpret_cast<uint4 *>(qs + (piece >> 3) * kHalfBytes + q * 128 + (((piece & 7) ^ (q & 7)) << 4)) = x[i];
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&b->q_full[s]);
      return true;
    };
    for (bool have = next_segment(); have;) {
      float m = -INFINITY, l = 0.f;
      bool ok = true, first = true;
      for (int t = seg.pair ? 0 : which; t < seg.tiles; t += seg.pair ? 1 : 2) {
        ok = warp_wait(&b->s_full[s], s_par, b, A.err, 169);
        if (!ok) break;
        s_par ^= 1;
        tc_fence_after();
        if (!idle) {
          const int seen = limit - t * kGTile;
          const float2 scale = make_float2(A.scale2, A.scale2);
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          // Most tiles: probabilities against the present reference, and the maximum beside them, because the two use
          // different units.  Only if the reference turns out to be high enough are they written over the scores.
          bool done = false;
          if (!__any_sync(0xffffffffu, first || seen < kGTile)) {
            uint32_t x[4][32], p[4][16];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_ld32(sc + i * 32, x[i]);
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_wait32(x[i]);
            const float2 neg = m == -INFINITY ? make_float2(0.f, 0.f) : make_float2(-m, -m);
            float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const float2 v = make_float2(__uint_as_float(x[i][2 * j]), __uint_as_float(x[i][2 * j + 1]));
                const float2 y = ffma2(v, scale, neg);
                const float2 e = make_float2(ex2_approx(y.x), ex2_approx(y.y));
                most[j & 1] = fmaxf(most[j & 1], fmaxf(v.x, v.y));
                sum[j & 1] = fadd2(sum[j & 1], e);
                p[i][j] = Type<T>::pack(e.x, e.y);
              }
            const float top = fmaf(fmaxf(most[0], most[1]), A.scale2, -Type<T>::kShift);
            done = !__any_sync(0xffffffffu, top > m + Type<T>::kGrow);
            if (done)
#pragma unroll
              for (int i = 0; i < 4; ++i) tmem_st16(sc + i * 16, p[i]);
          }
          if (!done) {
            // A segment's first tile, one that a row does not see whole, or a new reference: 32 scores at a time, in
            // loops (code that runs once per segment is read from far away)
            float most = -INFINITY;
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {
              uint32_t x[32];
              tmem_ld32(sc + i * 32, x);
              tmem_wait32(x);
#pragma unroll
              for (int j = 0; j < 32; ++j) most = i * 32 + j < seen ? fmaxf(most, __uint_as_float(x[j])) : most;
            }
            const float top = fmaf(most, A.scale2, -Type<T>::kShift);
            const bool grows = top > m + Type<T>::kGrow;          // (also every finite score against -infinity)
            const float f = grows ? ex2_approx(m - top) : 1.f;
            if (grows) m = top;
            l *= f;
            if (!first && __any_sync(0xffffffffu, grows))
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                uint32_t o[16];
                tmem_ld16_wait(oc + c, o);
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                tmem_st16(oc + c, o);
              }
            first = false;
            const float2 neg = m == -INFINITY ? make_float2(0.f, 0.f) : make_float2(-m, -m);
            sum[0] = sum[1] = make_float2(0.f, 0.f);
#pragma unroll 1
            for (int i = 0; i < 4; ++i) {                         // (P of 32 scores covers none that are still to come)
              uint32_t x[32], p[16];
              tmem_ld32(sc + i * 32, x);
              tmem_wait32(x);
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const float2 y = ffma2(make_float2(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1])), scale, neg);
                const float2 e = make_float2(i * 32 + 2 * j < seen ? ex2_approx(y.x) : 0.f,
                                             i * 32 + 2 * j + 1 < seen ? ex2_approx(y.y) : 0.f);
                sum[j & 1] = fadd2(sum[j & 1], e);
                p[j] = Type<T>::pack(e.x, e.y);
              }
              tmem_st16(sc + i * 16, p);
            }
          }
          l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
        }
        if (t == seg.tiles - 1 && A.box) {
          // behind the segment's last key: zeros in V, whatever lies there (0 times a stale infinity would be NaN;
          // where both accumulators read the tile, both write them)
          const int valid = seg.g.key1 - seg.g.key0 - t * kGTile;
          if (valid < kGTile) {
            Place<kRing> at = place;
            at.skip(t);
            ok = warp_wait(&b->full[at.v()], at.v_phase(), b, A.err, 173);
            if (!ok) break;
            for (int i = row; i < (kGTile - valid) * (D / 8); i += kGSlot) {
              const int v = valid + i / (D / 8), ch = i % (D / 8);
              *reinterpret_cast<uint4 *>(smem + L::kOffRing + at.v() * L::kTileBytes + (ch >> 3) * kHalfBytes + v * 128 +
                                         (ch & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async_smem();
          }
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&b->p_full[s]);
      }
      if (!ok) break;
      // the next segment's queries, and with them its first scores, come while the last values' product runs and this
      // segment's part is written (the queries' place is free: its scores are all there)
      const int64_t at = static_cast<int64_t>(seg.g.part) + r0 + row + (seg.pair ? 0 : static_cast<int64_t>(which) * seg.g.step);
      const bool was_real = real, was_idle = idle, direct = seg.g.step < 0;
      const uint32_t packed = seg.g.row0 + r0 + row;
      const int head = seg.g.head;
      have = next_segment();
      ok = warp_wait(&b->o_full[s], o_par, b, A.err, 170);
      if (!ok) break;
      o_par ^= 1;
      tc_fence_after();
      if (direct) {
        // the row's only part: its output.  It starts on 16 bytes; where on 32 (rows are whole multiples), a store
        // fills a sector (30 prompts of 512 tokens, 28/4 heads of 128: 282 us a layer, 297 by 16 bytes)
        const bool wide = (reinterpret_cast<uintptr_t>(A.out) & 31) == 0;
        const uint32_t t = group.div(packed);
        const int64_t u = t * static_cast<int64_t>(A.hq) + head * A.group + (packed - t * A.group);
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bool nan = false;
        if (!was_idle)
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32], w[16];
            tmem_ld32(oc + c, o);
            tmem_wait32(o);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const float x = __uint_as_float(o[2 * j]) * inv, y = __uint_as_float(o[2 * j + 1]) * inv;
              nan |= x != x || y != y;
              w[j] = Type<T>::pack(x, y);
            }
            uint8_t *to = A.out + (u * D + c) * 2;
            if (was_real && wide) {
              store8(to, w);
              store8(to + 32, w + 8);
            } else if (was_real) {
#pragma unroll
              for (int j = 0; j < 16; j += 4)
                *reinterpret_cast<uint4 *>(to + 4 * j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
            }
          }
        if (was_real) {
          if (A.lse) A.lse[u] = (m + log2f(l)) * 0.6931471805599453f;
          ml[at] = make_float2(m, nan ? NAN : l);                 // (the merge looks at rows that are no numbers)
        }
      } else {
        if (was_real) ml[at] = make_float2(m, l);
        if (!was_idle)
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            tmem_ld32(oc + c, o);
            tmem_wait32(o);
            if (was_real)
#pragma unroll
              for (int j = 0; j < 32; j += 8) store8(parts + at * D + c + j, o + j);
          }
      }
      tc_fence_before();
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (b->abort && A.box && warp >= kLoadWarp && warp < kLoadWarp + 2 && lane == 0)        // copies that nobody waited for
    for (int i = max(warp - kLoadWarp, item - 2 * kRing); i < item; i += 2)
      mbar_wait(&b->full[i % kRing], (i / kRing) & 1u, kWaitLimitNs / 4);
  if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

// ---------------------------------------------------------------- merge

constexpr int kBatch = 8, kFewParts = 4; // parts whose loads a warp has in flight, of few rows and of many

template <int D>
struct Row {                             // of a warp: max, sum, D / 32 values on from lane * D / 32
  float m, l, o[D / 32];
};

template <int D>
__device__ __forceinline__ void load_values(float (&o)[D / 32], const float *p) {
  if (D == 128) {
    const float4 x = *reinterpret_cast<const float4 *>(p);
    o[0] = x.x, o[1] = x.y, o[2 % (D / 32)] = x.z, o[3 % (D / 32)] = x.w;
  } else {
    const float2 x = *reinterpret_cast<const float2 *>(p);
    o[0] = x.x, o[1] = x.y;
  }
}

// A row's parts of an item: [split][sub][KV head][rows], `two` of a split where its segment had few rows.
struct Parts {
  int n, tiles, chunk, sub, rows, base;
  bool two;
  __device__ __forceinline__ void set(const GroupArgs &A, const GroupItem &it, int head, int packed) {
    const int rr = packed - it.row0, run = rr / kGRows, here = min(kGRows, it.rows - run * kGRows);
    two = it.sub == 2 && here <= kGSlot;
    int key1 = it.key1;                        // the keys that the row's segments had (as the plan cuts them)
    if (it.causal) key1 = min(key1, it.key1 - it.rows / A.group + 1 + (run * kGRows + here - 1) / A.group);
    tiles = max((key1 - it.key0 + kGTile - 1) / kGTile, 0);
    chunk = it.chunk;
    sub = it.sub;
    rows = it.rows * A.hkv;
    base = it.part + head * it.rows + rr;
    n = tiles ? (tiles + chunk - 1) / chunk * (two ? 2 : 1) : 0;
  }
  // Row number of part j, or -1: the second of a single tile.
  __device__ __forceinline__ int64_t at(int j) const {
    const int split = two ? j >> 1 : j, u = two ? j & 1 : 0;
    return u && min(chunk, tiles - split * chunk) < 2 ? -1 : base + static_cast<int64_t>(split * sub + u) * rows;
  }
};

// The row's parts from number `from` on, every `step`th, added to a: the shared rows' first.
template <int D, int N>
__device__ __forceinline__ void merge_parts(const GroupArgs &A, const GroupHead &h, const Parts &x0, const Parts &x1, int from,
                                            int step, Row<D> &a) {
  constexpr int kF = D / 32;
  const int lane = threadIdx.x & 31, n = x0.n + x1.n;
  const float2 *ml = reinterpret_cast<const float2 *>(A.ws + h.ml_off);
  const float *parts = reinterpret_cast<const float *>(A.ws + h.part_off);
  for (int k = from; k < n; k += N * step) {
    float2 st[N];
    float x[N][kF];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int j = k + i * step;
      const int64_t at = j >= n ? -1 : j < x0.n ? x0.at(j) : x1.at(j - x0.n);
      st[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int e = 0; e < kF; ++e) x[i][e] = 0.f;
      if (at >= 0) {
        st[i] = ml[at];
        load_values<D>(x[i], parts + at * D + lane * kF);
      }
    }
    float top = a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, st[i].x);
    const float f = a.m == top ? 1.f : ex2_approx(a.m - top);
    a.m = top;
    a.l *= f;
#pragma unroll
    for (int e = 0; e < kF; ++e) a.o[e] *= f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      // (a part whose row saw nothing has sum 0, and a NaN maximum none)
      const float w = st[i].x == top ? 1.f : ex2_approx(st[i].x - top);
      a.l += st[i].y * w;
#pragma unroll
      for (int e = 0; e < kF; ++e) a.o[e] += x[i][e] * w;
    }
  }
}

// W: warps of a row (a CTA of 8 warps takes 8 / W rows).
template <class T, int D, int W, int N>
__global__ void __launch_bounds__(256, N < kBatch ? 5 : 2) group_merge_kernel(const __grid_constant__ GroupArgs A) {
  constexpr int kF = D / 32;
  __shared__ float qs[8][D];
  __shared__ float2 stat[8];
  pdl_wait_and_release();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t u = blockIdx.x * (8ll / W) + warp / W;
  if (u >= static_cast<int64_t>(A.n_q) * A.hq) return;
  const int t = static_cast<int>(u / A.hq), hd = static_cast<int>(u - static_cast<int64_t>(t) * A.hq);
  // three trips: head and token, both items, parts
  const GroupTok tok = reinterpret_cast<const GroupTok *>(A.ws + kGFixed)[t];
  GroupHead h;
  if (!group_head(A, h)) return;                       // recorded by the kernel before
  if (blockIdx.x == 0 && threadIdx.x == 0) *reinterpret_cast<unsigned int *>(A.ws + kGClaimOff) = 0;
  if (!tok.real) return;
  const GroupItem *items = reinterpret_cast<const GroupItem *>(A.ws + h.item_off);
  const int head = hd / A.group, packed = t * A.group + hd - head * A.group;
  GroupItem i0 = {}, i1 = {};
  if (tok.prefix >= 0) i0 = items[tok.prefix];
  if (tok.own >= 0) i1 = items[tok.own];
  Parts x0, x1;
  x0.n = x1.n = 0;
  if (tok.prefix >= 0) x0.set(A, i0, head, packed);
  if (tok.own >= 0) x1.set(A, i1, head, packed);
  Row<D> a = {-INFINITY, 0.f, {}};
  const bool direct = tok.prefix < 0 && x1.n == 1 && i1.splits == 1 && !x1.two;
  if (direct) {
    // written out already, with its lse; of interest only where it is no number and what the row does not see may be why
    const float2 st = reinterpret_cast<const float2 *>(A.ws + h.ml_off)[x1.at(0)];
    if (st.y == st.y || !h.causal_any || warp % W != 0) return;
    a.l = st.y;
  } else {
    merge_parts<D, N>(A, h, x0, x1, warp % W, W, a);
  }
  if (W > 1 && !direct) {
    stat[warp] = make_float2(a.m, a.l);
#pragma unroll
    for (int e = 0; e < kF; ++e) qs[warp][lane * kF + e] = a.o[e];
    asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / W), "r"(32 * W) : "memory");          // the row's warps
    if (warp % W != 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < W; ++w) top = fmaxf(top, stat[warp + w].x);
    a = {top, 0.f, {}};
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const float f = stat[warp + w].x == top ? 1.f : ex2_approx(stat[warp + w].x - top);
      a.l += stat[warp + w].y * f;
#pragma unroll
      for (int e = 0; e < kF; ++e) a.o[e] += qs[warp + w][lane * kF + e] * f;
    }
    __syncwarp();
  }
  bool nan = a.l != a.l;
#pragma unroll
  for (int e = 0; e < kF; ++e) nan |= a.o[e] != a.o[e];
  if (h.causal_any && __any_sync(0xffffffffu, nan)) {
    // perhaps of a value that the row does not see (0 times NaN): key by key
    const T *q = reinterpret_cast<const T *>(A.q + t * A.q_stride) + hd * D;
    for (int i = lane; i < D; i += 32) qs[warp][i] = static_cast<float>(q[i]);
    __syncwarp();
    a = {-INFINITY, 0.f, {}};
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
      const int i = part ? tok.own : tok.prefix;
      if (i >= 0) group_row<T, D>(A, items[i].seq, head, items[i].key0, min(items[i].key1, tok.limit), qs[warp], a.m, a.l, a.o);
    }
  }
  const float inv = a.l == 0.f ? 0.f : 1.f / a.l;
  uint32_t w[kF / 2];
#pragma unroll
  for (int e = 0; e < kF / 2; ++e) w[e] = Type<T>::pack(a.o[2 * e] * inv, a.o[2 * e + 1] * inv);
  uint8_t *out = A.out + (u * D + lane * kF) * 2;
  if (D == 128)
    *reinterpret_cast<uint2 *>(out) = make_uint2(w[0], w[kF / 2 - 1]);
  else
    *reinterpret_cast<uint32_t *>(out) = w[0];
  if (A.lse && lane == 0) A.lse[u] = (a.m + log2f(a.l)) * 0.6931471805599453f;
}

template <class T, int D>
cudaError_t launch_group(const GroupArgs &A, const CUtensorMap &kmap, const CUtensorMap &vmap, cudaStream_t stream) {
  static std::atomic<uint64_t> attr{0};
  cudaError_t e = once_per_device(attr, [] {
    return cudaFuncSetAttribute(group_tc_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(Lay<D>::kBytes));
  });
  if (e != cudaSuccess) return e;
  const int sms = device_sm_count();
  e = launch_pdl(group_tc_kernel<T, D>, dim3(sms), dim3(kThreads), Lay<D>::kBytes, stream, A,
                 fast_div(static_cast<uint32_t>(A.group)), kmap, vmap);
  if (e != cudaSuccess) return e;
  count_launches(1);
  const int64_t rows = static_cast<int64_t>(A.n_q) * A.hq;
  // Few rows have many parts: several warps each; many have few, and there it is warps that count.  A layer with 28
  // query heads on 9,000 rows by 8 warps a row, by one with eight loads under way, and by one with four: 560 rows 20.5,
  // 23.2 and 36.1 us, 1,120 30.5, 29.5 and 44.5, 4,200 56.9, 33.4 and 34.5, 14,000 174, 80.0 and 79.1, 56,000 554, 265
  // and 245.
  auto merge = [&](auto kernel, int warps) {
    return launch_pdl(kernel, dim3(static_cast<unsigned>((rows * warps + 7) / 8)), dim3(256), 0, stream, A);
  };
  e = rows <= 8 * sms    ? merge(group_merge_kernel<T, D, 8, kBatch>, 8)
      : rows <= 64 * sms ? merge(group_merge_kernel<T, D, 1, kBatch>, 1)
                         : merge(group_merge_kernel<T, D, 1, kFewParts>, 1);
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
  A.seg_off = static_cast<int64_t>(s.seg_off);
  A.err = static_cast<DeviceError *>(ws);
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  CUtensorMap kmap, vmap;
  std::memset(&kmap, 0, sizeof(kmap));
  std::memset(&vmap, 0, sizeof(vmap));
  if (A.box && (!make_page_map(&kmap, cache, A.pool.k, A.box, 1) || !make_page_map(&vmap, cache, A.pool.v, A.box, 1)))
    return APACK_ECUDA;
  if (cache->dtype == APACK_BF16)
    return check_cuda(cache->head_dim == 128 ? launch_group<__nv_bfloat16, 128>(A, kmap, vmap, cs)
                                             : launch_group<__nv_bfloat16, 64>(A, kmap, vmap, cs));
  return check_cuda(cache->head_dim == 128 ? launch_group<__half, 128>(A, kmap, vmap, cs)
                                           : launch_group<__half, 64>(A, kmap, vmap, cs));
}
