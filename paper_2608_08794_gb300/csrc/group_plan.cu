// group_plan.cu -- the work of attention over shared rows, laid out on the device from lengths and groups.
//
// A step's plan serves all its layers, and lengths stay on the device, so that a captured step follows growing caches.
// One CTA: it finds each sequence's group (a search among the groups' bounds in shared memory), how many rows of its
// keys are the group's, how long the runs of keys should be, and writes items, segments and what each token sees.
//
// Bound by latency: trips to L2, block barriers, and reading code that runs once (64 sequences: 9 to 10 us, of which
// offsets and items 3.5, run lengths 3.5, places and segments 2; 300 19, 1,000 47, 4,096 156): once per step, not per
// layer.
//
// The length of a run.  A segment of c tiles costs about c + kSegCost tiles of one SM; n segments on S SMs end after
// max(sum of all / S, ceil(long ones / S) * (c + kSegCost)) at the least, and every part's row is written and read once
// more.  32 warps try two run lengths each over all items, and the least estimate wins.
#include <algorithm>
#include <cstring>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "group.cuh"

namespace apack {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = 32;
constexpr float kSegCost = 2.5f;               // tiles: queries, first loads, parts
constexpr float kRowCost = 1056.f / 65536.f;   // tiles: a part's row written and read, against a tile of K and V

struct PlanArgs {
  const int32_t *seqlens, *seqs, *cu_q, *cu_groups, *prefix;
  uint8_t *ws;
  int32_t n, groups, n_q, hq, hkv, group, head_dim;
  int32_t num_seqs, max_pages, page_tokens, num_pages, max_rows;
  int32_t align;                     // shared rows are cut to a multiple of this
  int32_t sms, halves;
  int64_t cap_rows, cap_segs;
  int64_t tok_off, item_off, seg_off, ml_off, part_off, total;
  DeviceError *err;
};

// Sequences of more new tokens have them written by all threads (the first kMany of them).
constexpr int kFew = 32, kMany = 1024;

struct Two {
  int64_t a, b;
};
struct PlanShared {
  int32_t cu_q[APACK_MAX_SEQS + 1], cu_g[APACK_MAX_SEQS + 1];
  int32_t rows[2 * APACK_MAX_SEQS], tiles[2 * APACK_MAX_SEQS];      // of the items: groups, then sequences
  int32_t seg0[2 * APACK_MAX_SEQS + 1];
  float est[2 * kWarps];
  Two warp_sum[kWarps];
  int32_t bad, longest, causal, many;
  int32_t many_entry[kMany];
  GroupTok many_tok[kMany];
};

__device__ __forceinline__ int runs_of(int rows) { return (rows + kGRows - 1) / kGRows; }
// Parts of a segment of at most 128 rows: two, where its tiles go to the accumulators in turn, or one, where the second
// accumulator has no rows.  Two halve the segment and double its parts; they pay where most segments are such, the
// rows one run (300 to 3,000 sequences of 400 rows, 28/4 heads: 85 to 635 us a layer, 99 to 794 with one).  Where only an
// item's last run is, one part is better: on 9,000 shared rows 40 sequences, 280 rows, 34.4 us against 36.7, 120
// sequences, 840 rows, 43.0 against 44.5; on 22,772 rows 350 of one sequence 34.1 against 37.9, 1,631 72.6 against 78.1.
// So items of more than four runs never write two.
__device__ __forceinline__ int sub_of(const PlanArgs &P, int rows) {
  const int last = rows - (runs_of(rows) - 1) * kGRows;
  return P.halves && rows <= 4 * kGRows && last <= kGSlot ? 2 : 1;
}

// Exclusive sums over the block's threads, and the totals, of two numbers each.
__device__ Two scan(Two v, PlanShared &s, Two *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto inclusive = [&](Two x) {
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int64_t ya = __shfl_up_sync(0xffffffffu, x.a, o), yb = __shfl_up_sync(0xffffffffu, x.b, o);
      if (lane >= o) x.a += ya, x.b += yb;
    }
    return x;
  };
  const Two x = inclusive(v);
  __syncthreads();
  if (lane == 31) s.warp_sum[warp] = x;
  __syncthreads();
  const Two w = inclusive(s.warp_sum[lane]);
  *total = Two{__shfl_sync(0xffffffffu, w.a, 31), __shfl_sync(0xffffffffu, w.b, 31)};
  const int64_t ba = __shfl_sync(0xffffffffu, w.a, (warp + 31) & 31), bb = __shfl_sync(0xffffffffu, w.b, (warp + 31) & 31);
  return Two{x.a - v.a + (warp ? ba : 0), x.b - v.b + (warp ? bb : 0)};
}

// The last i < n with at[i] <= j.
__device__ __forceinline__ int last_at(const int32_t *at, int n, int j) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (at[mid] <= j)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Run length number k of 64 that are tried: the longest item in 1 to 32 runs, then more of them, up to a tile each.
__device__ __forceinline__ int candidate(int k, int longest) {
  if (k < 32) return (longest + k) / (k + 1);
  const float runs = 32.f * exp2f(log2f(longest * (1.f / 32.f)) * (k - 31) * (1.f / 32.f));
  return max(1, min(longest, static_cast<int>(longest / fmaxf(runs, 1.f) + 0.999f)));
}
// Estimated time of two run lengths, in tiles of one SM; infinite where the workspace does not hold them.  By one warp.
__device__ void estimate(const PlanArgs &P, const PlanShared &s, int items, const int (&c)[2], float (&est)[2]) {
  const int lane = threadIdx.x & 31;
  float work = 0.f, segs[2] = {}, rows[2] = {}, big[2] = {}, most[2] = {};
  for (int i = lane; i < items; i += 32) {
    if (s.rows[i] == 0) continue;
    const float heads = static_cast<float>(P.hkv) * runs_of(s.rows[i]);
    const float part = static_cast<float>(s.rows[i]) * P.hkv * sub_of(P, s.rows[i]);
    work += heads * s.tiles[i];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int splits = (s.tiles[i] + c[j] - 1) / c[j];
      const float chunk = __fdividef(s.tiles[i], splits);
      segs[j] += heads * splits;
      rows[j] += part * splits;
      if (2.f * chunk > c[j]) {
        big[j] += heads * splits;
        most[j] = fmaxf(most[j], ceilf(chunk));
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    work += __shfl_xor_sync(0xffffffffu, work, o);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      segs[j] += __shfl_xor_sync(0xffffffffu, segs[j], o);
      rows[j] += __shfl_xor_sync(0xffffffffu, rows[j], o);
      big[j] += __shfl_xor_sync(0xffffffffu, big[j], o);
      most[j] = fmaxf(most[j], __shfl_xor_sync(0xffffffffu, most[j], o));
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const float even = (work + segs[j] * kSegCost) / P.sms, rounds = ceilf(big[j] / P.sms) * (most[j] + kSegCost);
    est[j] = rows[j] > 0.99f * P.cap_rows || segs[j] > 0.99f * P.cap_segs
                 ? INFINITY
                 : fmaxf(even, rounds) + rows[j] * kRowCost / P.sms;
  }
}

__global__ void __launch_bounds__(kThreads, 1) group_plan_kernel(const __grid_constant__ PlanArgs P) {
  extern __shared__ uint8_t raw[];
  PlanShared &s = *reinterpret_cast<PlanShared *>(raw);
  GroupHead *head = reinterpret_cast<GroupHead *>(P.ws + kGHeadOff);
  GroupItem *items = reinterpret_cast<GroupItem *>(P.ws + P.item_off);
  GroupTok *tok = reinterpret_cast<GroupTok *>(P.ws + P.tok_off);
  GroupSeg *segs = reinterpret_cast<GroupSeg *>(P.ws + P.seg_off);
  const int warp = threadIdx.x >> 5, n = P.n, ng = P.groups, G = P.group;
  if (threadIdx.x == 0) s.bad = s.longest = s.causal = s.many = 0;
  pdl_wait_and_release();
  for (int i = threadIdx.x; i <= n; i += kThreads) s.cu_q[i] = P.cu_q ? P.cu_q[i] : i;
  for (int i = threadIdx.x; i <= ng; i += kThreads) s.cu_g[i] = ng ? P.cu_groups[i] : 0;
  __syncthreads();
  for (int i = threadIdx.x; i <= n; i += kThreads) {
    const int at = s.cu_q[i];
    if (at < (i ? s.cu_q[i - 1] : 0) || at > P.n_q || (i == 0 && at != 0)) {
      raise_device_error(P.err, APACK_EDEVICE, 141, i, at);
      s.bad = 1;
    }
  }
  for (int i = threadIdx.x; i <= ng && ng; i += kThreads) {
    const int at = s.cu_g[i];
    if (at < (i ? s.cu_g[i - 1] : 0) || at > n) {
      raise_device_error(P.err, APACK_EDEVICE, 142, i, at);
      s.bad = 1;
    }
  }
  __syncthreads();
  const bool bad = s.bad;
  const int total_items = ng + n;
  // ---- items: every sequence finds its group's shared rows by itself, so that nothing waits between groups and
  // sequences
  for (int g = threadIdx.x; g < ng; g += kThreads) s.rows[g] = s.tiles[g] = s.seg0[g] = 0;
  __syncthreads();
  // seg0, for now: the runs of rows that a group's sequences make by themselves
  for (int e = threadIdx.x; e < n && ng && !bad; e += kThreads)
    if (e >= s.cu_g[0] && e < s.cu_g[ng]) atomicAdd(&s.seg0[last_at(s.cu_g, ng, e)], runs_of((s.cu_q[e + 1] - s.cu_q[e]) * G));
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += kThreads) {
    s.rows[ng + e] = s.tiles[ng + e] = 0;
    if (bad) continue;
    const int m = s.cu_q[e + 1] - s.cu_q[e];
    int g = -1, first = e, shared = 0, count = 0;
    if (ng && e >= s.cu_g[0] && e < s.cu_g[ng]) {
      g = last_at(s.cu_g, ng, e);
      first = s.cu_g[g];
      count = s.cu_g[g + 1] - first;
      shared = P.prefix[g];
    }
    const int b = P.seqs ? P.seqs[e] : e, b0 = P.seqs ? P.seqs[first] : first;
    const bool in = static_cast<uint32_t>(b) < static_cast<uint32_t>(P.num_seqs);
    const bool in0 = static_cast<uint32_t>(b0) < static_cast<uint32_t>(P.num_seqs);
    const int x = in ? P.seqlens[b] : 0, x0 = in0 ? P.seqlens[b0] : 0;
    const int len = min(max(x, 0), P.max_rows), len0 = min(max(x0, 0), P.max_rows);
    if (!in) raise_device_error(P.err, APACK_EDEVICE, 143, e, b);
    if (len != x) raise_device_error(P.err, APACK_EDEVICE, 144, b, x);
    if (m > len) raise_device_error(P.err, APACK_EDEVICE, 146, e, len);
    int cut = 0;                                   // rows that are read with the group's
    if (count > 1) {
      if (e == first && (shared < 0 || shared > len0)) raise_device_error(P.err, APACK_EDEVICE, 145, g, shared);
      cut = min(max(shared, 0), len0);
      cut -= cut % P.align;
      const int rows = (s.cu_q[first + count] - s.cu_q[first]) * G;
      // Reading rows together pays where it saves products: their tiles once per run of the group's rows, not of each
      // sequence's, against a segment more per run and a part more per row.  (13 prompts of 350 to 700 tokens behind
      // 255 shared rows, 28/4 heads of 128: 378 us together, 303 apart.)
      const int tiles = (cut + kGTile - 1) / kGTile, runs = runs_of(rows);
      if (!in0 || rows == 0 || static_cast<float>(s.seg0[g] - runs) * tiles <= runs * kSegCost + rows * kRowCost) cut = 0;
      if (e == first && cut > 0) {
        GroupItem it = {};
        it.seq = b0;
        it.key1 = cut;
        it.row0 = s.cu_q[first] * G;
        it.rows = s.rows[g] = rows;
        s.tiles[g] = (cut + kGTile - 1) / kGTile;
        atomicMax(&s.longest, s.tiles[g]);
        items[g] = it;
      }
    }
    if (m > 0 && in && cut < len) {
      GroupItem it = {};
      it.seq = b;
      it.key0 = cut;
      it.key1 = len;
      it.row0 = s.cu_q[e] * G;
      it.rows = s.rows[ng + e] = m * G;
      it.causal = m > 1;
      s.tiles[ng + e] = (len - cut + kGTile - 1) / kGTile;
      atomicMax(&s.longest, s.tiles[ng + e]);
      items[ng + e] = it;
    }
    if (m > 1 || cut > len - m + 1) s.causal = 1;  // (the latter: a token that does not see all of the shared rows)
    const GroupTok tk = {len - m + 1 - s.cu_q[e], cut > 0 ? g : -1, s.rows[ng + e] ? ng + e : -1, 1};
    const int i = m > kFew ? atomicAdd(&s.many, 1) : kMany;      // by all threads, below (in any order)
    if (i < kMany) {
      s.many_entry[i] = e;
      s.many_tok[i] = tk;
    } else {
      for (int t = s.cu_q[e]; t < s.cu_q[e + 1]; ++t) tok[t] = GroupTok{max(tk.limit + t, 0), tk.prefix, tk.own, 1};
    }
  }
  __syncthreads();
  const int n_tok = bad ? 0 : s.cu_q[n], many = min(s.many, kMany);
  for (int i = 0; i < many; ++i) {
    const int e = s.many_entry[i];
    const GroupTok tk = s.many_tok[i];
    for (int t = s.cu_q[e] + threadIdx.x; t < s.cu_q[e + 1]; t += kThreads)
      tok[t] = GroupTok{max(tk.limit + t, 0), tk.prefix, tk.own, 1};
  }
  for (int t = n_tok + threadIdx.x; t < P.n_q; t += kThreads) tok[t] = GroupTok{0, -1, -1, 0};
  // ---- the run length
  const int longest = max(s.longest, 1), lane = threadIdx.x & 31;
  {
    const int c[2] = {candidate(warp, longest), candidate(warp + 32, longest)};
    float est[2];
    estimate(P, s, total_items, c, est);
    if (lane == 0) {
      s.est[warp] = est[0];
      s.est[warp + 32] = est[1];
    }
  }
  __syncthreads();
  // the least, of equals the longest runs; none is finite: one run each, which the workspace holds
  float best = fminf(s.est[lane], s.est[lane + 32]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = fminf(best, __shfl_xor_sync(0xffffffffu, best, o));
  const unsigned hit = __ballot_sync(0xffffffffu, s.est[lane] == best), later = __ballot_sync(0xffffffffu, s.est[lane + 32] == best);
  const int chunk = best < INFINITY ? candidate(hit ? __ffs(hit) - 1 : 31 + __ffs(later), longest) : longest;
  // ---- places of segments and parts
  int64_t seg_at = 0, part_at = 0;
  for (int i0 = 0; i0 < total_items; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    int splits = 0, sub = 1;
    if (i < total_items && s.rows[i]) {
      splits = (s.tiles[i] + chunk - 1) / chunk;
      sub = sub_of(P, s.rows[i]);
    }
    const int64_t here = splits ? static_cast<int64_t>(splits) * P.hkv * runs_of(s.rows[i]) : 0;
    const int64_t part = splits ? static_cast<int64_t>(splits) * sub * P.hkv * s.rows[i] : 0;
    Two all;
    const Two before = scan(Two{here, part}, s, &all);
    const int64_t seg = seg_at + before.a, row = part_at + before.b;
    if (i < total_items) {
      s.seg0[i] = static_cast<int32_t>(min(seg, static_cast<int64_t>(INT32_MAX)));
      if (splits) {
        items[i].splits = splits;
        items[i].chunk = (s.tiles[i] + splits - 1) / splits;
        items[i].sub = sub;
        items[i].part = static_cast<int32_t>(min(row, static_cast<int64_t>(INT32_MAX)));
      }
    }
    seg_at += all.a;
    part_at += all.b;
  }
  const bool fits = seg_at <= P.cap_segs && part_at <= P.cap_rows;
  if (!fits && threadIdx.x == 0) raise_device_error(P.err, APACK_EDEVICE, 147, static_cast<int>(seg_at), static_cast<int>(part_at));
  __syncthreads();
  const int count = bad || !fits ? 0 : static_cast<int>(seg_at);
  for (int j = threadIdx.x; j < count; j += kThreads) {
    const int i = last_at(s.seg0, total_items, j), runs = runs_of(s.rows[i]);
    const GroupItem it = items[i];
    int x = j - s.seg0[i];
    const int run = x % runs;
    x /= runs;
    const int h = x % P.hkv, split = x / P.hkv;
    GroupSeg g;
    g.seq = it.seq;
    g.head = h;
    g.row0 = it.row0 + run * kGRows;
    g.rows = min(kGRows, it.rows - run * kGRows);
    g.key0 = it.key0 + split * it.chunk * kGTile;
    g.key1 = min(it.key1, g.key0 + it.chunk * kGTile);
    // (the last row's token sees the fewest rows too many: len - m + 1 + its number)
    if (it.causal) g.key1 = min(g.key1, it.key1 - it.rows / G + 1 + (run * kGRows + g.rows - 1) / G);
    g.part = it.part + (split * it.sub * P.hkv + h) * it.rows + run * kGRows;
    g.step = it.sub == 2 && g.rows <= kGSlot ? P.hkv * it.rows : it.splits == 1 && i >= ng && it.key0 == 0 ? -1 : 0;
    segs[j] = g;
  }
  if (threadIdx.x == 0) {
    GroupHead h = {};
    h.magic = bad || !fits ? 0 : kGMagic;          // without a plan the attention calls record an error and write nothing
    h.n_q = P.n_q;
    h.hq = P.hq;
    h.hkv = P.hkv;
    h.head_dim = P.head_dim;
    h.num_seqs = P.num_seqs;
    h.max_pages = P.max_pages;
    h.page_tokens = P.page_tokens;
    h.num_pages = P.num_pages;
    h.segs = count;
    h.causal_any = s.causal;
    h.item_off = P.item_off;
    h.ml_off = P.ml_off;
    h.part_off = P.part_off;
    h.total = P.total;
    *head = h;
    *reinterpret_cast<uint32_t *>(P.ws + kGClaimOff) = 0;
  }
}

}  // namespace

apack_status group_shape(const apack_paged_cache *c, int32_t hq, int32_t n_seqs, int64_t n_q, GroupShape *s) {
  if (hq < 1 || hq > 1024 || hq % c->num_kv_heads != 0) return APACK_EINVAL;
  if (n_seqs < 1 || n_seqs > APACK_MAX_SEQS || n_q < 0 || n_q > (1 << 24) || n_q * hq > (1 << 28)) return APACK_EINVAL;
  s->group = hq / c->num_kv_heads;
  const int64_t rows = n_q * hq, packed = n_q * s->group, sms = device_sm_count();
  // every item once (shared and own rows; twice in halves), and what runs of keys add for all SMs.  Halves double the
  // room for parts (1,170 tokens of 28/4 heads: a workspace of 149 MB), which is what bounds them here, by the tokens that
  // there is room for.  With more, 1,500 decode tokens take 409 us where halves would 326; 1,200 tokens of a prompt beside
  // 40 decode tokens take 145 and would 160.
  s->halves = packed <= 8192;
  s->cap_rows = rows * (s->halves ? 4 : 2) + std::min(rows * sms, sms * 4 * kGRows) + 64;
  s->cap_segs = c->num_kv_heads * (2 * (packed / kGRows) + 2 * static_cast<int64_t>(n_seqs)) + 8 * sms + 64;
  auto up = [](int64_t x) { return static_cast<size_t>((x + 255) & ~int64_t{255}); };
  // (places that the attention's kernels read first follow n_q alone, which they know without the plan's head)
  s->tok_off = kGFixed;
  s->seg_off = up(s->tok_off + n_q * sizeof(GroupTok));
  s->item_off = up(s->seg_off + s->cap_segs * sizeof(GroupSeg));
  s->ml_off = up(s->item_off + 2 * static_cast<int64_t>(n_seqs) * sizeof(GroupItem));
  s->part_off = up(s->ml_off + s->cap_rows * sizeof(float2));
  s->total = up(s->part_off + s->cap_rows * c->head_dim * sizeof(float));
  return APACK_OK;
}

}  // namespace apack

using namespace apack;

extern "C" {

apack_status apack_paged_group_workspace_size(const apack_paged_cache *cache, int32_t num_q_heads, int32_t n_seqs,
                                              int64_t n_q, size_t *bytes) {
  if (!bytes) return APACK_EINVAL;
  apack_status st = validate_pool(cache, true);
  if (st != APACK_OK) return st;
  GroupShape s;
  st = group_shape(cache, num_q_heads, n_seqs, n_q, &s);
  if (st == APACK_OK) *bytes = s.total;
  return st;
}

apack_status apack_paged_group_plan(const apack_paged_cache *cache, const int32_t *seqlens, int32_t num_q_heads,
                                    int32_t n_seqs, const int32_t *seqs, const int32_t *cu_q, int64_t n_q,
                                    int32_t n_groups, const int32_t *cu_groups, const int32_t *prefix, void *ws,
                                    size_t ws_bytes, void *stream) {
  apack_status st = validate_pool(cache, true);
  if (st != APACK_OK) return st;
  GroupShape s;
  st = group_shape(cache, num_q_heads, n_seqs, n_q, &s);
  if (st != APACK_OK) return st;
  if (!seqlens || !ws || (!seqs && n_seqs > cache->num_seqs) || (!cu_q && n_q != n_seqs)) return APACK_EINVAL;
  if (n_groups < 0 || n_groups > n_seqs || (n_groups > 0 && (!cu_groups || !prefix))) return APACK_EINVAL;
  if (((reinterpret_cast<uintptr_t>(seqlens) | reinterpret_cast<uintptr_t>(seqs) | reinterpret_cast<uintptr_t>(cu_q) |
        reinterpret_cast<uintptr_t>(cu_groups) | reinterpret_cast<uintptr_t>(prefix)) & 3) ||
      (reinterpret_cast<uintptr_t>(ws) & 255))
    return APACK_EINVAL;
  if (ws_bytes < s.total) return APACK_EWORKSPACE;
  PlanArgs P;
  std::memset(&P, 0, sizeof(P));
  P.seqlens = seqlens;
  P.seqs = seqs;
  P.cu_q = cu_q;
  P.cu_groups = cu_groups;
  P.prefix = prefix;
  P.ws = static_cast<uint8_t *>(ws);
  P.n = n_seqs;
  P.groups = n_groups;
  P.n_q = static_cast<int32_t>(n_q);
  P.hq = num_q_heads;
  P.hkv = cache->num_kv_heads;
  P.group = s.group;
  P.head_dim = cache->head_dim;
  P.num_seqs = cache->num_seqs;
  P.max_pages = cache->max_pages;
  P.page_tokens = cache->page_tokens;
  P.num_pages = cache->num_pages;
  P.max_rows = static_cast<int32_t>(
      std::min<int64_t>(1 << 30, static_cast<int64_t>(cache->max_pages) * cache->page_tokens));
  P.align = std::max(1, group_box(cache->page_tokens));
  P.sms = device_sm_count();
  P.halves = s.halves;
  P.cap_rows = s.cap_rows;
  P.cap_segs = s.cap_segs;
  P.tok_off = s.tok_off;
  P.item_off = s.item_off;
  P.seg_off = s.seg_off;
  P.ml_off = s.ml_off;
  P.part_off = s.part_off;
  P.total = s.total;
  P.err = static_cast<DeviceError *>(ws);
  static std::atomic<uint64_t> attr{0};
  cudaError_t e = once_per_device(attr, [] {
    return cudaFuncSetAttribute(group_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(sizeof(PlanShared)));
  });
  if (e == cudaSuccess)
    e = launch_pdl(group_plan_kernel, dim3(1), dim3(kThreads), sizeof(PlanShared), static_cast<cudaStream_t>(stream), P);
  if (e == cudaSuccess) count_launches(1);
  return check_cuda(e);
}

}  // extern "C"
