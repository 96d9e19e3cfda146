// pages.cu -- who holds which page of a paged key-value cache, on the device: page tables, lengths, reference counts
// and a stack of free pages, changed by kernels, so that a captured step of a server needs no host between its layers.
//
// What a call takes or gives back is a list in the order of its entries, then of their rows: page j of the list comes
// from (goes to) place free_count - 1 - j.  The list's positions are exclusive sums over the entries, so that nothing
// depends on the order in which threads run, and a release followed by an extension of as many pages restores the
// stack.
//
// Bound by latency: a chain of some five reads that depend on one another (entry, length, table, count, page), barriers
// between them, and one launch: release and extension of 61 sequences by a row each take 14.5 us, 256 drafts 19.3.  One
// CTA, or a cluster of eight where the lists may be long, because a split over the grid needs a second launch or a grid
// barrier, which cost more than the work.  Only the map from new rows to slots is large when prompts enter (16 bytes
// per row): above kInlineRows rows a second kernel on all SMs fills it (298,112 rows of 1,000 prompts: 7.1 us, 0.67
// TB/s).
#include <algorithm>
#include <cstring>

#include "paged.cuh"
#include "ptx.cuh"

namespace apack {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kPer = APACK_MAX_SEQS / kThreads;      // entries of a thread: kThreads apart, so that few entries take few steps
// Calls that may move more pages than this take a cluster: 64 questions that leave and come, whose 64,186 table entries
// name some 5,260 pages, take 409 us by one SM, which reads one random place per clock at best, and 88 by eight; 18,803
// pages of 1,000 prompts that leave and come 92 and 37.  A step of 61 sequences takes 0.5 us longer so (14.2 -> 14.8),
// but nothing on the host says how few pages it moves.
constexpr int kMaxCluster = 8;
constexpr int64_t kClusterPages = 16384;
// Rows of the slot map that the first kernel fills by itself.
constexpr int kInlineRows = 8192;

struct PagesView {
  int32_t *table;
  int64_t table_stride;
  int32_t *lengths, *refs, *free_list, *free_count;
  int32_t num_seqs, max_pages, num_pages;
  FastDiv page_tokens;
  __device__ __forceinline__ int pages_of(int rows) const {      // ceil(rows / page_tokens)
    const int full = page_tokens.div(rows);
    return full + (full * static_cast<int>(page_tokens.d) != rows);
  }
  __device__ __forceinline__ int in_page(int row) const { return row - page_tokens.div(row) * page_tokens.d; }
  __device__ __forceinline__ int32_t *row(int seq) const { return table + seq * table_stride; }
};

struct Call {
  PagesView t;
  int32_t n;
  const int32_t *seqs, *rows;        // rows: kept (release), added (extend); parents (fork)
  DeviceError *err;
};

struct Shared {
  int64_t warp_sum[kWarps];
  uint32_t seen[APACK_MAX_SEQS / 32];
  int32_t at[APACK_MAX_SEQS + 1];    // exclusive sums over the entries
  int32_t bad;                       // an entry, as every CTA finds by itself
  int32_t wrong, shared;             // a page; raised for the whole cluster, read behind its next barrier
  int32_t freed[kMaxCluster];
};

__device__ __forceinline__ void report(const Call &C, int where, int a, int b) {
  if (C.err) raise_device_error(C.err, APACK_EDEVICE, where, a, b);
}

// Exclusive sum over the block's threads, each with `v`; the block's sum in *total.
__device__ int64_t block_scan(int64_t v, Shared &s, int64_t *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t x = v;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();                   // warp_sum of the scan before has been read
  if (lane == 31) s.warp_sum[warp] = x;
  __syncthreads();
  int64_t w = s.warp_sum[lane];
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int64_t y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  *total = __shfl_sync(0xffffffffu, w, 31);
  const int64_t before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
  return x - v + (warp ? before : 0);
}

// Exclusive sums over the entries (entry k * kThreads + thread has v[k]), to at[0 .. n], at[n] their total.
__device__ int64_t entry_sums(const int (&v)[kPer], int n, int32_t *at, Shared &s) {
  int64_t carry = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (k * kThreads >= n) break;
    const int i = k * kThreads + threadIdx.x;
    int64_t sum;
    const int64_t x = carry + block_scan(v[k], s, &sum);
    if (i < n) at[i] = static_cast<int32_t>(min(x, static_cast<int64_t>(INT32_MAX)));
    carry += sum;
  }
  if (threadIdx.x == 0) at[n] = static_cast<int32_t>(min(carry, static_cast<int64_t>(INT32_MAX)));
  return carry;
}

// The sequence of entry i, or -1: outside the table, or named before.  Every sequence may be named once.
__device__ int entry_seq(const Call &C, Shared &s, int i) {
  const int b = C.seqs ? __ldg(C.seqs + i) : i;
  if (static_cast<uint32_t>(b) >= static_cast<uint32_t>(C.t.num_seqs)) {
    report(C, 120, i, b);
    return -1;
  }
  if (C.seqs && (atomicOr(&s.seen[b >> 5], 1u << (b & 31)) >> (b & 31) & 1u)) {
    report(C, 121, i, b);
    return -1;
  }
  return b;
}

__device__ __forceinline__ int32_t now(const int32_t *p) { return *const_cast<const volatile int32_t *>(p); }

// The entries of kBatch places of the list (the last i with at[i] <= j), side by side: every pass over a list is bound
// by the trips of its reads, so a thread has as many of them under way (by one SM: the 64 questions 563 us one by one,
// 409 so; 1,000 prompts 100 and 92; 256 drafts, which move 67 pages, 13.0 and 18.8).
constexpr int kBatch = 8;
__device__ __forceinline__ void entries_of(const int32_t *at, int n, const int (&j)[kBatch], int (&e)[kBatch]) {
#pragma unroll
  for (int k = 0; k < kBatch; ++k) e[k] = 0;
  for (int step = n > 1 ? 1 << (31 - __clz(n - 1)) : 0; step > 0; step >>= 1)
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int c = e[k] + step;
      if (c < n && at[c] <= j[k]) e[k] = c;
    }
}
// For the thread's places of a list of `sum`, in batches: first `load` for all of a batch, then `more`, then `use`.
template <int CL, class Load, class More, class Use>
__device__ __forceinline__ void for_places(const int32_t *at, int n, int sum, Load &&load, More &&more, Use &&use) {
  for (int j0 = (CL > 1 ? static_cast<int>(cluster_ctarank()) * kThreads : 0) + threadIdx.x; j0 < sum; j0 += kBatch * CL * kThreads) {
    int j[kBatch], e[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) j[k] = min(j0 + k * CL * kThreads, sum - 1);
    entries_of(at, n, j, e);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) load(k, j[k], e[k]);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) more(k);
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (j0 + k * CL * kThreads < sum) use(k, j[k], e[k]);
  }
}
struct Nothing {
  __device__ __forceinline__ void operator()(int) const {}
};

// CL: CTAs of the kernel's cluster, which share a list's places; every one of them looks at all entries by itself.
template <int CL>
__device__ __forceinline__ void sync_all() {
  if (CL > 1)
    cluster_sync();
  else
    __syncthreads();
}
template <int CL>
__device__ __forceinline__ void raise_flag(int32_t *flag) {
  if (CL == 1) {
    *flag = 1;
  } else if (*const_cast<volatile int32_t *>(flag) == 0) {
    for (int r = 0; r < CL; ++r)
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_shared_rank(flag, r)), "r"(1) : "memory");
  }
}

template <int CL>
__device__ void begin(Shared &s) {
  for (int i = threadIdx.x; i < APACK_MAX_SEQS / 32; i += kThreads) s.seen[i] = 0;
  if (threadIdx.x == 0) s.bad = s.wrong = s.shared = 0;
  pdl_wait_and_release();
  sync_all<CL>();                     // (no CTA writes another's flags before they are cleared)
}

// ---------------------------------------------------------------- release

// Every entry keeps its first rows[i] rows.  The pages behind them lose a holder; each that has none left goes to the
// stack once, at its first place in the call's list: while the list is walked a count of 0 becomes the least place at
// which the page is named (minus 2^31), which is found whatever the order of the threads.
template <int CL>
__global__ void __launch_bounds__(kThreads, 1) pages_release_kernel(const __grid_constant__ Call C) {
  __shared__ Shared s;
  // of an entry's first page to give up; read from here later on, because the rows to keep may be lengths, which others
  // of the call's threads write in the end
  __shared__ int32_t column[APACK_MAX_SEQS];
  begin<CL>(s);
  const PagesView &t = C.t;
  int seq[kPer], keep[kPer], drop[kPer];
  const int count = *t.free_count;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = k * kThreads + threadIdx.x;
    seq[k] = -1;
    drop[k] = keep[k] = 0;
    if (i >= C.n) continue;
    const int b = entry_seq(C, s, i);
    if (b < 0) {
      s.bad = 1;
      continue;
    }
    const int len = t.lengths[b];
    keep[k] = C.rows[i];
    if (len < 0 || keep[k] < 0 || keep[k] > len || t.pages_of(len) > t.max_pages) {
      report(C, 122, i, keep[k]);
      s.bad = 1;
      continue;
    }
    seq[k] = b;
    column[i] = t.pages_of(keep[k]);
    drop[k] = t.pages_of(len) - column[i];
  }
  const int64_t total = entry_sums(drop, C.n, s.at, s);
  if (total > INT32_MAX - 1 && threadIdx.x == 0) {
    report(C, 123, 0, 0);
    s.bad = 1;
  }
  __syncthreads();
  if (s.bad) return;                                        // nothing is changed
  // the pages are there, and held
  const int n = C.n, sum = static_cast<int>(total);
  auto place_of = [&](int j, int e) {                       // the table's entry of the list's page j
    const int b = C.seqs ? __ldg(C.seqs + e) : e;
    return t.row(b) + column[e] + (j - s.at[e]);
  };
  int32_t *place[kBatch];
  int p[kBatch], r[kBatch];
  auto load = [&](int k, int j, int e) {
    place[k] = place_of(j, e);
    p[k] = now(place[k]);
  };
  auto holders = [&](int k) { r[k] = static_cast<uint32_t>(p[k]) < static_cast<uint32_t>(t.num_pages) ? now(t.refs + p[k]) : 0; };
  for_places<CL>(s.at, n, sum, load, holders, [&](int k, int, int e) {
    if (r[k] < 1) {
      report(C, 124, e, p[k]);
      raise_flag<CL>(&s.wrong);
    }
    if (r[k] != 1) raise_flag<CL>(&s.shared);
  });
  if (count < 0 || count > t.num_pages) {
    if (threadIdx.x == 0) report(C, 125, count, 0);
    raise_flag<CL>(&s.wrong);
  }
  sync_all<CL>();
  if (s.wrong) return;
  const int room = t.num_pages - count;
  int top = count;
  if (!s.shared) {
    // every page was this sequence's alone: its place in the list is its place on the stack
    top += min(sum, room);
    if (sum > room && threadIdx.x == 0) report(C, 125, count, sum);   // more free pages than there are: the counts disagree
    for_places<CL>(s.at, n, sum, load, Nothing(), [&](int k, int j, int) {
      if (j < top - count) t.free_list[top - 1 - j] = p[k];
      t.refs[p[k]] = 0;
      *place[k] = -1;
    });
  } else {
    for_places<CL>(s.at, n, sum, load, Nothing(), [&](int k, int, int) { atomicSub(t.refs + p[k], 1); });
    sync_all<CL>();
    for_places<CL>(s.at, n, sum, load, holders, [&](int k, int j, int) {
      if (r[k] <= 0) atomicMin(t.refs + p[k], j + INT32_MIN);
    });
    sync_all<CL>();
    // the freed pages' places among themselves: a run of the list per CTA, counted, then placed
    const int rank = CL > 1 ? cluster_ctarank() : 0;
    const int per = (sum + CL - 1) / CL, lo = min(rank * per, sum), hi = min(lo + per, sum);
    int64_t here = 0, first = 0, all = 0;
    auto run = [&](auto &&take) {                           // in the list's order
      int64_t before = 0;
      for (int j0 = lo; j0 < hi; j0 += kBatch * kThreads) {
        int j[kBatch], e[kBatch], freed = 0;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) j[k] = min(j0 + static_cast<int>(threadIdx.x) * kBatch + k, sum - 1);
        entries_of(s.at, n, j, e);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) load(k, j[k], e[k]);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) holders(k);
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
          r[k] = j0 + static_cast<int>(threadIdx.x) * kBatch + k < hi && r[k] == j[k] + INT32_MIN;
          freed += r[k];
        }
        int64_t total_here;
        take(before + block_scan(freed, s, &total_here));
        before += total_here;
      }
      return before;
    };
    if (CL > 1) {
      here = run([](int64_t) {});
      if (threadIdx.x < CL)
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_shared_rank(&s.freed[rank], threadIdx.x)), "r"(static_cast<int>(here))
                     : "memory");
      sync_all<CL>();
      for (int i = 0; i < CL; ++i) {
        if (i < rank) first += s.freed[i];
        all += s.freed[i];
      }
    } else {
      all = run([](int64_t) {});
    }
    if (all > room) {
      if (threadIdx.x == 0) report(C, 125, count, static_cast<int>(all));
      all = room;
    }
    top += static_cast<int>(all);
    run([&](int64_t at) {
      at += first;
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (r[k]) {
          if (at < all) t.free_list[top - 1 - at] = p[k];
          ++at;
        }
    });
    sync_all<CL>();
    for_places<CL>(s.at, n, sum, load, holders, [&](int k, int, int) {
      if (r[k] < 0) atomicMax(t.refs + p[k], 0);
      *place[k] = -1;
    });
  }
  if (CL > 1 && cluster_ctarank() != 0) return;
  if (threadIdx.x == 0) *t.free_count = top;
#pragma unroll
  for (int k = 0; k < kPer; ++k)
    if (seq[k] >= 0) t.lengths[seq[k]] = keep[k];
}

// ---------------------------------------------------------------- fork

// Entry i's sequence takes over its parent's table row and length; every page gets a holder more.
template <int CL>
__global__ void __launch_bounds__(kThreads, 1) pages_fork_kernel(const __grid_constant__ Call C) {
  __shared__ Shared s;
  begin<CL>(s);
  const PagesView &t = C.t;
  int need[kPer], rows[kPer];
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = k * kThreads + threadIdx.x;
    need[k] = rows[k] = 0;
    if (i >= C.n) continue;
    const int b = entry_seq(C, s, i), from = C.rows[i];
    if (b < 0) {
      s.bad = 1;
      continue;
    }
    const bool there = static_cast<uint32_t>(from) < static_cast<uint32_t>(t.num_seqs);
    const int len = there ? t.lengths[from] : -1;
    if (!there || from == b || t.lengths[b] != 0 || len < 0 || t.pages_of(len) > t.max_pages) {
      report(C, 126, i, from);
      s.bad = 1;
      continue;
    }
    rows[k] = len;
    need[k] = t.pages_of(len);
  }
  const int64_t total = entry_sums(need, C.n, s.at, s);
  if (total > INT32_MAX - 1 && threadIdx.x == 0) {
    report(C, 123, 0, 0);
    s.bad = 1;
  }
  __syncthreads();
  if (s.bad) return;
  const int n = C.n, sum = static_cast<int>(total);
  int p[kBatch], r[kBatch];
  // (a sequence that is a child here was empty: as a parent it has no pages to read)
  auto load = [&](int k, int j, int e) { p[k] = now(t.row(C.rows[e]) + (j - s.at[e])); };
  auto holders = [&](int k) { r[k] = static_cast<uint32_t>(p[k]) < static_cast<uint32_t>(t.num_pages) ? now(t.refs + p[k]) : 0; };
  for_places<CL>(s.at, n, sum, load, holders, [&](int k, int, int e) {
    if (r[k] < 1) {
      report(C, 124, e, p[k]);
      raise_flag<CL>(&s.wrong);
    }
  });
  sync_all<CL>();
  if (s.wrong) return;
  for_places<CL>(s.at, n, sum, load, Nothing(), [&](int k, int j, int e) {
    atomicAdd(t.refs + p[k], 1);
    t.row(C.seqs ? __ldg(C.seqs + e) : e)[j - s.at[e]] = p[k];
  });
  if (CL > 1 && cluster_ctarank() != 0) return;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = k * kThreads + threadIdx.x;
    if (i < C.n) t.lengths[C.seqs ? __ldg(C.seqs + i) : i] = rows[k];
  }
}

// ---------------------------------------------------------------- extend

struct Maps {
  int32_t *cu, *rows, *row_seqs;
  int64_t *slots;
  int2 *pairs;
  int64_t max_rows;
};

// New rows number j0, j0 + stride, ... of the call, kBatch of them: row, sequence and slot.
__device__ __forceinline__ void write_maps(const Call &C, const Maps &M, const int32_t *cu, int64_t j0, int64_t stride) {
  int j[kBatch], e[kBatch], b[kBatch], row[kBatch], page[kBatch];
  const int last = cu[C.n] - 1;
#pragma unroll
  for (int k = 0; k < kBatch; ++k) j[k] = static_cast<int>(min(j0 + k * stride, static_cast<int64_t>(max(last, 0))));
  if (last >= 0) {
    entries_of(cu, C.n, j, e);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) b[k] = C.seqs ? __ldg(C.seqs + e[k]) : e[k];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) row[k] = now(C.t.lengths + b[k]) - cu[e[k] + 1] + j[k];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) page[k] = now(C.t.row(b[k]) + C.t.page_tokens.div(row[k]));
  }
#pragma unroll
  for (int k = 0; k < kBatch; ++k) {
    const int64_t at = j0 + k * stride;
    if (at >= M.max_rows) break;
    const bool real = at <= last;
    M.rows[at] = real ? row[k] : -1;
    if (M.row_seqs) M.row_seqs[at] = real ? b[k] : -1;
    if (M.slots) M.slots[at] = real ? static_cast<int64_t>(page[k]) * C.t.page_tokens.d + C.t.in_page(row[k]) : -1;
  }
}

// Entry i gets rows[i] more rows.  A last page that it shares and would write into is replaced by one of its own: of
// the sequences that hold it, all that the call extends but the last holder; the pair (old, new) is left for
// apack_copy_pages.
template <int CL>
__global__ void __launch_bounds__(kThreads, 1)
    pages_extend_kernel(const __grid_constant__ Call C, const __grid_constant__ Maps M) {
  __shared__ Shared s;
  __shared__ int32_t sharing[APACK_MAX_SEQS];
  __shared__ int n_sharing;
  if (threadIdx.x == 0) n_sharing = 0;
  begin<CL>(s);
  const PagesView &t = C.t;
  int seq[kPer], len[kPer], grow[kPer], take[kPer], last[kPer];
  const int count = *t.free_count;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = k * kThreads + threadIdx.x;
    seq[k] = last[k] = -1;
    len[k] = grow[k] = take[k] = 0;
    if (i >= C.n) continue;
    sharing[i] = -1;
    const int b = entry_seq(C, s, i);
    if (b < 0) {
      s.bad = 1;
      continue;
    }
    len[k] = t.lengths[b];
    grow[k] = C.rows[i];
    const int64_t end = static_cast<int64_t>(len[k]) + grow[k];
    if (len[k] < 0 || grow[k] < 0 || end > INT32_MAX || t.pages_of(static_cast<int>(end)) > t.max_pages) {
      report(C, 127, i, grow[k]);
      s.bad = 1;
      continue;
    }
    seq[k] = b;
    const int held = t.pages_of(len[k]);
    take[k] = t.pages_of(static_cast<int>(end)) - held;
    if (grow[k] > 0 && t.in_page(len[k]) != 0) {
      const int p = t.row(b)[held - 1];
      if (static_cast<uint32_t>(p) >= static_cast<uint32_t>(t.num_pages) || t.refs[p] < 1) {
        report(C, 124, i, p);
        s.bad = 1;
      } else if (t.refs[p] > 1) {
        last[k] = sharing[i] = p;
        n_sharing = 1;
      }
    }
  }
  __syncthreads();
  if (n_sharing) {
    // entries before this one that share its last page get pages of their own first
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = k * kThreads + threadIdx.x;
      if (last[k] < 0) continue;
      int left = t.refs[last[k]];
      for (int x = 0; x < i; ++x) left -= sharing[x] == last[k];
      if (left <= 1) {
        last[k] = -1;
      } else if (!M.pairs) {                                // nobody would learn which page to copy
        report(C, 130, i, last[k]);
        s.bad = 1;
      } else {
        ++take[k];
      }
    }
  }
  const int64_t total = entry_sums(take, C.n, s.at, s), all_rows = entry_sums(grow, C.n, M.cu, s);
  if (threadIdx.x == 0 && (count < 0 || count > t.num_pages || total > count || all_rows > M.max_rows)) {
    report(C, 128, static_cast<int>(min(total, static_cast<int64_t>(INT32_MAX))), count);
    s.bad = 1;
  }
  __syncthreads();
  // the pages that the call takes are the pool's, and nobody's
  const bool bad = s.bad;
  const int sum = bad ? 0 : static_cast<int>(total);
  __syncthreads();
  int p[kBatch], r[kBatch];
  auto load = [&](int k, int j, int) { p[k] = now(t.free_list + (count - 1 - j)); };
  auto holders = [&](int k) { r[k] = static_cast<uint32_t>(p[k]) < static_cast<uint32_t>(t.num_pages) ? now(t.refs + p[k]) : -1; };
  for_places<CL>(s.at, C.n, sum, load, holders, [&](int k, int j, int) {
    if (r[k] != 0) {
      report(C, 129, count - 1 - j, p[k]);
      raise_flag<CL>(&s.wrong);
    }
  });
  sync_all<CL>();
  const bool leads = CL == 1 || cluster_ctarank() == 0;
  if (bad || s.wrong) {                                     // nothing is changed, and nothing is there to be written
    for (int i = threadIdx.x; i <= C.n; i += kThreads) {
      M.cu[i] = 0;
      if (M.pairs && i < C.n) M.pairs[i] = make_int2(0, 0);
    }
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = k * kThreads + threadIdx.x;
      if (i >= C.n) continue;
      sharing[i] = t.pages_of(len[k]) - (last[k] >= 0);     // the column of the first page that it takes
      if (!leads) continue;
      int2 pair = make_int2(0, 0);
      if (last[k] >= 0) {
        pair = make_int2(last[k], t.free_list[count - 1 - s.at[i]]);
        atomicSub(t.refs + last[k], 1);
      }
      if (M.pairs) M.pairs[i] = pair;
      t.lengths[seq[k]] = len[k] + grow[k];
    }
    __syncthreads();
    for_places<CL>(s.at, C.n, sum, load, Nothing(), [&](int k, int j, int e) {
      t.row(C.seqs ? __ldg(C.seqs + e) : e)[sharing[e] + j - s.at[e]] = p[k];
      t.refs[p[k]] = 1;
    });
    if (threadIdx.x == 0 && leads) *t.free_count = count - sum;
  }
  __syncthreads();
  if constexpr (CL == 1) {                                  // (longer maps are the next kernel's)
    if (M.max_rows > kInlineRows) return;
    for (int i = threadIdx.x; i <= C.n; i += kThreads) s.at[i] = M.cu[i];
    __syncthreads();
    for (int64_t j = threadIdx.x; j < M.max_rows; j += kBatch * kThreads) write_maps(C, M, s.at, j, kThreads);
  }
}

__global__ void __launch_bounds__(256) pages_map_kernel(const __grid_constant__ Call C, const __grid_constant__ Maps M) {
  __shared__ int32_t cu[APACK_MAX_SEQS + 1];
  pdl_wait_and_release();
  for (int i = threadIdx.x; i <= C.n; i += 256) cu[i] = M.cu[i];
  __syncthreads();
  for (int64_t j = blockIdx.x * 256ll + threadIdx.x; j < M.max_rows; j += kBatch * 256ll * gridDim.x)
    write_maps(C, M, cu, j, 256ll * gridDim.x);
}

// ---------------------------------------------------------------- host side

bool int_aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

apack_status make_call(const apack_page_tables *t, int32_t n, const int32_t *seqs, const int32_t *rows, void *ws, Call *C) {
  if (!t || !t->page_table || !t->lengths || !t->refs || !t->free_list || !t->free_count) return APACK_EINVAL;
  if (t->num_seqs < 1 || t->num_seqs > APACK_MAX_SEQS || t->max_pages < 1 || t->num_pages < 1 ||
      t->table_stride < t->max_pages || t->page_tokens < 1 || t->page_tokens > (1 << 30))
    return APACK_EINVAL;
  if (n < 0 || n > APACK_MAX_SEQS || (!seqs && n > t->num_seqs) || (n > 0 && !rows)) return APACK_EINVAL;
  if (!int_aligned(t->page_table) || !int_aligned(t->lengths) || !int_aligned(t->refs) || !int_aligned(t->free_list) ||
      !int_aligned(t->free_count) || !int_aligned(seqs) || !int_aligned(rows) || (reinterpret_cast<uintptr_t>(ws) & 15))
    return APACK_EINVAL;
  std::memset(C, 0, sizeof(*C));
  C->t.table = t->page_table;
  C->t.table_stride = t->table_stride;
  C->t.lengths = t->lengths;
  C->t.refs = t->refs;
  C->t.free_list = t->free_list;
  C->t.free_count = t->free_count;
  C->t.num_seqs = t->num_seqs;
  C->t.max_pages = t->max_pages;
  C->t.num_pages = t->num_pages;
  C->t.page_tokens = fast_div(static_cast<uint32_t>(t->page_tokens));
  C->n = n;
  C->seqs = seqs;
  C->rows = rows;
  C->err = static_cast<DeviceError *>(ws);
  return APACK_OK;
}

// One CTA, or a cluster.
template <class... K, class... A>
cudaError_t launch_cluster(void (*kernel)(K...), int ctas, cudaStream_t stream, A &&...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = ctas;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<K>(args)...);
}

bool large(const Call &C) { return static_cast<int64_t>(C.n) * C.t.max_pages > kClusterPages; }

apack_status launched(cudaError_t e) {
  if (e == cudaSuccess) count_launches(1);
  return check_cuda(e);
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

apack_status apack_pages_release(const apack_page_tables *tables, int32_t n, const int32_t *seqs, const int32_t *keep_rows,
                                 void *ws, void *stream) {
  Call C;
  const apack_status st = make_call(tables, n, seqs, keep_rows, ws, &C);
  if (st != APACK_OK || n == 0) return st;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  return launched(large(C) ? launch_cluster(pages_release_kernel<kMaxCluster>, kMaxCluster, cs, C)
                           : launch_cluster(pages_release_kernel<1>, 1, cs, C));
}

apack_status apack_pages_fork(const apack_page_tables *tables, int32_t n, const int32_t *parents, const int32_t *seqs,
                              void *ws, void *stream) {
  Call C;
  const apack_status st = make_call(tables, n, seqs, parents, ws, &C);
  if (st != APACK_OK) return st;
  if (n > 0 && !seqs) return APACK_EINVAL;
  if (n == 0) return APACK_OK;
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  return launched(large(C) ? launch_cluster(pages_fork_kernel<kMaxCluster>, kMaxCluster, cs, C)
                           : launch_cluster(pages_fork_kernel<1>, 1, cs, C));
}

apack_status apack_pages_extend(const apack_page_tables *tables, int32_t n, const int32_t *seqs, const int32_t *new_rows,
                                int32_t *cu_new, int64_t max_rows, int32_t *rows, int32_t *row_seqs, int64_t *slots,
                                int32_t *pairs, void *ws, void *stream) {
  Call C;
  const apack_status st = make_call(tables, n, seqs, new_rows, ws, &C);
  if (st != APACK_OK) return st;
  if (!cu_new || max_rows < 0 || max_rows > INT32_MAX || (max_rows > 0 && !rows)) return APACK_EINVAL;
  if (!int_aligned(cu_new) || !int_aligned(rows) || !int_aligned(row_seqs) || (reinterpret_cast<uintptr_t>(slots) & 7) ||
      (reinterpret_cast<uintptr_t>(pairs) & 7))
    return APACK_EINVAL;
  Maps M{cu_new, rows, row_seqs, slots, reinterpret_cast<int2 *>(pairs), max_rows};
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  if (max_rows <= kInlineRows) return launched(launch_cluster(pages_extend_kernel<1>, 1, cs, C, M));
  // (as many pages as the new rows need at most)
  const bool many = std::min(max_rows / tables->page_tokens + 2 * static_cast<int64_t>(n), static_cast<int64_t>(C.t.num_pages)) > kClusterPages;
  const apack_status r = launched(many ? launch_cluster(pages_extend_kernel<kMaxCluster>, kMaxCluster, cs, C, M)
                                       : launch_cluster(pages_extend_kernel<1>, 1, cs, C, M));
  if (r != APACK_OK) return r;
  const int grid = static_cast<int>(std::min<int64_t>(4 * device_sm_count(), (max_rows + kBatch * 256 - 1) / (kBatch * 256)));
  return launched(launch_pdl(pages_map_kernel, dim3(grid), dim3(256), 0, cs, C, M));
}

}  // extern "C"
