// The tables of paged caches: the next step's (sequences that go on, fork, give rows back or end, and room for new
// rows), and the compaction of a cache to its rows of lowest key norm.  The tables are the only state: a page is free where no
// table names it below its sequence's length and it is not pinned, so every call works out anew which pages are held.
// Nothing can leak, and a call has the same result however often it is repeated.
//
//   page_begin_kernel   marks: nothing but the pinned pages is held
//   page_mark_kernel    every entry in use claims its page (atomicMax of rows used, then of the lower (b, l)); for a
//                       compaction, besides, a block per (b, l, h) takes its keys through the table and selects
//   page_deal_kernel    the free pages in ascending order, from counts per kPageGroup pages that the first claims have kept;
//                       one block: what each (b, l) asks for, and where its pages begin in that order
//   page_update_kernel  the new tables, and the rows of the pages that are copied
//   page_compact_kernel the new tables, and the kept rows, gathered as select_compact gathers them
#include <algorithm>
#include <climits>

#include "select_unit.cuh"
#include "tokens.cuh"

namespace l2kv {

constexpr int kPageThreads = 256;
constexpr int kDealThreads = 1024;
constexpr int kPageGroup = 256;                          // pages per count of held ones
constexpr int kCopyHeads = 4;                            // heads whose rows one block copies
constexpr uint32_t kPinned = 0xffffffffu;

// One (b, l) of a call.
struct PageAsk {
  int have, more;        // pages of the rows that it keeps, and with those it asks for
  int part;              // rows in the last kept page, where that is not full
  bool grows;
};
__device__ __forceinline__ int pages_of(long long rows, const PageView& v) { return (int)((rows + v.rows() - 1) >> v.shift); }
// The sequence that (b, l) goes on from; -1: none.
__device__ __forceinline__ int parent_of(const PageUpdate& a, int b) {
  const int p = a.parent[b];
  return p >= 0 && p < a.B_in ? p : -1;
}
__device__ __forceinline__ int kept_rows(const PageUpdate& a, int b, int l) {
  return parent_of(a, b) < 0 ? 0 : max(0, min(a.keep[(long long)b * a.L + l], a.in.cap << a.in.shift));
}
__device__ __forceinline__ PageAsk ask_of(const PageUpdate& a, int b, int l) {
  const int keep = kept_rows(a, b, l), grow = max(0, a.grow[b]);
  return {pages_of(keep, a.in), pages_of((long long)keep + grow, a.in), keep & (a.in.rows() - 1), grow > 0};
}
__device__ __forceinline__ int cached_rows(const PageCompact& a, long long u) { return max(0, min(a.len[u], min(a.max_len, a.in.cap << a.in.shift))); }

struct PageScratch {
  uint32_t* mark;
  int32_t* used;
  int32_t* order;
  int2* deal;            // per (b, l): where its pages begin in the order (-1: it gets none); update: whether its last
                         // page is copied, compaction: its length
  int entries;
};

// need[u] of a compaction: a page that is none among its entries
constexpr int kBadPage = -2;

__global__ void __launch_bounds__(kPageThreads)
page_begin_kernel(PageScratch w, const uint8_t* pin, int n_pages) {
  next_may_start();
  wait_for_previous();
  const int p = blockIdx.x * kPageGroup + threadIdx.x;
  const bool pinned = p < n_pages && pin && pin[p];
  if (p < n_pages) w.mark[p] = pinned ? kPinned : 0u;
  const int held = __syncthreads_count(pinned);
  if (threadIdx.x == 0) w.used[blockIdx.x] = held;
  for (long long u = (long long)blockIdx.x * kPageThreads + threadIdx.x; u < w.entries; u += (long long)gridDim.x * kPageThreads)
    w.deal[u] = make_int2(-1, 0);
}

// Claims of the entries [0, n) of one table row, by a warp, four to a lane at a time.  COUNT: the first claim on a page adds to
// its group's count of held ones.
template <bool COUNT>
__device__ __forceinline__ void claim_pages(const PageScratch& w, const PageView& in, const int32_t* row, int n, long long u, int rows,
                                            int32_t* status, bool* bad) {
  const uint32_t who = (1u << kClaimBits) - 1u - (uint32_t)u;
  for (int j0 = threadIdx.x & 31; j0 < n; j0 += 128) {
    int page[4];
    uint32_t was[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      page[i] = j0 + 32 * i < n ? row[j0 + 32 * i] : INT_MAX;
      was[i] = 1;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = j0 + 32 * i;
      if (in.valid(page[i])) {
        const uint32_t claim = (uint32_t)min(in.rows(), rows - (j << in.shift)) << kClaimBits | who;
        if (COUNT) was[i] = atomicMax(w.mark + page[i], claim);
        else atomicMax(w.mark + page[i], claim);
      } else if (j < n) {
        *bad = true;
      }
    }
    if (COUNT) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (was[i] == 0) atomicAdd(w.used + page[i] / kPageGroup, 1);
    }
  }
  *bad = __any_sync(0xffffffffu, *bad);
  if (*bad && (threadIdx.x & 31) == 0) atomicExch(status, (int)L2KV_ERR_OUT_OF_RANGE);
}

__global__ void __launch_bounds__(kPageThreads)
page_mark_kernel(const __grid_constant__ PageUpdate a, PageScratch w) {
  next_may_start();
  wait_for_previous();
  const long long u = (long long)blockIdx.x * (kPageThreads / 32) + (threadIdx.x >> 5);
  if (u >= w.entries) return;
  const int b = (int)(u / a.L), l = (int)(u % a.L);
  bool bad = a.parent[b] >= a.B_in;                      // (told, and taken as none)
  const int keep = kept_rows(a, b, l);
  claim_pages<true>(w, a.in, a.in.of(max(0, parent_of(a, b)), l), pages_of(keep, a.in), u, keep, a.status, &bad);
}

// A (b, l)'s keys in row order, and the selection, a block per head; further blocks claim.
struct CompactSelect {
  const float* sumsq;
  float* keys;
  UnitRec* units;
  int2* chunks;
  long long ld, total_rows;
  int n_chunks;
};
template <int NT>
__global__ void __launch_bounds__(NT, 1024 / NT)
page_mark_select_kernel(const __grid_constant__ PageCompact a, PageScratch w, CompactSelect c) {
  __shared__ SelectSmem sm;
  next_may_start();
  wait_for_previous();
  const long long units = (long long)w.entries * a.H;
  if (blockIdx.x >= units) {
    const long long u = (blockIdx.x - units) * (NT / 32) + (threadIdx.x >> 5);
    if (u >= w.entries) return;
    const int rows = cached_rows(a, u);
    bool bad = false;
    claim_pages<true>(w, a.in, a.in.of((int)(u / a.L), (int)(u % a.L)), pages_of(rows, a.in), u, rows, a.status, &bad);
    if (bad && (threadIdx.x & 31) == 0) w.deal[u].x = kBadPage;
    return;
  }
  const long long unit = blockIdx.x, u = unit / a.H;
  const int h = (int)(unit % a.H), len = cached_rows(a, u), keep = a.keep[u];
  if (keep >= len || keep <= 0) return;                  // stays whole, or keeps nothing
  const int32_t* const row = a.in.of((int)(u / a.L), (int)(u % a.L));
  const float* const from = c.sumsq + h * c.total_rows;
  float* const keys = c.keys + unit * c.ld;
  constexpr int kBatch = 8;
  for (int t0 = 0; t0 < len; t0 += kBatch * NT) {
    float x[kBatch];
    int page[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + i * NT + (int)threadIdx.x;
      page[i] = t < len ? row[t >> a.in.shift] : -1;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + i * NT + (int)threadIdx.x;
      x[i] = a.in.valid(page[i]) ? from[((long long)page[i] << a.in.shift) | (t & (a.in.rows() - 1))] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + i * NT + (int)threadIdx.x;
      if (t < len) keys[t] = x[i];
    }
  }
  __syncthreads();
  select_unit<NT>(sm, keys, len, keep, a.policy, 0, c.units + unit, c.chunks + unit * c.n_chunks);
}

// Inclusive sum over the block's threads; *total: of all.
template <typename N>
__device__ __forceinline__ N block_sum(N x, N* s_warp, N* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  N incl = x;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const N o = __shfl_up_sync(0xffffffffu, incl, off);
    if (lane >= off) incl += o;
  }
  __syncthreads();
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  N sums = lane < (int)blockDim.x / 32 ? s_warp[lane] : 0;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const N o = __shfl_up_sync(0xffffffffu, sums, off);
    if (lane >= off) sums += o;
  }
  *total = __shfl_sync(0xffffffffu, sums, 31);
  const N before = __shfl_sync(0xffffffffu, sums, max(0, warp - 1));
  return incl + (warp ? before : 0);
}

// What (b, l) = u asks for: pages, and whether its last kept page is copied.  A page that several hold stays with the one that
// has most rows in it, the first of several: it writes behind them; the others copy.
__device__ __forceinline__ int2 need_of(const PageUpdate& a, const PageScratch& w, long long u) {
  const int b = (int)(u / a.L), l = (int)(u % a.L);
  const PageAsk q = ask_of(a, b, l);
  if (!q.grows) return make_int2(0, 0);
  if (q.more > a.in.cap) {
    atomicExch(a.status, (int)L2KV_ERR_DEVICE_OVERFLOW);
    return make_int2(0, 0);
  }
  int copy = 0;
  if (q.part) {
    const int page = a.in.of(parent_of(a, b), l)[q.have - 1];
    const uint32_t claim = (uint32_t)q.part << kClaimBits | ((1u << kClaimBits) - 1u - (uint32_t)u);
    copy = a.in.valid(page) && w.mark[page] != claim;
  }
  return make_int2(q.more - q.have + copy, copy);
}
__device__ __forceinline__ int2 need_of(const PageCompact& a, const PageScratch& w, long long u) {
  const int len = cached_rows(a, u), keep = max(0, a.keep[u]);
  return make_int2(keep >= len || w.deal[u].x == kBadPage ? 0 : pages_of(keep, a.in), len);   // (len_out may be len)
}
__device__ __forceinline__ bool asks(const PageUpdate& a, const PageScratch&, long long u) {
  const PageAsk q = ask_of(a, (int)(u / a.L), (int)(u % a.L));
  return q.grows && q.more <= a.in.cap;
}
__device__ __forceinline__ bool asks(const PageCompact& a, const PageScratch& w, long long u) {
  return w.deal[u].x != kBadPage && max(0, a.keep[u]) < cached_rows(a, u);
}

// By a block of kDealThreads: what every (b, l) gets of the n_all free pages, into w.deal; the pages given in all are returned.
// Four (b, l) to a thread: what it takes is a chain of loads (the request, the last page, the claim on it) and sums.
constexpr int kAsks = 4;
template <typename A>
__device__ __forceinline__ long long deal_out(const A& a, const PageScratch& w, int n_all, int32_t* n_free) {
  __shared__ long long s_sums[32];
  long long before = 0, given = 0, all;
  for (int u0 = 0; u0 < w.entries; u0 += kAsks * kDealThreads) {
    int2 need[kAsks];
    bool wants[kAsks];
    long long mine = 0;
#pragma unroll
    for (int i = 0; i < kAsks; ++i) {
      const int u = u0 + (int)threadIdx.x * kAsks + i;
      need[i] = make_int2(0, 0);
      wants[i] = u < w.entries && asks(a, w, u);
      if (u < w.entries) need[i] = need_of(a, w, u);
      mine += need[i].x;
    }
    long long upto = before + block_sum<long long>(mine, s_sums, &all) - mine;
#pragma unroll
    for (int i = 0; i < kAsks; ++i) {
      const int u = u0 + (int)threadIdx.x * kAsks + i;
      upto += need[i].x;
      const bool gets = wants[i] && (need[i].x == 0 || upto <= n_all);
      if (wants[i] && !gets) atomicExch(a.status, (int)L2KV_ERR_DEVICE_OVERFLOW);
      if (u < w.entries) w.deal[u] = make_int2(!gets ? -1 : need[i].x ? (int)(upto - need[i].x) : 0, need[i].y);
      if (gets) given += need[i].x;
    }
    before += all;
  }
  block_sum(given, s_sums, &all);
  if (n_free && threadIdx.x == 0) *n_free = n_all - (int)all;
  return all;
}

template <typename A>
__global__ void __launch_bounds__(kDealThreads)
page_deal_kernel(const __grid_constant__ A a, PageScratch w, int n_pages, int n_groups, int32_t* n_free) {
  __shared__ int s_warp[32];
  next_may_start();
  wait_for_previous();
  // free pages before the block's own; in the last block, all
  const bool deals = blockIdx.x == gridDim.x - 1;
  const int first_group = deals ? n_groups : (int)blockIdx.x * (kPageBlock / kPageGroup);
  int x = 0, held;
  for (int i = threadIdx.x; i < first_group; i += kDealThreads) x += w.used[i];
  block_sum(x, s_warp, &held);
  if (!deals) {
    constexpr int kEach = kPageBlock / kDealThreads;
    const int p0 = (int)blockIdx.x * kPageBlock + (int)threadIdx.x * kEach;
    bool is_free[kEach];
    int n = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      is_free[i] = p0 + i < n_pages && w.mark[p0 + i] == 0;
      n += is_free[i];
    }
    int at = first_group * kPageGroup - held + block_sum(n, s_warp, &all) - n;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (is_free[i]) w.order[at++] = p0 + i;
    return;
  }
  deal_out(a, w, n_pages - held, n_free);
}

// Rows of one page to another, for heads [h0, h1): kCopyAhead pieces of K and of V per thread in flight.
constexpr int kCopyAhead = 4;
template <typename T, int D>
__device__ __forceinline__ void copy_rows(T* K, T* V, int32_t* idx, float* sumsq, const Geom& g, long long from, long long to, int rows,
                                          int h0, int h1, int thread, int threads) {
  constexpr int LPR = D / Elem<T>::kPerVec;
  const int n = (h1 - h0) * rows;
  const int piece = thread % LPR, step = threads / LPR;  // a row to LPR threads
  for (int e0 = thread / LPR; e0 < n; e0 += kCopyAhead * step) {
    uint4 k[kCopyAhead], v[kCopyAhead];
    long long at[kCopyAhead];
#pragma unroll
    for (int i = 0; i < kCopyAhead; ++i) {
      const int e = e0 + i * step, h = h0 + e / rows, r = e % rows;
      at[i] = h * g.sh + r * g.st + piece * Elem<T>::kPerVec;
      if (e >= n) continue;
      k[i] = ld_once(K + at[i] + from * g.st);
      v[i] = ld_once(V + at[i] + from * g.st);
      if (piece == 0) {
        const long long m = h * g.total_rows + r;
        if (idx) idx[m + to] = idx[m + from];
        if (sumsq) sumsq[m + to] = sumsq[m + from];
      }
    }
#pragma unroll
    for (int i = 0; i < kCopyAhead; ++i) {
      if (e0 + i * step >= n) continue;
      st_stream(K + at[i] + to * g.st, k[i]);
      st_stream(V + at[i] + to * g.st, v[i]);
    }
  }
}

// The new table of (b, l) = u, by `threads` threads; returns the page its last one is copied from, and through `to` and
// `rows` where; -1: none is.
__device__ __forceinline__ int write_table(const PageUpdate& a, const PageScratch& w, long long u, int thread, int threads, bool writes,
                                           int* to_page, int* rows) {
  const int b = (int)(u / a.L), l = (int)(u % a.L);
  const int2 deal = w.deal[u];
  const bool gets = deal.x >= 0, copies = gets && deal.y;
  const PageAsk q = ask_of(a, b, l);
  const int32_t* const old = a.in.of(max(0, parent_of(a, b)), l);
  if (writes) {
    int32_t* const to = a.out_table + b * a.out.sb + l * a.out.sl;
    const int begin = q.have - (copies ? 1 : 0), more = gets ? q.more : q.have;
#pragma unroll 4
    for (int j = thread; j < a.out.cap; j += threads)
      to[j] = j < begin ? old[j] : j >= more ? -1 : gets ? w.order[deal.x + j - begin] : old[j];
    if (a.out_room && thread == 0) a.out_room[u] = gets ? q.more << a.in.shift : kept_rows(a, b, l);
  }
  if (!copies) return -1;
  *to_page = w.order[deal.x];
  *rows = q.part;
  return old[q.have - 1];
}

// Blocks [0, table_blocks): the tables, a warp per (b, l).  The others, where copies are possible: a block per (b, l) and kCopyHeads heads.
template <typename T, int D>
__global__ void __launch_bounds__(kPageThreads)
page_update_kernel(const __grid_constant__ PageUpdate a, PageScratch w, T* K, T* V, int32_t* idx, float* sumsq, Geom g, int table_blocks,
                   int copy_groups) {
  next_may_start();
  wait_for_previous();
  int to, rows;
  if ((int)blockIdx.x < table_blocks) {
    const long long u = (long long)blockIdx.x * (kPageThreads / 32) + (threadIdx.x >> 5);
    if (u < w.entries) write_table(a, w, u, threadIdx.x & 31, 32, true, &to, &rows);
    return;
  }
  const int i = (int)blockIdx.x - table_blocks;
  const long long u = i / copy_groups;
  const int2 deal = w.deal[u];
  if (deal.x < 0 || !deal.y) return;
  const int from = write_table(a, w, u, 0, 1, false, &to, &rows), h0 = i % copy_groups * kCopyHeads;
  copy_rows<T, D>(K, V, idx, sumsq, g, (long long)from << a.in.shift, (long long)to << a.in.shift, rows, h0, min(g.H, h0 + kCopyHeads),
                  threadIdx.x, kPageThreads);
}

// Pools of up to kSmallPool pages: the claims in one block's shared memory, and with them the free pages and what
// everyone gets.  ALL: the tables and copies too, where they are few.
constexpr int kSmallPool = 49152, kSmallEntries = 65536, kSmallAsks = 4096;
constexpr long long kSmallCopy = 128 << 10;              // bytes that one block copies as fast as another kernel starts
template <typename T, int D, bool ALL>
__global__ void __launch_bounds__(kDealThreads)
page_update_small_kernel(const __grid_constant__ PageUpdate a, PageScratch w, T* K, T* V, int32_t* idx, float* sumsq, Geom g) {
  extern __shared__ uint32_t s_mark[];
  __shared__ int s_warp[32];
  const int tid = threadIdx.x, warp = tid >> 5, n_pages = a.in.n;
  next_may_start();
  wait_for_previous();
  PageScratch mine = w;
  mine.mark = s_mark;
  for (int p = tid; p < n_pages; p += kDealThreads) s_mark[p] = a.pin && a.pin[p] ? kPinned : 0u;
  __syncthreads();
  for (int u = warp; u < w.entries; u += kDealThreads / 32) {
    const int b = u / a.L, l = u % a.L;
    bool bad = a.parent[b] >= a.B_in;
    const int keep = kept_rows(a, b, l);
    claim_pages<false>(mine, a.in, a.in.of(max(0, parent_of(a, b)), l), pages_of(keep, a.in), u, keep, a.status, &bad);
  }
  __syncthreads();
  // a run of pages to each thread, of odd length: no two threads of a warp in one bank
  const int run = (n_pages + kDealThreads - 1) / kDealThreads | 1, p0 = min(n_pages, tid * run), p1 = min(n_pages, p0 + run);
  int n = 0, all;
  for (int p = p0; p < p1; ++p) n += s_mark[p] == 0;
  int at = block_sum(n, s_warp, &all) - n;
  const long long given = deal_out(a, mine, all, a.n_free);
  for (int p = p0; p < p1 && at < given; ++p)
    if (s_mark[p] == 0) w.order[at++] = p;
  if (!ALL) return;
  __syncthreads();
  for (int u = warp; u < w.entries; u += kDealThreads / 32) {
    int to, rows;
    const int from = write_table(a, w, u, tid & 31, 32, true, &to, &rows);
    if (from >= 0)
      copy_rows<T, D>(K, V, idx, sumsq, g, (long long)from << a.in.shift, (long long)to << a.in.shift, rows, 0, g.H, tid & 31, 32);
  }
}

// ---- the kept rows of a compaction ------------------------------------------------------------------
// A block per chunk of kGatherChunk rows of a unit, as in select_compact's gather, or, where those would leave SMs idle, several,
// a part of the chunk's kept rows each: the chunk's rows are ranked from the threshold, where each kept one comes from and
// goes to is noted, and they move 16 bytes a lane, kMoves rows of K and of V per lane in flight.
constexpr int kMoves = 4;
template <typename T, int D>
__global__ void __launch_bounds__(kPageThreads)
page_compact_kernel(const __grid_constant__ PageCompact a, PageScratch w, CompactSelect c, T* K, T* V, int32_t* idx, float* sumsq, Geom g,
                    int parts) {
  constexpr int LPR = D / Elem<T>::kPerVec, RPS = kPageThreads / LPR, TPT = kGatherChunk / kPageThreads;
  __shared__ int s_from[kGatherChunk], s_to[kGatherChunk];   // pool rows that the kept rows move from and to
  __shared__ int s_warp[32];
  next_may_start();
  wait_for_previous();
  const long long chunks = (long long)w.entries * a.H * c.n_chunks;
  if (blockIdx.x >= chunks * parts) {                    // the tables and lengths: a block per (b, l)
    const long long u = blockIdx.x - chunks * parts;
    const int b = (int)(u / a.L), l = (int)(u % a.L), len = w.deal[u].y, at = w.deal[u].x;
    const int rows = at >= 0 ? max(0, a.keep[u]) : len, n = pages_of(rows, a.in);
    const int32_t* const old = a.in.of(b, l);
    int32_t* const to = a.out_table + b * a.out.sb + l * a.out.sl;
    for (int j = threadIdx.x; j < a.out.cap; j += kPageThreads) to[j] = j >= n ? -1 : at >= 0 ? w.order[at + j] : old[j];
    if (threadIdx.x == 0) {
      a.len_out[u] = rows;
      if (a.out_room) a.out_room[u] = rows;
    }
    return;
  }
  const long long unit = blockIdx.x / parts / c.n_chunks, u = unit / a.H;
  const int part = (int)(blockIdx.x % parts), chunk = (int)(blockIdx.x / parts % c.n_chunks), h = (int)(unit % a.H), tid = threadIdx.x;
  const int2 deal = w.deal[u];
  const int len = deal.y, t0 = chunk * kGatherChunk, at = deal.x;
  if (t0 >= len || at < 0 || a.keep[u] <= 0) return;
  const UnitRec rec = c.units[unit];
  const int2 cr = c.chunks[unit * c.n_chunks + chunk];   // slot of the chunk's first kept row, ties before it
  const float* const key = c.keys + unit * c.ld;
  const int32_t* const row = a.in.of((int)(u / a.L), (int)(u % a.L));
  uint32_t bits[TPT];
  int page[TPT], count = 0;                              // rows below the threshold in the upper half, at it in the lower
#pragma unroll
  for (int i = 0; i < TPT; ++i) {
    const int t = t0 + tid * TPT + i;
    bits[i] = t < len ? order_bits(key[t], a.policy) : 0u;
    page[i] = t < len ? row[t >> a.in.shift] : 0;
    if (t < len) count += bits[i] < rec.thr ? 0x10000 : bits[i] == rec.thr;
  }
  int all;
  int before = block_sum(count, s_warp, &all) - count;
  const int taken = min(cr.y, rec.admit);                // ties taken in the chunks before
#pragma unroll
  for (int i = 0; i < TPT; ++i) {
    const int t = t0 + tid * TPT + i;
    if (t >= len) continue;
    const int ties = cr.y + (before & 0xffff);
    const bool less = bits[i] < rec.thr, tie = bits[i] == rec.thr;
    if (less || (tie && ties < rec.admit)) {
      const int j = (before >> 16) + min(ties, rec.admit) - taken, slot = cr.x + j;
      const bool ok = L2KV_BOUNDS(j >= 0 && j < kGatherChunk && slot >= 0 && slot < rec.n_keep, a.status);
      if (ok) {
        s_from[j] = (page[i] << a.in.shift) | (t & (a.in.rows() - 1));
        s_to[j] = (w.order[at + (slot >> a.in.shift)] << a.in.shift) | (slot & (a.in.rows() - 1));
      }
    }
    before += less ? 0x10000 : tie;
  }
  __syncthreads();
  const int n_kept = (all >> 16) + min(cr.y + (all & 0xffff), rec.admit) - taken;
  const int j1 = (int)((long long)n_kept * (part + 1) / parts);
  const int piece = tid % LPR, sub = tid / LPR;
  const long long mine = h * g.sh + piece * Elem<T>::kPerVec, meta = h * g.total_rows;
  for (int j0 = (int)((long long)n_kept * part / parts); j0 < j1; j0 += RPS * kMoves) {
    uint4 k[kMoves], v[kMoves];
    int from[kMoves], to[kMoves], pos[kMoves];
    float sum[kMoves];
#pragma unroll
    for (int i = 0; i < kMoves; ++i) {
      const int j = j0 + i * RPS + sub;
      from[i] = j < j1 ? s_from[j] : -1;
      if (from[i] >= 0 && !L2KV_BOUNDS(from[i] < g.total_rows && s_to[j] >= 0 && s_to[j] < g.total_rows, a.status)) from[i] = -1;
      if (from[i] < 0) continue;
      to[i] = s_to[j];
      k[i] = ld_once(K + mine + from[i] * g.st);
      v[i] = ld_once(V + mine + from[i] * g.st);
      if (piece == 0) {
        if (idx) pos[i] = idx[meta + from[i]];
        sum[i] = sumsq[meta + from[i]];
      }
    }
#pragma unroll
    for (int i = 0; i < kMoves; ++i) {
      if (from[i] < 0) continue;
      st_stream(K + mine + to[i] * g.st, k[i]);
      st_stream(V + mine + to[i] * g.st, v[i]);
      if (piece == 0) {
        if (idx) idx[meta + to[i]] = pos[i];
        sumsq[meta + to[i]] = sum[i];
      }
    }
  }
}

// ---- host ------------------------------------------------------------------------------------------

PagePlan plan_pages(long long entries, long long units, int n_pages, int max_len) {
  PagePlan p;
  size_t off = 0;
  auto take = [&](long long bytes) {
    const size_t at = off;
    off += (size_t)round_up_ll(bytes, 256);
    return at;
  };
  p.ld = round_up_ll(max_len > 0 ? max_len : 1, 64);
  p.n_chunks = std::max(1, (max_len + kGatherChunk - 1) / kGatherChunk);
  p.mark_off = take(4ll * n_pages);
  p.used_off = take(4ll * std::max(1, (n_pages + kPageGroup - 1) / kPageGroup));
  p.order_off = take(4ll * n_pages);
  p.need_off = take(8 * entries);
  p.key_off = take(4 * units * p.ld);
  p.unit_off = take(16 * units);
  p.chunk_off = take(8 * units * p.n_chunks);
  p.total = off;
  return p;
}

static PageScratch scratch_of(const PagePlan& p, char* base, long long entries) {
  return PageScratch{reinterpret_cast<uint32_t*>(base + p.mark_off), reinterpret_cast<int32_t*>(base + p.used_off),
                     reinterpret_cast<int32_t*>(base + p.order_off), reinterpret_cast<int2*>(base + p.need_off), (int)entries};
}
static int groups_of(int n_pages) { return std::max(1, (n_pages + kPageGroup - 1) / kPageGroup); }
static int begin_pages(const PageScratch& w, const uint8_t* pin, int n_pages, cudaStream_t s) {
  return launch_chained(page_begin_kernel, groups_of(n_pages), 1, kPageThreads, 0, s, w, pin, n_pages);
}
template <typename A>
static int deal_pages(const A& a, const PageScratch& w, int n_pages, int32_t* n_free, cudaStream_t s) {
  return launch_chained(page_deal_kernel<A>, (n_pages + kPageBlock - 1) / kPageBlock + 1, 1, kDealThreads, 0, s, a, w, n_pages,
                        (n_pages + kPageGroup - 1) / kPageGroup, n_free);
}

template <typename T, int D, bool ALL>
static int launch_ps(const PageUpdate& a, const PageScratch& w, void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, cudaStream_t s) {
  auto kern = page_update_small_kernel<T, D, ALL>;
  const size_t smem = ((size_t)a.in.n * 4 + 15) / 16 * 16;
  if (smem > 40 << 10 && cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallPool * 4) != cudaSuccess)
    return L2KV_ERR_CUDA;
  return launch_chained(kern, 1, 1, kDealThreads, smem, s, a, w, static_cast<T*>(K), static_cast<T*>(V), idx, sumsq, g);
}

template <typename T, int D>
static int launch_pu(const PageUpdate& a, const PageScratch& w, void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, cudaStream_t s) {
  int rc;
  if (a.in.n <= kSmallPool && w.entries <= kSmallAsks && (long long)w.entries * a.in.cap <= kSmallEntries) {
    // (what all of them together can have to copy)
    const bool all = w.entries <= 32 && (long long)w.entries * g.H * (2 * (D * sizeof(T) + 4) << a.in.shift) <= kSmallCopy;
    if (all) return launch_ps<T, D, true>(a, w, K, V, idx, sumsq, g, s);
    rc = launch_ps<T, D, false>(a, w, K, V, idx, sumsq, g, s);
  } else {
    rc = begin_pages(w, a.pin, a.in.n, s);
    if (rc != L2KV_OK) return rc;
    constexpr int kWarps = kPageThreads / 32;
    rc = launch_chained(page_mark_kernel, (w.entries + kWarps - 1) / kWarps, 1, kPageThreads, 0, s, a, w);
    if (rc != L2KV_OK) return rc;
    rc = deal_pages(a, w, a.in.n, a.n_free, s);
  }
  if (rc != L2KV_OK) return rc;
  const long long table_blocks = (w.entries + kPageThreads / 32 - 1) / (kPageThreads / 32), groups = (g.H + kCopyHeads - 1) / kCopyHeads;
  if (table_blocks + w.entries * groups > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  return launch_chained(page_update_kernel<T, D>, table_blocks + w.entries * groups, 1, kPageThreads, 0, s, a, w, static_cast<T*>(K),
                        static_cast<T*>(V), idx, sumsq, g, (int)table_blocks, (int)groups);
}

int launch_page_update(const PageUpdate& a, void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, int dtype,
                       char* scratch, cudaStream_t s) {
  const long long entries = (long long)a.B * a.L;
  const PageScratch w = scratch_of(plan_pages(entries, 0, a.in.n, 0), scratch, entries);
  if (dtype == L2KV_BF16) return g.D == 128 ? launch_pu<__nv_bfloat16, 128>(a, w, K, V, idx, sumsq, g, s) : launch_pu<__nv_bfloat16, 64>(a, w, K, V, idx, sumsq, g, s);
  return g.D == 128 ? launch_pu<float, 128>(a, w, K, V, idx, sumsq, g, s) : launch_pu<float, 64>(a, w, K, V, idx, sumsq, g, s);
}

template <int NT>
static int launch_select(const PageCompact& a, const PageScratch& w, const CompactSelect& c, long long units, cudaStream_t s) {
  return launch_chained(page_mark_select_kernel<NT>, units + (w.entries + NT / 32 - 1) / (NT / 32), 1, NT, 0, s, a, w, c);
}

template <typename T, int D>
static int launch_pc(const PageCompact& a, const PageScratch& w, const CompactSelect& c, void* K, void* V, int32_t* idx, float* sumsq,
                     const Geom& g, cudaStream_t s) {
  const long long chunks = (long long)w.entries * a.H * c.n_chunks;
  const int parts = chunks < 2 * 148 ? 4 : 1;
  return launch_chained(page_compact_kernel<T, D>, chunks * parts + w.entries, 1, kPageThreads, 0, s, a, w, c, static_cast<T*>(K),
                        static_cast<T*>(V), idx, sumsq, g, parts);
}

int launch_page_compact(const PageCompact& a, void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, int dtype,
                        char* scratch, cudaStream_t s) {
  const long long entries = (long long)a.B * a.L, units = entries * a.H;
  const PagePlan p = plan_pages(entries, units, a.in.n, a.max_len);
  if (p.n_chunks > kMaxChunks || units * p.n_chunks + entries > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  const PageScratch w = scratch_of(p, scratch, entries);
  const CompactSelect c{sumsq, reinterpret_cast<float*>(scratch + p.key_off), reinterpret_cast<UnitRec*>(scratch + p.unit_off),
                        reinterpret_cast<int2*>(scratch + p.chunk_off), p.ld, g.total_rows, p.n_chunks};
  int rc = begin_pages(w, a.pin, a.in.n, s);
  if (rc != L2KV_OK) return rc;
  // a block per unit: as many threads as the SMs have room for at once
  rc = units <= 148 ? launch_select<1024>(a, w, c, units, s) : launch_select<512>(a, w, c, units, s);
  if (rc != L2KV_OK) return rc;
  rc = deal_pages(a, w, a.in.n, nullptr, s);
  if (rc != L2KV_OK) return rc;
  if (dtype == L2KV_BF16) return g.D == 128 ? launch_pc<__nv_bfloat16, 128>(a, w, c, K, V, idx, sumsq, g, s) : launch_pc<__nv_bfloat16, 64>(a, w, c, K, V, idx, sumsq, g, s);
  return g.D == 128 ? launch_pc<float, 128>(a, w, c, K, V, idx, sumsq, g, s) : launch_pc<float, 64>(a, w, c, K, V, idx, sumsq, g, s);
}

}  // namespace l2kv
