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
constexpr int kCopyHeads = 8;                            // heads whose rows one block copies
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

// Claims of the entries [0, n) of one table row, by a warp.
__device__ __forceinline__ void claim_pages(const PageScratch& w, const PageView& in, const int32_t* row, int n, long long u, int rows,
                                            int32_t* status, bool* bad) {
  const uint32_t who = (1u << kClaimBits) - 1u - (uint32_t)u;
  for (int j = threadIdx.x & 31; j < n; j += 32) {
    const int page = row[j];
    if (!in.valid(page)) { *bad = true; continue; }
    const uint32_t claim = (uint32_t)min(in.rows(), rows - (j << in.shift)) << kClaimBits | who;
    if (atomicMax(w.mark + page, claim) == 0) atomicAdd(w.used + page / kPageGroup, 1);
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
  claim_pages(w, a.in, a.in.of(max(0, parent_of(a, b)), l), pages_of(keep, a.in), u, keep, a.status, &bad);
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
__global__ void __launch_bounds__(kPageThreads)
page_mark_select_kernel(const __grid_constant__ PageCompact a, PageScratch w, CompactSelect c) {
  __shared__ SelectSmem sm;
  next_may_start();
  wait_for_previous();
  const long long units = (long long)w.entries * a.H;
  if (blockIdx.x >= units) {
    const long long u = (blockIdx.x - units) * (kPageThreads / 32) + (threadIdx.x >> 5);
    if (u >= w.entries) return;
    const int rows = cached_rows(a, u);
    bool bad = false;
    claim_pages(w, a.in, a.in.of((int)(u / a.L), (int)(u % a.L)), pages_of(rows, a.in), u, rows, a.status, &bad);
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
  for (int t0 = 0; t0 < len; t0 += kBatch * kPageThreads) {
    float x[kBatch];
    int page[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + i * kPageThreads + (int)threadIdx.x;
      page[i] = t < len ? row[t >> a.in.shift] : -1;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + i * kPageThreads + (int)threadIdx.x;
      x[i] = a.in.valid(page[i]) ? from[((long long)page[i] << a.in.shift) | (t & (a.in.rows() - 1))] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = t0 + i * kPageThreads + (int)threadIdx.x;
      if (t < len) keys[t] = x[i];
    }
  }
  __syncthreads();
  select_unit<kPageThreads>(sm, keys, len, keep, a.policy, 0, c.units + unit, c.chunks + unit * c.n_chunks);
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
__device__ __forceinline__ bool asks(const PageUpdate& a, long long u, int) {
  const PageAsk q = ask_of(a, (int)(u / a.L), (int)(u % a.L));
  return q.grows && q.more <= a.in.cap;
}
__device__ __forceinline__ bool asks(const PageCompact& a, long long u, int was) {
  return was != kBadPage && max(0, a.keep[u]) < cached_rows(a, u);
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
  const int n_all = n_pages - held;
  __shared__ long long s_sums[32];
  long long before = 0, given = 0, all;
  for (int u0 = 0; u0 < w.entries; u0 += kDealThreads) {
    const int u = u0 + (int)threadIdx.x;
    int2 need = make_int2(0, 0);
    bool wants = false;
    if (u < w.entries) {
      wants = asks(a, u, w.deal[u].x);
      need = need_of(a, w, u);
    }
    const long long upto = before + block_sum<long long>(need.x, s_sums, &all);
    const bool gets = wants && (need.x == 0 || upto <= n_all);
    if (wants && !gets) atomicExch(a.status, (int)L2KV_ERR_DEVICE_OVERFLOW);
    if (u < w.entries) w.deal[u] = make_int2(!gets ? -1 : need.x ? (int)(upto - need.x) : 0, need.y);
    if (gets) given += need.x;
    before += all;
  }
  block_sum(given, s_sums, &all);
  if (n_free && threadIdx.x == 0) *n_free = n_all - (int)all;
}

// Rows of one page to another, for some heads.
template <typename T, int D>
__device__ __forceinline__ void copy_rows(T* K, T* V, int32_t* idx, float* sumsq, const Geom& g, long long from, long long to, int rows,
                                          int h0, int h1) {
  constexpr int LPR = D / Elem<T>::kPerVec;
  const int n = (h1 - h0) * rows * LPR;
  for (int e = threadIdx.x; e < n; e += kPageThreads) {
    const int piece = e % LPR, r = e / LPR % rows, h = h0 + e / LPR / rows;
    const long long at = h * g.sh + piece * Elem<T>::kPerVec;
    const uint4 k = ld_once(K + at + (from + r) * g.st), v = ld_once(V + at + (from + r) * g.st);
    st_stream(K + at + (to + r) * g.st, k);
    st_stream(V + at + (to + r) * g.st, v);
    if (piece == 0) {
      const long long m = h * g.total_rows;
      if (idx) idx[m + to + r] = idx[m + from + r];
      if (sumsq) sumsq[m + to + r] = sumsq[m + from + r];
    }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kPageThreads)
page_update_kernel(const __grid_constant__ PageUpdate a, PageScratch w, T* K, T* V, int32_t* idx, float* sumsq, Geom g) {
  next_may_start();
  wait_for_previous();
  const long long u = blockIdx.x;
  const int b = (int)(u / a.L), l = (int)(u % a.L);
  const int2 deal = w.deal[u];
  const bool gets = deal.x >= 0, copies = gets && deal.y;
  if (blockIdx.y > 0 && !copies) return;
  const PageAsk q = ask_of(a, b, l);
  const int32_t* const old = a.in.of(max(0, parent_of(a, b)), l);
  if (blockIdx.y == 0) {
    int32_t* const to = a.out_table + b * a.out.sb + l * a.out.sl;
    const int begin = q.have - (copies ? 1 : 0), more = gets ? q.more : q.have;
    for (int j = threadIdx.x; j < a.out.cap; j += kPageThreads)
      to[j] = j < begin ? old[j] : j >= more ? -1 : gets ? w.order[deal.x + j - begin] : old[j];
    if (a.out_room && threadIdx.x == 0) a.out_room[u] = gets ? q.more << a.in.shift : kept_rows(a, b, l);
  }
  if (copies) {
    const int h0 = (int)blockIdx.y * kCopyHeads;
    copy_rows<T, D>(K, V, idx, sumsq, g, (long long)old[q.have - 1] << a.in.shift, (long long)w.order[deal.x] << a.in.shift, q.part, h0,
                    min(g.H, h0 + kCopyHeads));
  }
}

// ---- the kept rows of a compaction ------------------------------------------------------------------
// A block per chunk of kGatherChunk rows of a unit, as in select_compact's gather: the chunk's kept rows are ranked from the
// threshold, and moved 16 bytes a lane, kMoves rows of K and of V per lane in flight.
constexpr int kMoves = 4;
template <typename T, int D>
__global__ void __launch_bounds__(kPageThreads)
page_compact_kernel(const __grid_constant__ PageCompact a, PageScratch w, CompactSelect c, T* K, T* V, int32_t* idx, float* sumsq, Geom g) {
  constexpr int LPR = D / Elem<T>::kPerVec, RPS = kPageThreads / LPR, TPT = kGatherChunk / kPageThreads;
  __shared__ int s_from[kGatherChunk];                   // pool rows of the kept rows
  __shared__ int s_warp[32];
  next_may_start();
  wait_for_previous();
  const long long units = (long long)w.entries * a.H;
  if (blockIdx.x >= units * c.n_chunks) {                // the tables and lengths: a block per (b, l)
    const long long u = blockIdx.x - units * c.n_chunks;
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
  const long long unit = blockIdx.x / c.n_chunks, u = unit / a.H;
  const int chunk = (int)(blockIdx.x % c.n_chunks), h = (int)(unit % a.H), tid = threadIdx.x;
  const int len = w.deal[u].y, t0 = chunk * kGatherChunk, at = w.deal[u].x;
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
    if (less || (tie && ties < rec.admit))
      s_from[(before >> 16) + min(ties, rec.admit) - taken] = (page[i] << a.in.shift) | (t & (a.in.rows() - 1));
    before += less ? 0x10000 : tie;
  }
  __syncthreads();
  const int n_kept = (all >> 16) + min(cr.y + (all & 0xffff), rec.admit) - taken;
  const int piece = tid % LPR, sub = tid / LPR;
  const long long mine = h * g.sh + piece * Elem<T>::kPerVec, meta = h * g.total_rows;
  for (int j0 = 0; j0 < n_kept; j0 += RPS * kMoves) {
    uint4 k[kMoves], v[kMoves];
    int from[kMoves];
#pragma unroll
    for (int i = 0; i < kMoves; ++i) {
      const int j = j0 + i * RPS + sub;
      from[i] = j < n_kept ? s_from[j] : -1;
      if (from[i] >= 0 && !L2KV_BOUNDS(from[i] < g.total_rows, a.status)) from[i] = -1;
      if (from[i] < 0) continue;
      k[i] = ld_once(K + mine + from[i] * g.st);
      v[i] = ld_once(V + mine + from[i] * g.st);
    }
#pragma unroll
    for (int i = 0; i < kMoves; ++i) {
      if (from[i] < 0) continue;
      const int slot = cr.x + j0 + i * RPS + sub;
      if (!L2KV_BOUNDS(slot >= 0 && slot < rec.n_keep, a.status)) continue;
      const long long to = ((long long)w.order[at + (slot >> a.in.shift)] << a.in.shift) | (slot & (a.in.rows() - 1));
      st_stream(K + mine + to * g.st, k[i]);
      st_stream(V + mine + to * g.st, v[i]);
      if (piece == 0) {
        if (idx) idx[meta + to] = idx[meta + from[i]];
        sumsq[meta + to] = sumsq[meta + from[i]];
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

template <typename T, int D>
static int launch_pu(const PageUpdate& a, const PageScratch& w, void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, cudaStream_t s) {
  return launch_chained(page_update_kernel<T, D>, w.entries, (unsigned)((g.H + kCopyHeads - 1) / kCopyHeads), kPageThreads, 0, s, a, w,
                        static_cast<T*>(K), static_cast<T*>(V), idx, sumsq, g);
}

int launch_page_update(const PageUpdate& a, void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, int dtype,
                       char* scratch, cudaStream_t s) {
  const long long entries = (long long)a.B * a.L;
  const PageScratch w = scratch_of(plan_pages(entries, 0, a.in.n, 0), scratch, entries);
  int rc = begin_pages(w, a.pin, a.in.n, s);
  if (rc != L2KV_OK) return rc;
  constexpr int kWarps = kPageThreads / 32;
  rc = launch_chained(page_mark_kernel, (entries + kWarps - 1) / kWarps, 1, kPageThreads, 0, s, a, w);
  if (rc != L2KV_OK) return rc;
  rc = deal_pages(a, w, a.in.n, a.n_free, s);
  if (rc != L2KV_OK) return rc;
  if (dtype == L2KV_BF16) return g.D == 128 ? launch_pu<__nv_bfloat16, 128>(a, w, K, V, idx, sumsq, g, s) : launch_pu<__nv_bfloat16, 64>(a, w, K, V, idx, sumsq, g, s);
  return g.D == 128 ? launch_pu<float, 128>(a, w, K, V, idx, sumsq, g, s) : launch_pu<float, 64>(a, w, K, V, idx, sumsq, g, s);
}

template <typename T, int D>
static int launch_pc(const PageCompact& a, const PageScratch& w, const CompactSelect& c, void* K, void* V, int32_t* idx, float* sumsq,
                     const Geom& g, cudaStream_t s) {
  return launch_chained(page_compact_kernel<T, D>, (long long)w.entries * a.H * c.n_chunks + w.entries, 1, kPageThreads, 0, s, a, w, c,
                        static_cast<T*>(K), static_cast<T*>(V), idx, sumsq, g);
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
  constexpr int kWarps = kPageThreads / 32;
  rc = launch_chained(page_mark_select_kernel, units + (entries + kWarps - 1) / kWarps, 1, kPageThreads, 0, s, a, w, c);
  if (rc != L2KV_OK) return rc;
  rc = deal_pages(a, w, a.in.n, nullptr, s);
  if (rc != L2KV_OK) return rc;
  if (dtype == L2KV_BF16) return g.D == 128 ? launch_pc<__nv_bfloat16, 128>(a, w, c, K, V, idx, sumsq, g, s) : launch_pc<__nv_bfloat16, 64>(a, w, c, K, V, idx, sumsq, g, s);
  return g.D == 128 ? launch_pc<float, 128>(a, w, c, K, V, idx, sumsq, g, s) : launch_pc<float, 64>(a, w, c, K, V, idx, sumsq, g, s);
}

}  // namespace l2kv
