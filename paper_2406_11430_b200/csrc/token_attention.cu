// Prompt and tree attention over bf16 caches: packed new tokens, each sequence against its own cached
// rows, on the tensor cores (tcgen05.mma, operands by TMA in shared memory, accumulators in tensor
// memory).
//
// A query tile is 128 rows: the (token, head-of-the-group) pairs of 128 / G tokens that share a KV
// head.  Cached rows are taken in sub-blocks of 64; for each one
//   S = Q K^T  (128 x 64, fp32, tensor memory)  ->  softmax threads: masks, running maximum,
//   P = 2^(s - m) as bf16 over the score columns  ->  O += P V  (tensor memory).
// A CTA always works on two such chains at a time, so that one's matrix products run under the other's
// softmax: two neighbouring query tiles that share every K and V tile ("pair"), or, where a sequence
// has no more tokens than one tile holds, the even and the odd sub-blocks of one query tile ("alternate"),
// joined at the end.  Each chain has two score tiles, so S(j + 1) is formed while S(j) is worked on.
//
// Roles: 4 softmax warps per chain (one thread per query row), a warp per chain that issues its matrix
// products, one that works out the items and fetches tiles through a ring each for K and V.  A fixed grid of
// CTAs takes equal shares of the call's work, a list of items (tile or pair of one sequence, layer and KV
// head); an item that a share's end cuts leaves partial results that a second kernel joins.
// Every wait is bounded; one that gives up ends the CTA and marks the workspace.
//
// Rounded to fewer bits than 32 are two things.  The weights, to bf16: the tensor core takes them as the other
// operand is, and a second product with what the rounding leaves out would add 512 of its cycles to the 1312 below (D =
// 128); sums are of the weights before rounding.  The result, to bf16: the type in which the projection behind it reads
// its input.  Against 64 bits the relative error is 0.0018 to 0.0023, and 0.0016 with the result's rounding alone.
//
// What bounds it (cycle counters and probes; per sub-block, both chains): the exponentials need 1024 cycles of
// the MUFU pipe, the products 1312 of the tensor core (Q K^T at N = 64 50 cycles per instruction, bound by
// its operands' way out of shared memory; P V 64), and a sub-block takes about 1650: the exponentials of one
// chain take 660 with the pipe to themselves, and the chains hand them to each other in turn.  Long prompts
// run into the GPU's power limit besides: 16 k tokens, 32 heads of 128, take 1.75 ms at 1965 MHz and
// 1.97 ms (1117 TFLOP/s) at the 1570 MHz that are left after a while; ragged prompts to 2048 0.31 ms (850 TFLOP/s).
// Tree batches that fit one tile are bound by memory (88 us for 478 MB, 74 at the copy rate).
// Tried, correct and not faster: blocks of 128 rows with one score tile per chain (products at N = 128, 10 to
// 20 % slower: the chain softmax - product - softmax has no slack), two softmax warps for the same 32 rows,
// a share of the exponentials as a polynomial on the FMA pipe (any share from 1/8 to 1/2), no maxima after the
// first sub-block.
#include <algorithm>
#include <climits>
#include <cstring>

#include "tokens.cuh"
#include "umma.cuh"

namespace l2kv {

constexpr int kTaRows = 128;                    // query rows per tile, cached rows per block
constexpr int kTaSub = 64;                      // cached rows per sub-block: one K tile, one V tile
constexpr int kTaHalf = kTaRows * 128;          // query rows, [128][64 bf16], swizzled: 16 KB
constexpr int kTaSubHalf = kTaSub * 128;        // cached rows, [64][64 bf16]: 8 KB
constexpr int kTaStage = 2048;                  // bytes per softmax warp on the way out
constexpr int kTaThreads = 352;                 // 2 x 4 softmax warps, issuing warps 8 and 10, fetching warp 9
constexpr int kTaGrid = 148;                    // one CTA per SM (512 tensor-memory columns each)
constexpr int kTaCtrl = 1024 + 2 * kTaRows * 8;  // barriers and items; row statistics
constexpr int kTaPolls = 18;                    // log2 of the polls a wait may take
constexpr int kTaItemCost = 4;                  // what starting and finishing an item costs, in sub-blocks
constexpr int kTaMinShare = 12;                 // no shorter shares where items are cut, in sub-blocks
constexpr int kTaJoinCost = 12;                 // what cutting items costs a call, in sub-blocks
constexpr int kTaWholeLen = 1216;               // caches up to this length are never cut
constexpr int kTaGroup = 4;                     // pairs of weights whose exponentials go side by side
constexpr float kTaRescaleGap = 8.f;            // log2 units a maximum may drift before O is rescaled

template <int D> constexpr int kTaQTile = D / 64 * kTaHalf;
template <int D> constexpr int kTaTile = D / 64 * kTaSubHalf;
template <int D> constexpr int kTaSlots = 512 / D;    // K tiles, and V tiles, in flight: 64 KB each
template <int D> constexpr int kTaSmem = 2 * kTaQTile<D> + 2 * kTaSlots<D> * kTaTile<D> + 8 * kTaStage + kTaCtrl;
// as in the other kernels: fp32 accumulators, bf16 operands, N / 8 from bit 17, M / 16 from bit 24; V is
// N-major
constexpr uint32_t kTaIdescQK = (1u << 4) | (1u << 7) | (1u << 10) | ((64u >> 3) << 17) | ((128u >> 4) << 24);
template <int D> constexpr uint32_t kTaIdescPV =
    (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);

// One unit of a CTA's work.
struct TaItem {
  int b, l, h;
  int tok0, s0, nq;      // first token in the list and in its sequence, tokens of the item
  int base, end;         // row of the sequence's first new token; rows that some token of the item sees
  int row0, n, n0;       // first row, sub-blocks of the item (pair: of chain 1 and of chain 0)
  int pair;              // two query tiles; else one whose sub-blocks the chains take in turn
  int slot;              // where the partial result of a piece goes; -1: the result itself
  int stop;              // no more items
};

struct TaSpot;
struct TaArgs {
  TokenAttention a;
  int G, QT;             // query heads per KV head, tokens per tile
  TaSpot* plan;          // [kTaGrid] where each CTA's share begins, for the joining kernel; null: items stay whole
  float* part;           // [2 kTaGrid][slot_rows][D] rows, then [2 kTaGrid][slot_rows] log2-sum-exps
  float* part_lse;
  int slot_rows;
};

// ---- the items, worked out by a warp from the device's lengths ------------------------------------

struct TaEntry { int n, cur, base; };
__device__ __forceinline__ TaEntry ta_entry(const TokenAttention& a, int b, int l, int h) {
  const long long bl = (long long)b * a.g.L + l;
  const int n = tokens_of(a.tok_off, b, a.n_tokens).n;
  const int cur = max(0, min(a.lens.at(bl, h, a.g.H), min(a.max_len, a.g.cap(bl))));
  return {n, cur, cur - n};
}
// Rows that the first `upto` tokens of the sequence see at most, and their sub-blocks.
__device__ __forceinline__ int ta_end(const TokenAttention& a, const TaEntry& e, int upto) {
  return a.mask ? e.cur : max(0, min(e.cur, e.base + min(upto, e.n)));
}
__device__ __forceinline__ int ta_subs(int rows) { return (rows + kTaSub - 1) / kTaSub; }
// An entry as the shares see it: with a length per head, the longest head's.
__device__ __forceinline__ TaEntry ta_plan_entry(const TokenAttention& a, int e) {
  const int b = e / a.g.L, l = e % a.g.L;
  TaEntry x = ta_entry(a, b, l, 0);
  if (a.lens.per_head && x.n > 0) {
    for (int h = 1; h < a.g.H; ++h) x.cur = max(x.cur, ta_entry(a, b, l, h).cur);
    x.base = x.cur - x.n;
  }
  return x;
}
// Cost of the first m items (pairs of tiles, one head) of an entry: their sub-blocks, and kTaItemCost for each.
__device__ __forceinline__ long long ta_cost(const TokenAttention& a, const TaEntry& e, int QP, int m) {
  const int pairs = (e.n + QP - 1) / QP;
  if (m <= 0) return 0;
  if (a.mask) return (long long)m * (ta_subs(e.cur) + kTaItemCost);
  long long sum = (long long)m * kTaItemCost;
  if (m >= pairs) { sum += ta_subs(e.cur); m = pairs - 1; }                  // the last one ends where the cache does
  // the others see base + k QP rows, k = 1 .. m
  if (e.base < 0) {
    for (int k = 1; k <= m; ++k) sum += ta_subs(max(0, e.base + k * QP));
  } else if (QP % kTaSub == 0) {
    sum += (long long)m * ta_subs(e.base) + (long long)(QP / kTaSub) * m * (m + 1) / 2;
  } else {                                               // QP is half a sub-block: odd and even k
    const long long even = m / 2, odd = (m + 1) / 2;
    sum += even * ta_subs(e.base) + even * (even + 1) / 2 + odd * ta_subs(e.base + QP) + odd * (odd - 1) / 2;
  }
  return sum;
}

// A place in the list of all items, (b, l) by (b, l), within it tile pair by tile pair, within that head by
// head: an item, the cost of everything before it, and a number of its sub-blocks.
struct TaSpot {
  long long at;
  int e, p, h, off;
};

// The shares of the CTAs: stretches of the list that cost the same.  Where a share ends inside an item the item
// is cut, unless there is no room for partial results or cutting would not pay: then the share ends with the
// item.  One warp; the first 32 entries stay in registers.
struct TaShares {
  const TaArgs& A;
  TaEntry mine;                // entry number `lane`
  int entries, QP;
  long long share;
  bool cut, one_each;          // one_each: no more items than CTAs, one to each
  __device__ __forceinline__ TaEntry entry(int e0) const {
    const int e = e0 + (threadIdx.x & 31);
    if (e0 == 0) return mine;
    return e < entries ? ta_plan_entry(A.a, e) : TaEntry{0, 0, 0};
  }
  // Cost of the first m items of an entry and one head.
  __device__ __forceinline__ long long cost(const TaEntry& e, int m) const { return one_each ? m : ta_cost(A.a, e, QP, m); }
  __device__ __forceinline__ long long cost_of(const TaEntry& e) const {
    return e.n > 0 ? cost(e, (e.n + QP - 1) / QP) * A.a.g.H : 0;
  }
  __device__ __forceinline__ explicit TaShares(const TaArgs& args) : A(args) {
    const int lane = threadIdx.x & 31;
    QP = 2 * A.QT;
    entries = A.a.g.B * A.a.g.L;
    mine = lane < entries ? ta_plan_entry(A.a, lane) : TaEntry{0, 0, 0};
    one_each = false;
    long long sum = 0;
    int items = 0, longest = 0;
    for (int e0 = 0; e0 < entries; e0 += 32) {
      const TaEntry e = entry(e0);
      sum += cost_of(e);
      items += (e.n + QP - 1) / QP;
      if (e.n > 0) longest = max(longest, ta_subs(e.cur) + kTaItemCost);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    items = (int)__reduce_add_sync(0xffffffffu, (unsigned)items) * A.a.g.H;
    longest = (int)__reduce_max_sync(0xffffffffu, (unsigned)longest);
    const int grid = (int)gridDim.x;
    const long long fair = (sum + grid - 1) / grid;
    share = fair;
    cut = false;
    if (A.plan) {
      // With an item each at most, the longest one decides, or, where that is more, memory: with all SMs at it a
      // sub-block takes 0.77 us instead of 0.57.  Cut, it is the share or memory, and the partial rows and their
      // joining.  (8 heads of trees of 12 to 24 tokens, whole / cut in us: 1 tree behind 1.1k rows 16.4 / 19.7,
      // 3k 34 / 21, 16k 136 / 35; 16 trees behind 3k 42 / 48, 16k 175 / 177; 12 trees behind 3k 39 / 41, 16k
      // 147 / 136.)  With more items shares end up to half an item late, or, at equal lengths, after a number of
      // items.  (24 trees behind 1.1k 40 / 36, 16k 319 / 258; a prompt of 2k tokens 65 / 52; 32 pieces of 128 tokens
      // behind 2k 159 / 160.)
      const long long memory = fair * 27 / 20, least = max((long long)kTaMinShare, fair);
      cut = items <= grid ? max((long long)longest, memory) > max(least, memory) + kTaJoinCost
                          : max(longest / 2ll, (items + grid - 1) / grid * (sum / items) - fair) > kTaJoinCost * 3 / 4;
      if (cut) share = least;
    }
    if (!cut && items <= grid) { one_each = true; share = 1; }
  }
  // The next item of the list.
  __device__ __forceinline__ void next(TaSpot& s, long long cost, int n_tokens) const {
    s.at += cost;
    s.off = 0;
    if (++s.h == A.a.g.H) { s.h = 0; ++s.p; }
    if (s.p * QP >= n_tokens) {
      s.p = 0;
      do ++s.e; while (s.e < entries && tokens_of(A.a.tok_off, s.e / A.a.g.L, A.a.n_tokens).n == 0);
    }
  }
  // Where the share of CTA c begins (c = the number of CTAs: behind everything).  A spot close to an item's
  // start or end is moved there, so that no sliver is cut off.
  __device__ __forceinline__ TaSpot begin(int c) const {
    const int lane = threadIdx.x & 31, H = A.a.g.H;
    const long long x = c * share;
    long long before = 0;
    for (int e0 = 0; e0 < entries; e0 += 32) {
      const TaEntry y = entry(e0);
      const long long here = cost_of(y);
      long long incl = here;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += o;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, x < before + incl);
      if (hit) {
        const int who = __ffs(hit) - 1;
        const long long start = before + __shfl_sync(0xffffffffu, incl - here, who), rest = x - start;
        const TaEntry z{__shfl_sync(0xffffffffu, y.n, who), __shfl_sync(0xffffffffu, y.cur, who),
                        __shfl_sync(0xffffffffu, y.base, who)};
        // the last tile pair that begins at or before `rest`: the lanes try 32 of them at a time
        int lo = 0, step = (z.n + QP - 1) / QP;          // in [lo, lo + step)
        while (step > 1) {
          step = (step + 31) / 32;
          const unsigned m = __ballot_sync(0xffffffffu, cost(z, lo + lane * step) * H <= rest);
          lo += step * (31 - __clz(m));                  // (costs grow with p; behind the last they stay above rest)
        }
        const long long first = cost(z, lo);
        const int each = (int)(cost(z, lo + 1) - first), inside = (int)(rest - first * H);
        const int n = each - kTaItemCost, near = cut ? 4 + (int)min(share / 64, 64ll) : (n + 1) / 2 + 1;
        TaSpot s{start + first * H + (long long)(inside / each) * each, e0 + who, lo, inside / each, 0};
        if (one_each) return s;
        s.off = max(0, inside % each - kTaItemCost);
        if (s.off < near) s.off = 0;
        else if (n - s.off < near) next(s, each, z.n);
        return s;
      }
      before += __shfl_sync(0xffffffffu, incl, 31);
    }
    return {before, entries, 0, 0, 0};
  }
};

// The smallest calls, where this is a good part of the time: no more items than CTAs, none of them to be cut, no
// more than 32 entries.  CTA c takes item c.  (5 k cycles by the general way, about 1 k by this one.)
__device__ __forceinline__ bool ta_small_call(const TaArgs& A, TaSpot& spot, TaSpot& end) {
  const TokenAttention& a = A.a;
  const int lane = threadIdx.x & 31, entries = a.g.B * a.g.L, QP = 2 * A.QT, H = a.g.H;
  if (A.plan || entries > 32) return false;
  const int pairs = lane < entries ? (tokens_of(a.tok_off, lane / a.g.L, a.n_tokens).n + QP - 1) / QP : 0;
  int incl = pairs;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, incl, off);
    if (lane >= off) incl += o;
  }
  const int total = __shfl_sync(0xffffffffu, incl, 31);
  if (total > (int)gridDim.x / H) return false;
  const int c = (int)blockIdx.x / H, e = __popc(__ballot_sync(0xffffffffu, incl <= c));   // the entry that holds pair c
  const int before = __shfl_sync(0xffffffffu, incl - pairs, e & 31);
  spot = TaSpot{(long long)blockIdx.x, e, c - before, (int)blockIdx.x % H, 0};
  end = spot;
  if (c < total) ++end.at;
  return true;
}

// Sub-blocks [from, to) of the item of (b, l), tile pair p, head h.
__device__ __forceinline__ TaItem ta_item(const TaArgs& A, int b, int l, int p, int h, int from, int to, int slot) {
  const TokenAttention& a = A.a;
  const int QP = 2 * A.QT;
  const TaEntry e = ta_entry(a, b, l, h);
  TaItem it;
  it.b = b; it.l = l; it.h = h;
  it.s0 = p * QP;
  it.tok0 = tokens_of(a.tok_off, b, a.n_tokens).first + it.s0;
  it.nq = min(QP, e.n - it.s0);
  it.base = e.base;
  it.end = ta_end(a, e, it.s0 + QP);
  it.pair = it.nq > A.QT;
  it.row0 = from * kTaSub;
  it.n = max(0, min(to, ta_subs(it.end)) - from);
  it.n0 = max(0, min(to, ta_subs(ta_end(a, e, it.s0 + A.QT))) - from);       // what the first tile's tokens see
  it.slot = slot;
  it.stop = 0;
  return it;
}

// K and V tiles come through a ring each.  Sub-block g of an item takes place pos + g of both; an alternate item
// takes an even number of places (of an odd number of sub-blocks the last stays empty).  A wait on a barrier
// tells a phase from its neighbours only, so whoever waits for a tile has to know that the tile before it in the same
// slot has landed.  So it is: within an item that one is a tile the same chain has waited for (an alternate
// item deals the slots to the chains by turns, and their number is even), and an item begins when all tiles of
// those before it have landed (a pair's chains wait for all of them, those of an alternate item for each
// other at its end).
__device__ __forceinline__ int ta_places(int n, bool pair) { return pair ? n : (n + 1) & ~1; }

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1,
                                            int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
               "[%0], [%1, {%3, %4, %5, %6}], [%2];"
               :: "r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
               : "memory");
}
// The lowest x bits.
__device__ __forceinline__ uint32_t low_bits(int x) { return x >= 32 ? 0xffffffffu : x <= 0 ? 0u : (1u << x) - 1u; }

// The way out: columns of this warp's 32 rows, one row per lane, through 2 KB of shared memory, so that a store
// instruction fills whole sectors of eight rows (a thread that stored its own row would put 16 bytes into each
// of 32 different lines).  64 bytes of each row at a time: lane i holds piece i & 3 of the rows 8 k + (i >> 2), whose
// addresses it asks their owners for once.
struct TaRows {
  char* to[4];                                           // null: no such row
  __device__ __forceinline__ explicit TaRows(void* own) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      char* const row = reinterpret_cast<char*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(own), 8 * k + (lane >> 2)));
      to[k] = row ? row + (lane & 3) * 16 : row;
    }
  }
  // pieces[i]: bytes [16 i, 16 i + 16) of the lane's own 64
  __device__ __forceinline__ void store(const uint4 (&pieces)[4], int byte, uint4* stage) const {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) stage[lane * 4 + (i ^ (lane >> 1 & 3))] = pieces[i];
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = 8 * k + (lane >> 2);
      const uint4 x = stage[r * 4 + ((lane & 3) ^ (r >> 1 & 3))];
      if (to[k]) *reinterpret_cast<uint4*>(to[k] + byte) = x;
    }
  }
};

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{ .reg .b64 x, y, z, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; "
      "fma.rn.f32x2 w, x, y, z; mov.b64 {%0, %1}, w; }"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{ .reg .b64 x, y, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 w, x, y; mov.b64 {%0, %1}, w; }"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
template <int D, bool TREE>
__global__ void __launch_bounds__(kTaThreads, 1)
token_attention_kernel(const __grid_constant__ TaArgs A, const __grid_constant__ CUtensorMap map_q,
                       const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  constexpr int QTILE = kTaQTile<D>, TILE = kTaTile<D>, SLOTS = kTaSlots<D>;
  extern __shared__ __align__(1024) unsigned char smem[];
  const TokenAttention& a = A.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t base = smem_u32(smem);
  const uint32_t s_q = base, s_k = base + 2 * QTILE, s_v = s_k + SLOTS * TILE;
  unsigned char* const stage_base = smem + 2 * QTILE + 2 * SLOTS * TILE;
  unsigned char* const ctrl = stage_base + 8 * kTaStage;
  const uint32_t bars = smem_u32(ctrl);
  TaItem* const items = reinterpret_cast<TaItem*>(ctrl + 512);            // [2]
  TaSpot* const s_end = reinterpret_cast<TaSpot*>(ctrl + 640);
  volatile int* const s_fail = reinterpret_cast<volatile int*>(ctrl + 768);
  uint32_t* const s_tmem = reinterpret_cast<uint32_t*>(ctrl + 772);
  volatile int* const s_marked = reinterpret_cast<volatile int*>(ctrl + 776);
  volatile int* const s_turn = reinterpret_cast<volatile int*>(ctrl + 896);   // [2][4]: exponentials done, by chain and lane quarter
  float2* const s_stat = reinterpret_cast<float2*>(ctrl + 1024);          // [2][128]: maximum, sum
  auto k_full = [&](uint32_t at) { return bars + 8u * (at % SLOTS); };
  auto v_full = [&](uint32_t at) { return bars + 64u + 8u * (at % SLOTS); };
  auto k_empty = [&](uint32_t at) { return bars + 128u + 8u * (at % SLOTS); };
  auto v_empty = [&](uint32_t at) { return bars + 192u + 8u * (at % SLOTS); };
  const uint32_t more = bars + 256u;
  const uint32_t q_full = more, q_free = more + 8u, sync256 = more + 16u;
  auto item_full = [&](uint32_t i) { return more + 24u + 8u * (i & 1u); };
  auto item_free = [&](uint32_t i) { return more + 40u + 8u * (i & 1u); };
  auto s_full = [&](int c, uint32_t i) { return more + 56u + 16u * (uint32_t)c + 8u * (i & 1u); };
  auto p_full = [&](int c, uint32_t i) { return more + 88u + 16u * (uint32_t)c + 8u * (i & 1u); };
  // Complete once per P V, by the parity of its running number: a wait tells a phase from its two neighbours
  // only, and the one rescaling waits for can be two products behind.
  auto pv_done = [&](int c, uint32_t i) { return more + 120u + 16u * (uint32_t)c + 8u * (i & 1u); };
  auto o_full = [&](int c) { return more + 152u + 8u * (uint32_t)c; };
  const uint32_t issued = more + 184u;
  auto drained = [&](int c) { return more + 168u + 8u * (uint32_t)c; };

  if (tid == 0) {
    // a tile and the query rows are given back once per chain
    for (int i = 0; i < SLOTS; ++i) {
      mbar_init(k_full(i), 1); mbar_init(v_full(i), 1);
      mbar_init(k_empty(i), 2); mbar_init(v_empty(i), 2);
    }
    mbar_init(q_full, 1); mbar_init(q_free, 2); mbar_init(sync256, 8); mbar_init(issued, 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(item_full(i), 1); mbar_init(item_free(i), 10);
      mbar_init(s_full(0, i), 1); mbar_init(s_full(1, i), 1);
      mbar_init(p_full(0, i), 4); mbar_init(p_full(1, i), 4);
      mbar_init(pv_done(0, i), 1); mbar_init(pv_done(1, i), 1);
      mbar_init(o_full(i), 1); mbar_init(drained(i), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    *s_fail = 0;
    for (int i = 0; i < 8; ++i) s_turn[i] = 0;
  }
  __syncwarp();
  if (warp == 9 && lane < 3) {
    const CUtensorMap* const map = lane == 0 ? &map_q : lane == 1 ? &map_k : &map_v;
    asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
  }
  __syncwarp();
  wait_for_previous();
  // (tensor memory is taken behind the kernel before, which may need it, and before the next one may start)
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 :: "r"(smem_u32(s_tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // A wait that gave up in an earlier call marks the workspace; nothing runs until it is cleared.
  if (tid == 32) *s_marked = a.status ? *reinterpret_cast<volatile int32_t*>(a.status + 2) : 0;
  // (while the others set up) where this CTA's share of the work begins (warp 9) and ends (warp 10)
  TaSpot spot{0, 0, 0, 0, 0};
  bool one_each = false;
  if (warp == 9 || warp == 10) {
    TaSpot end;
    one_each = ta_small_call(A, spot, end);
    if (!one_each) {
      const TaShares shares(A);
      spot = end = shares.begin((int)blockIdx.x + (warp == 10));
      one_each = shares.one_each;
    }
    if (lane == 0) {
      if (warp == 10) *s_end = end;
      else if (A.plan) A.plan[blockIdx.x] = spot;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *s_tmem;
  auto free_tmem = [&]() {
    if (warp == 0)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(512) : "memory");
  };
  next_may_start();
  if (*s_marked) { free_tmem(); return; }
  // A wait that another role's failure ends too.
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (mbar_test(bar, parity)) return true;
    return *s_fail == 0 && mbar_wait<kTaPolls>(bar, parity);
  };
  auto k_landed = [&](uint32_t at) { return wait(k_full(at), (at / SLOTS) & 1u); };
  auto v_landed = [&](uint32_t at) { return wait(v_full(at), (at / SLOTS) & 1u); };
  uint32_t pos = 0;                                      // the rings' place of the item's first tiles
  // The tiles of an item, K `ahead` of V (one thread): the order in which they can be used, so that none waits
  // for a place behind one that is not needed yet.
  auto fetch = [&](const TaItem& it) {
    const int row0 = (int)a.g.row0((long long)it.b * a.g.L + it.l) + it.row0;
    const int tm_l = a.g.row_off ? 0 : it.l, tm_b = a.g.row_off ? 0 : it.b;
    const int places = ta_places(it.n, it.pair), ahead = it.pair ? 2 : 4;
    bool ok = true;
    auto one = [&](bool is_k, int g) {
      const uint32_t at = pos + g, full = is_k ? k_full(at) : v_full(at), empty = is_k ? k_empty(at) : v_empty(at);
      if (at >= SLOTS) ok = wait(empty, (at / SLOTS - 1) & 1u);
      if (!ok) return;
      if (!it.pair) mbar_arrive(empty);                  // for the chain that does not use it
      if (g >= it.n) {                                   // an empty place: landed and given back at once
        mbar_arrive(full);
        mbar_arrive(empty);
        return;
      }
      mbar_expect_tx(full, TILE);
      for (int c = 0; c < D / 64; ++c)
        tma_load_5d((is_k ? s_k : s_v) + (at % SLOTS) * TILE + c * kTaSubHalf, is_k ? &map_k : &map_v, full, c * 64,
                    row0 + g * kTaSub, it.h, tm_l, tm_b);
    };
    for (int g = 0; ok && g < places + ahead; ++g) {
      if (g < places) one(true, g);
      if (ok && g >= ahead) one(false, g - ahead);
    }
    return ok;
  };
  // After a failure: copies that may still be in flight, the last ones of every slot.
  auto drain = [&]() {
    for (int i = 0; i < SLOTS; ++i)
      for (uint32_t parity = 0; parity < 2; ++parity) {
        mbar_wait<12>(k_full(i), parity);
        mbar_wait<12>(v_full(i), parity);
      }
  };

  if (warp == 9) {
    // ---- items and tiles ---------------------------------------------------------------------------
    const int QP = 2 * A.QT, L = a.g.L;
    const TaSpot end = *s_end;
    bool ok = true;
    uint32_t n_pub = 0, n_q = 0;
    while (ok) {
      TaItem it;
      it.stop = 1;
      it.n = 0;
      if (spot.at < end.at || (spot.at == end.at && spot.off < end.off)) {
        const TaEntry e = ta_plan_entry(a, spot.e);
        const int n = ta_subs(ta_end(a, e, (spot.p + 1) * QP));
        const int to = spot.at == end.at ? end.off : n;
        // a piece that does not begin its item goes to this CTA's first slot, one that does to its second
        const int slot = spot.off > 0 ? 2 * (int)blockIdx.x : to < n ? 2 * (int)blockIdx.x + 1 : -1;
        it = ta_item(A, spot.e / L, spot.e % L, spot.p, spot.h, spot.off, to, slot);
        spot.at += one_each ? 1 : n + kTaItemCost;
        spot.off = 0;
        if (++spot.h == a.g.H) { spot.h = 0; ++spot.p; }
        if (spot.p * QP >= e.n) {
          spot.p = 0;
          do ++spot.e; while (spot.e < a.g.B * L && tokens_of(a.tok_off, spot.e / L, a.n_tokens).n == 0);
        }
      }
      if (n_pub >= 2) ok = wait(item_free(n_pub), (n_pub / 2 - 1) & 1u);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      if (lane == 0) {
        items[n_pub & 1] = it;
        mbar_arrive(item_full(n_pub));
      }
      ++n_pub;
      if (it.stop) break;
      if (it.n == 0) continue;
      if (lane == 0) {
        // (the copies themselves stay inside)
        (void)L2KV_BOUNDS(a.g.holds((long long)it.b * L + it.l, it.row0) && a.g.holds((long long)it.b * L + it.l, it.end - 1), a.status);
        const int tiles = it.pair ? 2 : 1;
        if (n_q > 0) ok = wait(q_free, (n_q - 1) & 1u);
        if (ok) {
          mbar_expect_tx(q_full, tiles * QTILE);
          for (int t = 0; t < tiles; ++t)
            for (int c = 0; c < D / 64; ++c)
              tma_load_4d(s_q + t * QTILE + c * kTaHalf, &map_q, q_full, c * 64, it.h * A.G, it.tok0 + t * A.QT, it.l);
        }
        ok = ok && fetch(it);
      }
      ok = __shfl_sync(0xffffffffu, ok, 0);
      pos += ta_places(it.n, it.pair);
      ++n_q;
    }
    if (!ok) {
      *s_fail = 1;
      if (lane == 0) {
        drain();
        mbar_wait<12>(q_full, 0); mbar_wait<12>(q_full, 1);
      }
    }
  } else if (warp == 8 || warp == 10) {
    // ---- matrix products of one chain: the whole warp walks the items, one elected lane issues --------
    const int c = warp == 10;
    bool ok = true;
    uint32_t n_item = 0, n_q = 0, n_s = 0, n_p = 0, n_alt = 0;   // running numbers: items, scores issued, weights used, ...
    const uint32_t t_c = __shfl_sync(0xffffffffu, tmem, 0) + c * 256;
    auto commit = [&](uint32_t bar) { if (elect_one()) umma_commit(bar); };
    while (true) {
      ok = __all_sync(0xffffffffu, wait(item_full(n_item), (n_item / 2) & 1u));
      if (!ok) break;
      const bool stop = __shfl_sync(0xffffffffu, items[n_item & 1].stop, 0);
      const bool pair = __shfl_sync(0xffffffffu, items[n_item & 1].pair, 0);
      const int n = __shfl_sync(0xffffffffu, items[n_item & 1].n, 0);
      const int n0 = __shfl_sync(0xffffffffu, items[n_item & 1].n0, 0);
      __syncwarp();
      if (lane == 0) mbar_arrive(item_free(n_item));
      ++n_item;
      if (stop) break;
      if (n == 0) continue;
      const int mine = pair ? (c ? n : n0) : (n + 1 - c) / 2;
      auto place = [&](int u) { return pos + (pair ? u : 2 * u + c); };
      const uint64_t dq = umma_desc(s_q + (pair ? c * QTILE : 0), 16, 1024);
      auto qk = [&](uint32_t at) {                       // S[n_s & 1] = Q K^T; elected lane only
        const uint64_t dk = umma_desc(s_k + (at % SLOTS) * TILE, 16, 1024);
#pragma unroll
        for (int k = 0; k < D / 16; ++k)                 // (the address fields count 16 bytes)
          umma_ss(t_c + (n_s & 1) * 64, dq + (((k >> 2) * kTaHalf + (k & 3) * 32) >> 4),
                  dk + (((k >> 2) * kTaSubHalf + (k & 3) * 32) >> 4), kTaIdescQK, k > 0);
        umma_commit(s_full(c, n_s));
        umma_commit(k_empty(at));
      };
      ok = wait(q_full, n_q & 1u);
      ++n_q;
      for (int u = 0; u < min(2, mine); ++u, ++n_s) {
        const uint32_t at = place(u);
        ok = k_landed(at) && ok;
        tc_fence_after();
        if (elect_one()) qk(at);
      }
      if (mine <= 2) commit(q_free);
      for (int u = 0; u < mine; ++u, ++n_p) {
        // Everything that will be there anyway is checked before the weights are waited for: a check costs
        // about 100 cycles, and the softmax waits for what is issued behind the weights.
        const uint32_t v = place(u), kn = place(u + 2);
        const bool next = u + 2 < mine;
        ok = v_landed(v) && ok;
        if (next) ok = k_landed(kn) && ok;
        ok = wait(p_full(c, n_p), (n_p >> 1) & 1u) && ok;
        if (!__all_sync(0xffffffffu, ok)) break;
        tc_fence_after();
        const uint64_t dv = umma_desc(s_v + (v % SLOTS) * TILE, kTaSubHalf, 1024);
        if (elect_one()) {                               // O += P V(u)
#pragma unroll
          for (int k = 0; k < kTaSub / 16; ++k)
            umma_ts(t_c + 128, t_c + (n_p & 1) * 64 + k * 8, dv + (k * 2048 >> 4), kTaIdescPV<D>, u > 0 || k > 0);
          umma_commit(v_empty(v));
          // The score columns that P V(u) reads its weights from take scores u + 2: both products come
          // from one thread and run on one tensor core, which takes them in the order of issue.
          if (next) qk(kn);
          umma_commit(pv_done(c, n_p));
          if (u + 1 == mine) umma_commit(o_full(c));
          if (u + 3 == mine) umma_commit(q_free);
        }
        if (next) ++n_s;
      }
      // tiles behind the last that chain 0 of a pair has a use for
      if (pair && c == 0)
        for (int g = mine; ok && g < n; ++g) {
          ok = k_landed(pos + g) && v_landed(pos + g);
          if (lane == 0) { mbar_arrive(k_empty(pos + g)); mbar_arrive(v_empty(pos + g)); }
          __syncwarp();
        }
      if (!pair) {                                       // until all tiles of the item have landed
        __syncwarp();
        if (lane == 0) mbar_arrive(issued);
        ok = ok && wait(issued, n_alt & 1u);
        ++n_alt;
      }
      pos += ta_places(n, pair);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
    }
    if (!ok) {
      *s_fail = 1;
      commit(drained(c));                                // products in flight read this CTA's shared memory
      mbar_wait<14>(drained(c), 0);
    }
  } else if (warp < 8) {
    // ---- softmax: one thread per query row of its chain -----------------------------------------------
    const int chain = warp >> 2, row = tid & (kTaRows - 1);
    const uint32_t t_c = tmem + chain * 256 + ((uint32_t)((warp & 3) * 32) << 16), t_o = t_c + 128;
    const uint32_t t_o0 = tmem + 128 + ((uint32_t)((warp & 3) * 32) << 16), t_o1 = t_o0 + 256;
    uint4* const stage = reinterpret_cast<uint4*>(stage_base + warp * kTaStage);
    const int tok_in_tile = row / A.G, head_in_group = row % A.G;
    uint32_t n_item = 0, n_s = 0, n_o = 0, n_sync = 0;
    int other_s = 0;                                     // the other chain's n_s at the start of the item
    volatile int* const my_turn = s_turn + chain * 4 + (warp & 3);
    volatile int* const other_turn = s_turn + (1 - chain) * 4 + (warp & 3);
    bool ok = true;
    auto sync_chains = [&]() {                           // all eight softmax warps, bounded
      __syncwarp();
      if (lane == 0) mbar_arrive(sync256);
      ok = ok && wait(sync256, n_sync & 1u);
      ++n_sync;
      ok = __all_sync(0xffffffffu, ok);
      return ok;
    };
    while (true) {
      ok = __all_sync(0xffffffffu, wait(item_full(n_item), (n_item / 2) & 1u));
      if (!ok) break;
      const TaItem it = items[n_item & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(item_free(n_item));
      ++n_item;
      if (it.stop) break;
      const int q = (it.pair ? chain * A.QT : 0) + tok_in_tile;             // token within the item
      const bool valid = q < it.nq;
      const bool warp_valid = __any_sync(0xffffffffu, valid);
      // rows this token sees: all below `limit`, and, from row `base` on, those of its mask
      const int limit = !valid ? 0 : TREE ? it.end : min(it.end, it.base + it.s0 + q + 1);
      const uint32_t* mask = TREE ? a.mask + (long long)(it.tok0 + (valid ? q : 0)) * 2 * a.mask_words : nullptr;
      const int mine = it.pair ? (chain ? it.n : it.n0) : (it.n + 1 - chain) / 2;
      const int others = it.pair ? (chain ? it.n0 : it.n) : (it.n + chain) / 2;
      // rows below `clear` are seen by all rows of the warp
      const int clear = TREE ? it.base : (int)__reduce_min_sync(0xffffffffu, (unsigned)max(0, limit));
      float m_ref = -INFINITY, sum = 0.f;

      for (int u = 0; u < mine; ++u, ++n_s) {
        const int g = it.pair ? u : 2 * u + chain;                           // sub-block within the item
        const int r0 = it.row0 + g * kTaSub;                                 // its first row
        const uint32_t t_s = t_c + (n_s & 1) * 64;
        ok = wait(s_full(chain, n_s), (n_s >> 1) & 1u);  // (voted on below)
        tc_fence_after();
        // Rows of the V tile that no token of the item sees can hold anything; clear them, so that a zero
        // weight times Inf or NaN cannot reach O (in a pair both chains write the same zeros).
        if (it.end - r0 < kTaSub) {
          const uint32_t v = pos + g;
          ok = v_landed(v) && ok;
          if (row < kTaSub && row >= it.end - r0) {
#pragma unroll
            for (int c = 0; c < D / 8; ++c)
              st_shared16(s_v + (v % SLOTS) * TILE + (c >> 3) * kTaSubHalf + row * 128 + ((c & 7) << 4), 0, 0, 0, 0);
          }
          proxy_fence();
        }
        if (warp_valid) {
          uint32_t x[64];
          tmem_ld64(t_s, x);
          if (r0 + kTaSub > clear) {
            // the bits of a word of 32 columns that this thread's row sees
#pragma unroll
            for (int w = 0; w < 2; ++w) {
              uint32_t bits = low_bits(limit - r0 - 32 * w);
              if constexpr (TREE) {
                const int c = r0 + 32 * w - it.base;     // mask column of the word's first row
                if (c > -32 && bits) {
                  const int i = c >= 0 ? c >> 5 : 0, n_words = 2 * a.mask_words;
                  const uint32_t lo = c < 0 || i < n_words ? mask[i] : 0u;
                  bits &= c < 0 ? low_bits(-c) | lo << -c
                                : __funnelshift_r(lo, i + 1 < n_words ? mask[i + 1] : 0u, c & 31);
                }
              }
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(bits >> i & 1u)) x[32 * w + i] = 0xff800000u;          // -inf
            }
          }
          float t[4] = {__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2]), __uint_as_float(x[3])};
#pragma unroll
          for (int i = 4; i < 60; i += 8)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              t[e] = fmaxf(t[e], fmaxf(__uint_as_float(x[i + 2 * e]), __uint_as_float(x[i + 2 * e + 1])));
#pragma unroll
          for (int e = 0; e < 4; ++e) t[e] = fmaxf(t[e], __uint_as_float(x[60 + e]));
          const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
          const float m_new = fmaxf(m_ref, top * a.scale_log2e);
          if (u == 0) m_ref = m_new;
          const bool need = m_new > m_ref + kTaRescaleGap;
          if (__any_sync(0xffffffffu, need || !ok)) {
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            // O is quiet once P V(u - 1) is done (P V(u) waits for this warp)
            ok = __all_sync(0xffffffffu, wait(pv_done(chain, n_s - 1), ((n_s - 1) >> 1) & 1u));
            if (!ok) break;
            tc_fence_after();
            const float factor = need ? fast_exp2(m_ref - m_new) : 1.f;
#pragma unroll 1
            for (int c = 0; c < D; c += 8) tmem_scale8(t_o + c, factor);
            if (need) { sum *= factor; m_ref = m_new; }
          }
          const float neg_m = m_ref == -INFINITY ? 0.f : -m_ref;             // a row that has seen nothing yet
          const float2 sc2 = make_float2(a.scale_log2e, a.scale_log2e), nm2 = make_float2(neg_m, neg_m);
          float2 sums = make_float2(0.f, 0.f);
          // The two warps of a scheduler, one per chain, take turns in the exponentials: side by side both are
          // slowed to half speed and then wait for the tensor core together, in step for good (7 to 10 % slower
          // on long and on ragged prompts).  Only the pace depends on it: a turn that does not come is not waited for.
          if (chain ? u < others : u <= others) {
            const int until = other_s + u + chain;
            for (int spin = 0; spin < 128 && *other_turn - until < 0; ++spin) {}
          }
          // Four pairs at a time, one stage apart: the exponentials of one group beside the arguments of the next
          // and the sums and roundings of the one before.  (All arguments first, then all exponentials, then all sums: 4
          // to 10 % slower; groups of 2 or 8 pairs: 4 % slower, the same.)
          uint32_t pk[32];
          float2 arg[kTaGroup], w[kTaGroup], done[kTaGroup];
          auto args_of = [&](int g) {
#pragma unroll
            for (int i = 0; i < kTaGroup; ++i) {
              const int k = 2 * (kTaGroup * g + i);
              arg[i] = fma2(make_float2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), sc2, nm2);
            }
          };
          auto finish = [&](int g) {
#pragma unroll
            for (int i = 0; i < kTaGroup; ++i) {
              sums = add2(sums, done[i]);
              pk[kTaGroup * g + i] = pack_bf16(done[i].x, done[i].y);
            }
          };
          args_of(0);
#pragma unroll
          for (int g = 0; g < 32 / kTaGroup; ++g) {
            __syncwarp();                                // (a fence for the compiler's scheduling)
#pragma unroll
            for (int i = 0; i < kTaGroup; ++i) w[i] = make_float2(fast_exp2(arg[i].x), fast_exp2(arg[i].y));
            if (g + 1 < 32 / kTaGroup) args_of(g + 1);
            if (g > 0) finish(g - 1);
#pragma unroll
            for (int i = 0; i < kTaGroup; ++i) done[i] = w[i];
          }
          finish(32 / kTaGroup - 1);
          if (lane == 0)                                 // the turn; the store takes the last weights as an operand, so it comes behind them
            asm volatile("{ .reg .b32 t; mov.b32 t, %2; st.volatile.shared.b32 [%0], %1; }"
                         :: "r"(smem_u32(const_cast<int*>(my_turn))), "r"(n_s + 1), "r"(pk[31]) : "memory");
          tmem_st32(t_s, pk);
          tmem_wait_st();
          sum += sums.x + sums.y;
        } else {
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (lane == 0) *my_turn = (int)n_s + 1;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(chain, n_s));
      }
      if (!ok) break;
      pos += ta_places(it.n, it.pair);
      other_s += others;

      // ---- the item's rows go out --------------------------------------------------------------------
      if (mine > 0) {
        ok = __all_sync(0xffffffffu, wait(o_full(chain), n_o & 1u));
        ++n_o;
        if (!ok) break;
      }
      tc_fence_after();
      const int tok = it.tok0 + q, head = it.h * A.G + head_in_group;
      const long long part_row = (long long)it.slot * A.slot_rows + (it.pair ? chain * kTaRows : 0) + row;
      const bool writes = valid && L2KV_BOUNDS(tok >= 0 && tok < a.n_tokens && head < a.g.Hq && it.slot < 2 * (int)gridDim.x &&
                                                   (it.pair ? chain * kTaRows : 0) + row < (A.plan ? A.slot_rows : 2 * kTaRows), a.status);
      __nv_bfloat16* const out = writes ? a.out.row<__nv_bfloat16>(it.l, tok, head) : nullptr;
      float* const part = writes && it.slot >= 0 ? A.part + part_row * D : nullptr;
      float f0 = 1.f, f1 = 0.f, total = sum, m = m_ref;
      int c_lo = 0, c_hi = D;
      if (!it.pair) {
        // one query tile, two chains: each joins half of the columns of both
        s_stat[chain * kTaRows + row] = make_float2(m_ref, sum);
        tc_fence_before();                               // the other chain's warps have seen its O complete
        if (!sync_chains()) break;
        tc_fence_after();
        const float2 st0 = s_stat[row], st1 = s_stat[kTaRows + row];
        m = fmaxf(st0.x, st1.x);
        const float low = m == -INFINITY ? 0.f : m;
        f0 = fast_exp2(st0.x - low);
        f1 = it.n > 1 ? fast_exp2(st1.x - low) : 0.f;
        total = st0.y * f0 + st1.y * f1;
        c_lo = chain * 64;                               // (64-wide heads: chain 0 has them all)
        c_hi = min(c_lo + 64, D);
      }
      const bool any = it.pair ? mine > 0 : it.n > 0;
      const float inv = total == 0.f ? 0.f : 1.f / total;
      f0 *= inv;
      f1 *= inv;
      if (warp_valid) {
        const TaRows rows(it.slot >= 0 ? static_cast<void*>(part) : static_cast<void*>(out));
        // 32 columns at a time, in a loop that stays one: unrolled, the kernel spilled (a prompt of 2k tokens 66 us
        // instead of 56).  An item costs about 6000 cycles beyond its sub-blocks, 3600 of them here; exchanging pieces
        // by shuffles instead of shared memory, or two columns per instruction, changed nothing.
#pragma unroll 1
        for (int c = c_lo; c < c_hi; c += 32) {
          uint32_t x[32];
          float v[32];
          tmem_ld32((it.pair ? t_o : t_o0) + c, x);
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(x[i]) * f0;
          if (!it.pair && it.n > 1) {
            tmem_ld32(t_o1 + c, x);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __fmaf_rn(__uint_as_float(x[i]), f1, v[i]);
          }
          if (!any) {                                    // (tensor memory holds whatever it held)
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
          }
          uint4 pieces[4];
          if (it.slot >= 0) {
#pragma unroll
            for (int d = 0; d < 2; ++d) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                pieces[i] = make_uint4(__float_as_uint(v[16 * d + 4 * i]), __float_as_uint(v[16 * d + 4 * i + 1]),
                                       __float_as_uint(v[16 * d + 4 * i + 2]), __float_as_uint(v[16 * d + 4 * i + 3]));
              rows.store(pieces, c * 4 + 64 * d, stage);
            }
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              pieces[i] = make_uint4(pack_bf16(v[8 * i], v[8 * i + 1]), pack_bf16(v[8 * i + 2], v[8 * i + 3]),
                                     pack_bf16(v[8 * i + 4], v[8 * i + 5]), pack_bf16(v[8 * i + 6], v[8 * i + 7]));
            rows.store(pieces, c * 2, stage);
          }
        }
        if (writes && (it.pair || chain == 0)) {
          const float lse2 = total == 0.f ? -INFINITY : m + log2f(total);
          if (it.slot >= 0) A.part_lse[part_row] = lse2;
          else if (a.lse) a.lse[((long long)it.l * a.n_tokens + tok) * a.g.Hq + head] = lse2 * 0.6931471805599453f;
        }
      }
      tc_fence_before();
      // the next item's first products overwrite what both chains have just read
      if (!it.pair && !sync_chains()) break;
    }
    if (!ok) *s_fail = 1;
  }
  __syncthreads();
  tc_fence_after();
  if (*s_fail && tid == 0) record_timeout(a.status);
  tc_fence_before();
  __syncthreads();
  free_tmem();
}

// Joins the pieces of items that were cut: out = sum_c w_c O_c / sum_c w_c, w_c = 2^(lse_c - max lse), piece by
// piece in order.  A block per CTA share and 32 rows of the item that the share's start cuts, eight lanes per row,
// so that a warp's four rows are loaded together; an item that several starts cut is the first one's.  What it
// takes is the chain plan - sums - rows of loads.
constexpr int kTaJoinWarps = 8;
template <int D>
__global__ void __launch_bounds__(32 * kTaJoinWarps)
token_attention_join_kernel(const __grid_constant__ TaArgs A) {
  constexpr int V = D / 8;                               // columns per lane: four at a time, 32 apart
  const TokenAttention& a = A.a;
  next_may_start();
  wait_for_previous();
  if (a.status && a.status[2] != 0) return;              // a wait gave up: no output
  const int piece = threadIdx.x & 7, r = (int)blockIdx.y * 32 + ((int)threadIdx.x >> 3), c0 = (int)blockIdx.x + 1;
  const TaSpot s = A.plan[c0], before = A.plan[c0 - 1];
  if (s.off == 0 || (before.at == s.at && before.off > 0)) return;
  int c1 = c0 + 1;                                       // shares [c0, c1) begin inside the item
  while (c1 < kTaGrid && A.plan[c1].at == s.at && A.plan[c1].off > 0) ++c1;
  const int nc = c1 - c0 + 1;
  auto row = [&](int c) { return (long long)(c == 0 ? 2 * c0 - 1 : 2 * (c0 + c - 1)) * A.slot_rows + r; };
  if (!L2KV_BOUNDS(s.e >= 0 && s.e < a.g.B * a.g.L && s.h >= 0 && s.h < a.g.H && before.at <= s.at, a.status)) return;
  const TaItem it = ta_item(A, s.e / a.g.L, s.e % a.g.L, s.p, s.h, 0, INT_MAX, 0);
  if (r >= it.nq * A.G) return;
  if (!L2KV_BOUNDS(r < A.slot_rows && it.tok0 >= 0 && it.tok0 + it.nq <= a.n_tokens, a.status)) return;
  float top = -INFINITY;
#pragma unroll 4
  for (int c = 0; c < nc; ++c) top = fmaxf(top, A.part_lse[row(c)]);
  const float low = top == -INFINITY ? 0.f : top;
  float den = 0.f, num[V] = {};
#pragma unroll 2
  for (int c = 0; c < nc; ++c) {
    const float lse2 = A.part_lse[row(c)];
    const float w = lse2 == -INFINITY ? 0.f : exp2f(lse2 - low);
    const float4* const from = reinterpret_cast<const float4*>(A.part + row(c) * D) + piece;
    float4 x[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) x[i] = from[8 * i];
    den += w;
    if (w == 0.f) continue;                              // (rows of a piece that sees nothing are zeros)
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      num[4 * i] = fmaf(w, x[i].x, num[4 * i]);
      num[4 * i + 1] = fmaf(w, x[i].y, num[4 * i + 1]);
      num[4 * i + 2] = fmaf(w, x[i].z, num[4 * i + 2]);
      num[4 * i + 3] = fmaf(w, x[i].w, num[4 * i + 3]);
    }
  }
  const float inv = den == 0.f ? 0.f : 1.f / den;
  const int tok = it.tok0 + r / A.G, head = it.h * A.G + r % A.G;
  uint2* const to = reinterpret_cast<uint2*>(a.out.row<__nv_bfloat16>(it.l, tok, head)) + piece;
#pragma unroll
  for (int i = 0; i < V / 4; ++i)
    to[8 * i] = make_uint2(pack_bf16(num[4 * i] * inv, num[4 * i + 1] * inv),
                           pack_bf16(num[4 * i + 2] * inv, num[4 * i + 3] * inv));
  if (a.lse && piece == 0)
    a.lse[((long long)it.l * a.n_tokens + tok) * a.g.Hq + head] =
        den == 0.f ? -INFINITY : (top + log2f(den)) * 0.6931471805599453f;
}

// ---- host ------------------------------------------------------------------------------------------

// Room for the pieces of items that are cut; none where caches are too short for it to pay.
struct TaRoom {
  long long items;        // at most
  int slot_rows;          // 0: items are never cut
  size_t bytes;
};
constexpr size_t kTaPlanBytes = (kTaGrid * sizeof(TaSpot) + 255) / 256 * 256;
static TaRoom ta_room(const Geom& g, int n_tokens, int max_len) {
  const int G = g.Hq / g.H, QP = 2 * (kTaRows / G);
  TaRoom r{((long long)n_tokens / QP + std::min(g.B, n_tokens)) * g.L * g.H, 0, 0};
  if (max_len > kTaWholeLen) {
    r.slot_rows = (long long)n_tokens * G <= kTaRows ? kTaRows : 2 * kTaRows;
    r.bytes = kTaPlanBytes + (size_t)2 * kTaGrid * r.slot_rows * (g.D + 1) * sizeof(float);
  }
  return r;
}

size_t token_attention_scratch(const Geom& g, int dtype, int n_tokens, int max_len) {
  return dtype == L2KV_BF16 ? ta_room(g, n_tokens, max_len).bytes : 0;
}

// Rank-4 map of the queries (head_dim, head, token, layer); a box is one half row of a tile's rows.
static bool make_query_map(CUtensorMap* map, const TokenAttention& a) {
  const Geom& g = a.g;
  const int G = g.Hq / g.H;
  const long long tight = g.D;
  const cuuint64_t dims[4] = {(cuuint64_t)g.D, (cuuint64_t)g.Hq, (cuuint64_t)a.n_tokens, (cuuint64_t)g.L};
  const cuuint64_t strides[3] = {(cuuint64_t)(g.Hq > 1 ? a.q.sh : tight) * 2, (cuuint64_t)(a.n_tokens > 1 ? a.q.st : tight) * 2,
                                 (cuuint64_t)(g.L > 1 ? a.q.sl : tight) * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)G, (cuuint32_t)(kTaRows / G), 1};
  return encode_bf16_map(map, 4, a.q.p, dims, strides, box);
}

template <int D, bool TREE>
static int launch_ta(const TaArgs& A, const void* K, const void* V, long long items, cudaStream_t s) {
  const TokenAttention& a = A.a;
  alignas(64) CUtensorMap map_q, map_k, map_v;
  std::memset(&map_q, 0, sizeof map_q);
  std::memset(&map_k, 0, sizeof map_k);
  std::memset(&map_v, 0, sizeof map_v);
  if (!make_query_map(&map_q, a) || !make_cache_map(&map_k, K, a.g, kTaSub) || !make_cache_map(&map_v, V, a.g, kTaSub))
    return L2KV_ERR_UNSUPPORTED;
  auto kern = token_attention_kernel<D, TREE>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kTaSmem<D>) != cudaSuccess)
    return L2KV_ERR_CUDA;
  const unsigned grid = (unsigned)std::min<long long>(kTaGrid, A.plan ? kTaGrid : items);
  const int rc = launch_early(kern, dim3(grid), kTaThreads, kTaSmem<D>, s, A, map_q, map_k, map_v);
  if (rc != L2KV_OK || !A.plan) return rc;
  return launch_early(token_attention_join_kernel<D>, dim3(kTaGrid - 1, (unsigned)(A.slot_rows / 32)), 32 * kTaJoinWarps, 0,
                      s, A);
}

int launch_token_attention(const TokenAttention& a, const void* K, const void* V, int dtype, char* scratch,
                           size_t scratch_bytes, cudaStream_t s) {
  if (dtype != L2KV_BF16) return launch_token_attention_fp32(a, K, V, s);
  const TaRoom room = ta_room(a.g, a.n_tokens, a.max_len);
  if (room.items > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  TaArgs A{};
  A.a = a;
  A.G = a.g.Hq / a.g.H;
  A.QT = kTaRows / A.G;
  A.slot_rows = room.slot_rows;
  if (room.slot_rows > 0 && scratch && scratch_bytes >= room.bytes) {
    A.plan = reinterpret_cast<TaSpot*>(scratch);
    A.part = reinterpret_cast<float*>(scratch + kTaPlanBytes);
    A.part_lse = A.part + (size_t)2 * kTaGrid * room.slot_rows * a.g.D;
  }
  if (a.g.D == 128)
    return a.mask ? launch_ta<128, true>(A, K, V, room.items, s) : launch_ta<128, false>(A, K, V, room.items, s);
  return a.mask ? launch_ta<64, true>(A, K, V, room.items, s) : launch_ta<64, false>(A, K, V, room.items, s);
}

}  // namespace l2kv
