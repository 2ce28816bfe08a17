// Rows of new tokens in and around the cache: rotary positions with the cache write, and the move of a
// drafted tree's accepted path down to the end of the committed rows.  Both move each row once
// and compute next to nothing, so what bounds them is the memory traffic, or, for a handful of
// tokens, the chain of dependent loads before the first row can go out.
#include <climits>

#include "tokens.cuh"

namespace l2kv {

// ---- rotary positions and cache write ------------------------------------------------------------
// A token's rows (the heads of q, k and v of one layer) are one warp's, or, for calls with few tokens, shared by
// several warps.  A row belongs to LPR adjacent lanes, a 16-byte piece each, as everywhere in the
// library; a half-split pair's other element is in another lane of the row, an interleaved pair's in the
// same piece.  A lane meets the same piece of every row, so it keeps that piece's cosines and sines in
// registers.  Rows are read kRotaryBatch pieces per lane at a time, the first batch before
// anything is known of the token; angle, sequence and cache row are worked out under those loads.
constexpr int kRotaryThreads = 256;
constexpr int kRotaryWarps = kRotaryThreads / 32;
struct RotaryArgs {
  TokView q, k, v, q_out;
  Geom g;
  const int32_t* tok_off;
  const int32_t* pos;
  const double* freq;
  const int32_t* start;
  int32_t* cur_len;
  int32_t* idx;
  float* sumsq;
  int32_t* status;
  int n_tokens, rot_dim, interleaved, per_head;
  double scale;
};

template <typename T>
__device__ __forceinline__ uint4 pack_piece(const float (&y)[Elem<T>::kPerVec]);
template <>
__device__ __forceinline__ uint4 pack_piece<float>(const float (&y)[4]) {
  return make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
}
template <>
__device__ __forceinline__ uint4 pack_piece<__nv_bfloat16>(const float (&y)[8]) {
  auto two = [](float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
  };
  return make_uint4(two(y[0], y[1]), two(y[2], y[3]), two(y[4], y[5]), two(y[6], y[7]));
}

// A 16-byte load that leaves no line in L1.  (Not through the read-only path: q_out may be q.)
__device__ __forceinline__ uint4 ld_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

// Cosine and sine of the angle a in fp64, to about 1e-15: their fp32 roundings are those of the exact values
// but for one in some 10^7.  a / 2 pi is formed as a sum of two doubles and the nearest quarter turn taken off it,
// which leaves the rest exact for any position; at most an eighth of a turn is left, where the Taylor series
// are short (the first terms left out: x^17 / 17! < 4.7e-17, x^16 / 16! < 1.01e-15).
__device__ __forceinline__ void cos_sin(double a, double* c, double* s) {
  constexpr double kHi = 0.15915494309189535, kLo = -9.839338337591243e-18;   // 1 / 2 pi
  const double t = a * kHi;
  const double rest = __fma_rn(a, kLo, __fma_rn(a, kHi, -t));
  const double quarters = rint(4.0 * t);
  const double x = (__fma_rn(-0.25, quarters, t) + rest) * 6.283185307179586, z = x * x;
  double sx = __fma_rn(z, -1.0 / 1307674368000.0, 1.0 / 6227020800.0);
  double cx = __fma_rn(z, -1.0 / 87178291200.0, 1.0 / 479001600.0);
  sx = __fma_rn(z, sx, -1.0 / 39916800.0);
  cx = __fma_rn(z, cx, -1.0 / 3628800.0);
  sx = __fma_rn(z, sx, 1.0 / 362880.0);
  cx = __fma_rn(z, cx, 1.0 / 40320.0);
  sx = __fma_rn(z, sx, -1.0 / 5040.0);
  cx = __fma_rn(z, cx, -1.0 / 720.0);
  sx = __fma_rn(z, sx, 1.0 / 120.0);
  cx = __fma_rn(z, cx, 1.0 / 24.0);
  sx = __fma_rn(z, sx, -1.0 / 6.0);
  cx = __fma_rn(z, cx, -0.5);
  sx = __fma_rn(x * z, sx, x);
  cx = __fma_rn(z, cx, 1.0);
  const int q = (int)(long long)quarters;                // only its last two bits count
  const double u = q & 1 ? sx : cx, v = q & 1 ? cx : sx;
  *c = (q + 1) & 2 ? -u : u;
  *s = q & 2 ? -v : v;
}

// WPT: warps that share a token.  PAIRS: interleaved pairs.
template <typename T, int D, int WPT, bool PAIRS>
__global__ void __launch_bounds__(kRotaryThreads, 3)
rotary_write_kernel(const __grid_constant__ RotaryArgs a, T* K, T* V) {
  constexpr int EPV = Elem<T>::kPerVec, LPR = D / EPV, RPW = 32 / LPR;
  constexpr int U = WPT == 1 ? 8 : 4;                    // pieces per lane in flight
  constexpr int TPB = kRotaryWarps / WPT;                // tokens per block
  constexpr int STEP = WPT * RPW;                        // rows that a token's warps take at once
  __shared__ float2 s_turn[kRotaryWarps][D / 2];
  const Geom& g = a.g;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane % LPR;
  next_may_start();
  wait_for_previous();
  const unsigned n_rows = (unsigned)a.n_tokens * (unsigned)g.L, token_blocks = (n_rows + TPB - 1) / TPB;
  if (blockIdx.x >= token_blocks) {
    // trailing blocks: the new lengths (sequences without new tokens have one too)
    const long long u = (long long)(blockIdx.x - token_blocks) * kRotaryThreads + threadIdx.x;
    const long long units = (long long)g.B * g.L * (a.per_head ? g.H : 1);
    if (u >= units) return;
    const long long bl = a.per_head ? u / g.H : u;
    const int n = tokens_of(a.tok_off, (int)(bl / g.L), a.n_tokens).n;
    a.cur_len[u] = (int)min((long long)g.cap(bl), (long long)max(0, a.start[u]) + n);
    return;
  }
  const unsigned il = blockIdx.x * TPB + warp / WPT;     // token * layers + layer
  if (il >= n_rows) return;
  const int i = (int)(il / (unsigned)g.L), l = (int)(il % (unsigned)g.L);
  const int group = (warp % WPT) * RPW, row0 = group + lane / LPR;           // this lane's first row of each kind

  // Rows of one kind, U at a time: `from` the lane's piece of row 0, rows `stride` bytes apart.
  auto load = [&](uint4 (&x)[U], const char* from, long long stride, int r0, int n) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      x[u] = r0 + u * STEP < n ? ld_once(from + (r0 + u * STEP) * stride) : make_uint4(0, 0, 0, 0);
  };
  const char* const q_from = reinterpret_cast<const char*>(a.q.row<T>(l, i, 0)) + piece * 16;
  const long long q_stride = a.q.sh * (long long)sizeof(T);
  uint4 x[U];
  load(x, q_from, q_stride, row0, g.Hq);

  const int half = a.rot_dim / 2, pos = a.pos[i];
  for (int p = lane; p < half; p += 32) {
    double c, s;
    cos_sin((double)pos * a.freq[p], &c, &s);
    s_turn[warp][p] = make_float2((float)(c * a.scale), (float)(s * a.scale));
  }
  const int b = sequence_of(a.tok_off, g.B, a.n_tokens, i);
  if (b < 0) return;                                     // a token of no sequence (the whole warp)
  const int at = i - tokens_of(a.tok_off, b, a.n_tokens).first;
  __syncwarp();

  const int rot_pieces = a.rot_dim / EPV, hp = rot_pieces / 2;
  const bool turns = piece < rot_pieces, upper = piece >= hp;
  const int partner = PAIRS || !turns ? lane : upper ? lane - hp : lane + hp;   // lane with the pairs' other elements
  float cs[EPV], sn[EPV];                                // y = x * cs + other * sn
#pragma unroll
  for (int e = 0; e < EPV; ++e) {
    const int p = PAIRS ? (piece * EPV + e) / 2 : (upper ? piece - hp : piece) * EPV + e;
    const float2 t = s_turn[warp][turns ? p : 0];
    cs[e] = t.x;
    sn[e] = (PAIRS ? (e & 1) != 0 : upper) ? t.y : -t.y;
  }
  auto rotated = [&](const uint4& v) {                   // whole warps
    float f[EPV], o[EPV], y[EPV];
    Elem<T>::unpack(v, f);
    if constexpr (PAIRS) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) o[e] = f[e ^ 1];
    } else {
      uint4 w;
      w.x = __shfl_sync(0xffffffffu, v.x, partner); w.y = __shfl_sync(0xffffffffu, v.y, partner);
      w.z = __shfl_sync(0xffffffffu, v.z, partner); w.w = __shfl_sync(0xffffffffu, v.w, partner);
      Elem<T>::unpack(w, o);
    }
#pragma unroll
    // Two products and a sum, each rounded: the arithmetic of the formula as it is written, so that a stored bf16
    // key, and with it the ordering key, is the one any plain fp32 form of it stores
    for (int e = 0; e < EPV; ++e) y[e] = __fadd_rn(__fmul_rn(f[e], cs[e]), __fmul_rn(o[e], sn[e]));
    const uint4 r = pack_piece<T>(y);
    return turns ? r : v;                                // (dimensions from rot_dim on are copied)
  };

  char* const q_to = reinterpret_cast<char*>(a.q_out.row<T>(l, i, 0)) + piece * 16;
  const long long q_to_stride = a.q_out.sh * (long long)sizeof(T);
  for (int r0 = row0; r0 - row0 + group < g.Hq; r0 += U * STEP) {
    if (r0 != row0) load(x, q_from, q_stride, r0, g.Hq);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint4 y = rotated(x[u]);
      if (r0 + u * STEP < g.Hq) st_stream(q_to + (r0 + u * STEP) * q_to_stride, y);
    }
  }

  // keys and values side by side, half a batch of each
  const long long bl = (long long)b * g.L + l;
  const int cap = g.cap(bl);
  const long long slot_all = a.per_head ? 0 : (long long)max(0, a.start[bl]) + at;
  const char* const k_from = reinterpret_cast<const char*>(a.k.row<T>(l, i, 0)) + piece * 16;
  const char* const v_from = reinterpret_cast<const char*>(a.v.row<T>(l, i, 0)) + piece * 16;
  const long long k_stride = a.k.sh * (long long)sizeof(T), v_stride = a.v.sh * (long long)sizeof(T);
  const long long cache0 = g.base(b, l, 0) + piece * EPV, meta0 = g.meta(bl * g.H);
  const long long meta_h = g.row_off ? g.total_rows : (long long)g.t_cap;
  for (int r0 = row0; r0 - row0 + group < g.H; r0 += U / 2 * STEP) {
#pragma unroll
    for (int u = 0; u < U / 2; ++u) {
      const int h = r0 + u * STEP;
      x[2 * u] = h < g.H ? ld_once(k_from + h * k_stride) : make_uint4(0, 0, 0, 0);
      x[2 * u + 1] = h < g.H ? ld_once(v_from + h * v_stride) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < U / 2; ++u) {
      const int h = r0 + u * STEP;
      const uint4 y = rotated(x[2 * u]);
      const float key = piece_sumsq_reduce<T, LPR>(y);   // of the row as it is stored
      if (h >= g.H) continue;
      const long long slot = a.per_head ? (long long)max(0, a.start[bl * g.H + h]) + at : slot_all;
      if (slot >= cap) {
        if (piece == 0) atomicExch(a.status, (int)L2KV_ERR_DEVICE_OVERFLOW);
        continue;
      }
      if (!L2KV_BOUNDS(g.holds(bl, slot), a.status)) continue;
      const long long to = cache0 + h * g.sh + slot * g.st;
      *reinterpret_cast<uint4*>(K + to) = y;
      *reinterpret_cast<uint4*>(V + to) = x[2 * u + 1];
      if (piece == 0) {
        const long long m = meta0 + h * meta_h + slot;
        if (a.idx) a.idx[m] = pos;
        if (a.sumsq) a.sumsq[m] = key;
      }
    }
  }
}

template <typename T, int D, int WPT, bool PAIRS>
static int launch_rw(const RotaryArgs& a, void* K, void* V, cudaStream_t s) {
  constexpr int TPB = kRotaryWarps / WPT;
  const long long units = (long long)a.g.B * a.g.L * (a.per_head ? a.g.H : 1);
  const long long blocks = ((long long)a.n_tokens * a.g.L + TPB - 1) / TPB + (units + kRotaryThreads - 1) / kRotaryThreads;
  if (blocks * TPB > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  return launch_early(rotary_write_kernel<T, D, WPT, PAIRS>, dim3((unsigned)blocks), kRotaryThreads, 0, s, a,
                      static_cast<T*>(K), static_cast<T*>(V));
}
// One warp per token where that gives every SM a block of them (148 of 8), else a block per token.  (32 + 8 heads of 128,
// warp / block in us: 300 tokens 7.0 / 5.3, 600 8.9 / 8.2, 1200 12.3 / 12.7, 2400 13.8 / 22.5, 9600 42.6 / 89.4.)
template <typename T, int D>
static int launch_rw_t(const RotaryArgs& a, void* K, void* V, cudaStream_t s) {
  const bool many = (long long)a.n_tokens * a.g.L >= 148 * kRotaryWarps;
  if (a.interleaved) return many ? launch_rw<T, D, 1, true>(a, K, V, s) : launch_rw<T, D, kRotaryWarps, true>(a, K, V, s);
  return many ? launch_rw<T, D, 1, false>(a, K, V, s) : launch_rw<T, D, kRotaryWarps, false>(a, K, V, s);
}

int launch_rotary_write(const TokView& q, const TokView& k, const TokView& v, const TokView& q_out,
                        const int32_t* tok_off, int n_tokens, const int32_t* pos, const double* freq,
                        int rot_dim, double scale, int interleaved, void* K, void* V, int32_t* idx,
                        float* sumsq, const Geom& g, int dtype, const int32_t* start, int32_t* cur_len,
                        int per_head, int32_t* status, cudaStream_t s) {
  const RotaryArgs a{q, k, v, q_out, g, tok_off, pos, freq, start, cur_len, idx, sumsq, status,
                     n_tokens, rot_dim, interleaved, per_head, scale};
  if (dtype == L2KV_BF16) return g.D == 128 ? launch_rw_t<__nv_bfloat16, 128>(a, K, V, s) : launch_rw_t<__nv_bfloat16, 64>(a, K, V, s);
  return g.D == 128 ? launch_rw_t<float, 128>(a, K, V, s) : launch_rw_t<float, 64>(a, K, V, s);
}

// ---- the accepted path of a tree -----------------------------------------------------------------
// One block per (b, l), a warp per head: it has read every length before it writes one, so the lengths may be
// updated in place, and no two warps touch the same rows.  A path is strictly increasing, so path[j] >= j:
// entries are taken in passes of ascending j, everything a pass moves is loaded before anything is stored,
// and no store can meet a row that a later pass still needs.  What a call takes is a chain of three round
// trips to memory (path and lengths, rows, stores); kCommitRows rows of K and of V per lane are in flight.
constexpr int kCommitWarps = 8;
constexpr int kCommitRows = 4;

template <typename T, int D>
__global__ void __launch_bounds__(32 * kCommitWarps)
tree_commit_kernel(T* K, T* V, int32_t* idx, float* sumsq, Geom g, const int32_t* start_dev, const int32_t* cur_dev,
                   const int32_t* path, int path_cap, const int32_t* n_path, int32_t* len_out, int per_head,
                   int32_t* status) {
  constexpr int EPV = Elem<T>::kPerVec, LPR = D / EPV, RPW = 32 / LPR;
  const long long bl = blockIdx.x;
  const int b = (int)(bl / g.L), l = (int)(bl % g.L);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane % LPR;
  const int32_t* p = path + (long long)b * path_cap;
  next_may_start();
  wait_for_previous();
  const int first = lane < path_cap ? p[lane] : 0;       // (asked for before n_path is known)
  const int want = max(0, min(n_path[b], path_cap)), cap = g.cap(bl);
  int len = 0;                                           // of the last head this warp took
  bool bad = false;
  for (int h = warp; h < g.H; h += kCommitWarps) {
    const long long u = per_head ? bl * g.H + h : bl;
    const int start = max(0, min(start_dev[u], cap)), tail = max(0, min(cur_dev[u], cap) - start);
    const long long base = g.base(b, l, h) + (long long)start * g.st + piece * EPV, meta = g.meta(bl * g.H + h) + start;
    int kept = 0, last = -1;                             // last: the entry before this group of 32
    while (kept < want) {
      const int j0 = kept, mine = j0 == 0 ? first : j0 + lane < want ? p[j0 + lane] : 0;
      int before = __shfl_up_sync(0xffffffffu, mine, 1);
      if (lane == 0) before = last;
      // entries of this group before the first that does not increase or leaves the tree
      const unsigned wrong = __ballot_sync(0xffffffffu, j0 + lane < want && (mine <= before || mine >= tail));
      const int n = min(min(32, want - j0), wrong ? __ffs(wrong) - 1 : 32);
      for (int e0 = 0; e0 < n; e0 += RPW * kCommitRows) {
        uint4 vk[kCommitRows], vv[kCommitRows];
        int32_t vi[kCommitRows];
        float vs[kCommitRows];
        bool go[kCommitRows];
#pragma unroll
        for (int r = 0; r < kCommitRows; ++r) {
          const int e = e0 + r * RPW + lane / LPR;
          const int from = __shfl_sync(0xffffffffu, mine, e & 31);
          go[r] = e < n && from != j0 + e;
          if (go[r]) go[r] = L2KV_BOUNDS(from > j0 + e && g.holds(bl, (long long)start + from), status);
          if (!go[r]) continue;
          vk[r] = *reinterpret_cast<const uint4*>(K + base + from * g.st);
          vv[r] = *reinterpret_cast<const uint4*>(V + base + from * g.st);
          if (piece == 0) {
            if (idx) vi[r] = idx[meta + from];
            if (sumsq) vs[r] = sumsq[meta + from];
          }
        }
        __syncwarp();
#pragma unroll
        for (int r = 0; r < kCommitRows; ++r) {
          if (!go[r]) continue;
          const int to = j0 + e0 + r * RPW + lane / LPR;
          *reinterpret_cast<uint4*>(K + base + to * g.st) = vk[r];
          *reinterpret_cast<uint4*>(V + base + to * g.st) = vv[r];
          if (piece == 0) {
            if (idx) idx[meta + to] = vi[r];
            if (sumsq) sumsq[meta + to] = vs[r];
          }
        }
        __syncwarp();
      }
      kept += n;
      last = __shfl_sync(0xffffffffu, mine, 31);
      if (n < 32) break;
    }
    bad |= kept < want;
    len = start + kept;
    if (per_head && lane == 0) len_out[u] = len;         // (nobody else reads this head's lengths)
  }
  if (bad && lane == 0) atomicExch(status, (int)L2KV_ERR_OUT_OF_RANGE);
  if (per_head) return;
  __syncthreads();                                       // every warp has read the lengths
  if (threadIdx.x == 0) len_out[bl] = len;
}

template <typename T, int D>
static int launch_tc(void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, const int32_t* start,
                     const int32_t* cur, const int32_t* path, int path_cap, const int32_t* n_path,
                     int32_t* len_out, int per_head, int32_t* status, cudaStream_t s) {
  const long long blocks = (long long)g.B * g.L;
  if (blocks > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  return launch_early(tree_commit_kernel<T, D>, dim3((unsigned)blocks), 32 * kCommitWarps, 0, s, static_cast<T*>(K),
                      static_cast<T*>(V), idx, sumsq, g, start, cur, path, path_cap, n_path, len_out, per_head, status);
}

int launch_tree_commit(void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, int dtype,
                       const int32_t* start, const int32_t* cur, const int32_t* path, int path_cap,
                       const int32_t* n_path, int32_t* len_out, int per_head, int32_t* status, cudaStream_t s) {
#define L2KV_TC(T, D) \
  return launch_tc<T, D>(K, V, idx, sumsq, g, start, cur, path, path_cap, n_path, len_out, per_head, status, s)
  if (dtype == L2KV_BF16) {
    if (g.D == 128) L2KV_TC(__nv_bfloat16, 128);
    L2KV_TC(__nv_bfloat16, 64);
  }
  if (g.D == 128) L2KV_TC(float, 128);
  L2KV_TC(float, 64);
#undef L2KV_TC
}

}  // namespace l2kv
