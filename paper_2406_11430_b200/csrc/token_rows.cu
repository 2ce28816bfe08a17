// Rows of new tokens in and around the cache: rotary positions with the cache write, and the move of a
// drafted tree's accepted path down to the end of the committed rows.  Both move each row once
// and compute next to nothing, so what bounds them is the memory traffic, or, for a handful of
// tokens, the chain of dependent loads before the first row can go out.
#include <climits>

#include "tokens.cuh"

namespace l2kv {

// ---- rotary positions and cache write ------------------------------------------------------------
// One block per (token, layer).  A row (one head of q, k or v) belongs to LPR adjacent lanes, a
// 16-byte piece each, as everywhere in the library; a half-split pair's other element is in another
// lane of the row, an interleaved pair's in the same piece.  A thread meets the same piece of
// every row, so it keeps that piece's cosines and sines in registers.
constexpr int kRotaryThreads = 256;

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

template <typename T, int D>
__global__ void __launch_bounds__(kRotaryThreads)
rotary_write_kernel(const __grid_constant__ RotaryArgs a, T* __restrict__ K, T* __restrict__ V) {
  constexpr int EPV = Elem<T>::kPerVec, LPR = D / EPV, RPB = kRotaryThreads / LPR;
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 31, piece = tid % LPR;
  const long long n_rows = (long long)a.n_tokens * g.L;
  if (blockIdx.x >= n_rows) {
    // trailing blocks: the new lengths (sequences without new tokens have one too)
    const long long u = (blockIdx.x - n_rows) * kRotaryThreads + tid;
    const long long units = (long long)g.B * g.L * (a.per_head ? g.H : 1);
    if (u >= units) return;
    const long long bl = a.per_head ? u / g.H : u;
    const int b = (int)(bl / g.L);
    const int n = tokens_of(a.tok_off, b, a.n_tokens).n;
    a.cur_len[u] = (int)min((long long)g.cap(bl), (long long)max(0, a.start[u]) + n);
    return;
  }
  const int i = (int)(blockIdx.x / g.L), l = (int)(blockIdx.x % g.L);
  __shared__ float s_cos[D / 2], s_sin[D / 2];
  const int half = a.rot_dim / 2;
  if (tid < half) {
    double s, c;
    sincos((double)a.pos[i] * a.freq[tid], &s, &c);
    s_cos[tid] = (float)(c * a.scale);
    s_sin[tid] = (float)(s * a.scale);
  }
  const int b = sequence_of(a.tok_off, g.B, a.n_tokens, i);
  if (b < 0) return;                                    // a token of no sequence (whole block)
  const int at = i - tokens_of(a.tok_off, b, a.n_tokens).first;
  __syncthreads();

  const int rot_pieces = a.rot_dim / EPV;
  float cs[EPV], sn[EPV];                                // y = x * cs + partner * sn
  int from = lane;                                       // lane that holds the partner's piece
  if (piece < rot_pieces) {
    if (a.interleaved) {
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const int p = (piece * EPV + e) / 2;
        cs[e] = s_cos[p];
        sn[e] = e & 1 ? s_sin[p] : -s_sin[p];
      }
    } else {
      const int hp = rot_pieces / 2;
      const bool upper = piece >= hp;
      from = upper ? lane - hp : lane + hp;
#pragma unroll
      for (int e = 0; e < EPV; ++e) {
        const int p = (upper ? piece - hp : piece) * EPV + e;
        cs[e] = s_cos[p];
        sn[e] = upper ? s_sin[p] : -s_sin[p];
      }
    }
  }

  const int rows = g.Hq + 2 * g.H;
  for (int r0 = 0; r0 < rows; r0 += RPB) {
    const int r = r0 + tid / LPR;
    const bool is_q = r < g.Hq, is_k = !is_q && r < g.Hq + g.H, any = r < rows;
    const int h = is_q ? r : is_k ? r - g.Hq : r - g.Hq - g.H;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (any) {
      const TokView& from_t = is_q ? a.q : is_k ? a.k : a.v;
      x = *reinterpret_cast<const uint4*>(from_t.row<T>(l, i, h) + piece * EPV);
    }
    uint4 other;
    other.x = __shfl_sync(0xffffffffu, x.x, from); other.y = __shfl_sync(0xffffffffu, x.y, from);
    other.z = __shfl_sync(0xffffffffu, x.z, from); other.w = __shfl_sync(0xffffffffu, x.w, from);
    if ((is_q || is_k) && piece < rot_pieces) {
      float f[EPV], o[EPV], y[EPV];
      Elem<T>::unpack(x, f);
      Elem<T>::unpack(other, o);
#pragma unroll
      for (int e = 0; e < EPV; ++e)
        y[e] = __fmaf_rn(f[e], cs[e], (a.interleaved ? f[e ^ 1] : o[e]) * sn[e]);
      x = pack_piece<T>(y);
    }
    // the key of the row as it is stored
    float key = 0.f;
    if (__any_sync(0xffffffffu, is_k)) key = piece_sumsq_reduce<T, LPR>(x);
    if (!any) continue;
    if (is_q) {
      *reinterpret_cast<uint4*>(a.q_out.row<T>(l, i, h) + piece * EPV) = x;
      continue;
    }
    const long long bl = (long long)b * g.L + l, unit = bl * g.H + h;
    const long long slot = (long long)max(0, a.start[a.per_head ? unit : bl]) + at;
    if (slot >= g.cap(bl)) {
      if (piece == 0) atomicExch(a.status, (int)L2KV_ERR_DEVICE_OVERFLOW);
      continue;
    }
    const long long to = g.base(b, l, h) + slot * g.st + piece * EPV;
    *reinterpret_cast<uint4*>((is_k ? K : V) + to) = x;
    if (is_k && piece == 0) {
      const long long m = g.meta(unit) + slot;
      if (a.idx) a.idx[m] = a.pos[i];
      if (a.sumsq) a.sumsq[m] = key;
    }
  }
}

template <typename T, int D>
static int launch_rw(const RotaryArgs& a, void* K, void* V, cudaStream_t s) {
  const long long units = (long long)a.g.B * a.g.L * (a.per_head ? a.g.H : 1);
  const long long blocks = (long long)a.n_tokens * a.g.L + (units + kRotaryThreads - 1) / kRotaryThreads;
  if (blocks > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  rotary_write_kernel<T, D><<<(unsigned)blocks, kRotaryThreads, 0, s>>>(a, static_cast<T*>(K), static_cast<T*>(V));
  return cudaGetLastError() == cudaSuccess ? L2KV_OK : L2KV_ERR_CUDA;
}

int launch_rotary_write(const TokView& q, const TokView& k, const TokView& v, const TokView& q_out,
                        const int32_t* tok_off, int n_tokens, const int32_t* pos, const double* freq,
                        int rot_dim, double scale, int interleaved, void* K, void* V, int32_t* idx,
                        float* sumsq, const Geom& g, int dtype, const int32_t* start, int32_t* cur_len,
                        int per_head, int32_t* status, cudaStream_t s) {
  const RotaryArgs a{q, k, v, q_out, g, tok_off, pos, freq, start, cur_len, idx, sumsq, status,
                     n_tokens, rot_dim, interleaved, per_head, scale};
  if (dtype == L2KV_BF16) return g.D == 128 ? launch_rw<__nv_bfloat16, 128>(a, K, V, s) : launch_rw<__nv_bfloat16, 64>(a, K, V, s);
  return g.D == 128 ? launch_rw<float, 128>(a, K, V, s) : launch_rw<float, 64>(a, K, V, s);
}

// ---- the accepted path of a tree -----------------------------------------------------------------
// One block per (b, l), all heads: it has read every length before it writes one, so the lengths may
// be updated in place.  A path is strictly increasing, so path[j] >= j: rows are taken in
// passes of ascending j, everything a pass moves is loaded before anything is stored, and no store
// can meet a row that a later pass still needs.  Two rows of K and of V in flight per thread.
constexpr int kCommitThreads = 512;
constexpr int kCommitRows = 2;

template <typename T, int D>
__global__ void __launch_bounds__(kCommitThreads)
tree_commit_kernel(T* __restrict__ K, T* __restrict__ V, int32_t* __restrict__ idx,
                   float* __restrict__ sumsq, Geom g, const int32_t* start_dev, const int32_t* cur_dev,
                   const int32_t* __restrict__ path, int path_cap, const int32_t* __restrict__ n_path,
                   int32_t* len_out, int per_head, int32_t* __restrict__ status) {
  constexpr int EPV = Elem<T>::kPerVec, LPR = D / EPV, RPB = kCommitThreads / LPR;
  __shared__ int s_ok;                                   // entries before the first that does not increase
  const long long bl = blockIdx.x;
  const int b = (int)(bl / g.L), l = (int)(bl % g.L);
  const int tid = threadIdx.x, piece = tid % LPR;
  const int32_t* p = path + (long long)b * path_cap;
  const int want = max(0, min(n_path[b], path_cap));
  const int cap = g.cap(bl);
  auto start_of = [&](int h) { return max(0, min(start_dev[per_head ? bl * g.H + h : bl], cap)); };
  auto tail_of = [&](int h) { return max(0, min(cur_dev[per_head ? bl * g.H + h : bl], cap) - start_of(h)); };
  if (tid == 0) s_ok = want;
  __syncthreads();
  for (int j = tid; j < want; j += kCommitThreads)
    if (p[j] <= (j ? p[j - 1] : -1)) atomicMin(&s_ok, j);
  __syncthreads();
  const int ok = s_ok;

  const long long moves = (long long)ok * g.H;           // move f: entry f / H, head f % H
  for (long long f0 = 0; f0 < moves; f0 += RPB * kCommitRows) {
    uint4 vk[kCommitRows], vv[kCommitRows];
    int32_t vi[kCommitRows];
    float vs[kCommitRows];
    bool go[kCommitRows];
#pragma unroll
    for (int u = 0; u < kCommitRows; ++u) {
      const long long f = f0 + u * RPB + tid / LPR;
      const int j = (int)(f / g.H), h = (int)(f % g.H);
      go[u] = false;
      if (f >= moves) continue;
      const int from = p[j];
      go[u] = from != j && from < tail_of(h);
      if (!go[u]) continue;
      const int row0 = start_of(h);
      const long long at = g.base(b, l, h) + (long long)(row0 + from) * g.st + piece * EPV;
      vk[u] = *reinterpret_cast<const uint4*>(K + at);
      vv[u] = *reinterpret_cast<const uint4*>(V + at);
      if (piece == 0) {
        const long long m = g.meta(bl * g.H + h) + row0 + from;
        if (idx) vi[u] = idx[m];
        if (sumsq) vs[u] = sumsq[m];
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kCommitRows; ++u) {
      if (!go[u]) continue;
      const long long f = f0 + u * RPB + tid / LPR;
      const int j = (int)(f / g.H), h = (int)(f % g.H);
      const int row0 = start_of(h);
      const long long at = g.base(b, l, h) + (long long)(row0 + j) * g.st + piece * EPV;
      *reinterpret_cast<uint4*>(K + at) = vk[u];
      *reinterpret_cast<uint4*>(V + at) = vv[u];
      if (piece == 0) {
        const long long m = g.meta(bl * g.H + h) + row0 + j;
        if (idx) idx[m] = vi[u];
        if (sumsq) sumsq[m] = vs[u];
      }
    }
  }

  // The new lengths.  Every read of the old ones by another thread lies before this barrier.  Entries
  // are increasing, so those inside the tail are the first ones.
  __syncthreads();
  for (int h = tid; h < (per_head ? g.H : 1); h += kCommitThreads) {
    const int tail = tail_of(h);
    int lo = 0, hi = ok;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (p[mid] < tail) lo = mid + 1; else hi = mid;
    }
    if (lo < want) atomicExch(status, (int)L2KV_ERR_OUT_OF_RANGE);
    len_out[per_head ? bl * g.H + h : bl] = start_of(h) + lo;
  }
}

template <typename T, int D>
static int launch_tc(void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, const int32_t* start,
                     const int32_t* cur, const int32_t* path, int path_cap, const int32_t* n_path,
                     int32_t* len_out, int per_head, int32_t* status, cudaStream_t s) {
  const long long blocks = (long long)g.B * g.L;
  if (blocks > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  tree_commit_kernel<T, D><<<(unsigned)blocks, kCommitThreads, 0, s>>>(
      static_cast<T*>(K), static_cast<T*>(V), idx, sumsq, g, start, cur, path, path_cap, n_path, len_out,
      per_head, status);
  return cudaGetLastError() == cudaSuccess ? L2KV_OK : L2KV_ERR_CUDA;
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
