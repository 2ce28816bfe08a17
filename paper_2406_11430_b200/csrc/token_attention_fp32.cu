// Prompt and tree attention on the CUDA cores, fp32 throughout: the path of fp32 caches, which have no
// exact tensor-core form.  A block per 32 query rows (tokens x heads of a group that share a KV head), an online
// softmax over the cache in blocks of 32 rows, which come through shared memory so that each cached element is
// fetched once per 32 rows.  128 threads: eight share two query rows, for scores with a quarter of the cached rows
// each (every eighth, so that their reads meet different banks), for the output with an eighth of the dimensions.
// Rows that a token does not see are neither counted nor multiplied, whatever they hold.  Bound by shared-memory
// reads, ten of 16 bytes per 64 FMAs: 2 prompts of 1000 tokens, 32 heads of 128 (16.4 GFLOP), 0.93 ms (a warp
// per row, which reads the cache through L1, 5.97); one token behind 2000 rows, 32 heads, 0.52 ms (0.68).
#include <algorithm>
#include <climits>

#include "tokens.cuh"

namespace l2kv {

constexpr int kTfRows = 32, kTfCols = 32;
template <int D> constexpr int kTfSmem = (kTfRows * D + kTfCols * (D + 4) + kTfCols * D + kTfRows * (kTfCols + 4)) * 4;

template <int D>
__global__ void __launch_bounds__(128)
token_attention_fp32_kernel(const __grid_constant__ TokenAttention a, const float* __restrict__ K,
                            const float* __restrict__ V) {
  extern __shared__ __align__(16) float smem_f[];
  float* const s_q = smem_f;                             // [rows][D]
  float* const s_k = s_q + kTfRows * D;                  // [cols][D + 4]
  float* const s_v = s_k + kTfCols * (D + 4);            // [cols][D]
  float* const s_p = s_v + kTfCols * D;                  // [rows][cols + 4]
  const Geom& g = a.g;
  const int tid = threadIdx.x, lane = tid & 31, tx = tid & 7, r0 = 2 * (tid >> 3), G = g.Hq / g.H;
  const int h = (int)(blockIdx.x % (unsigned)g.H), l = (int)(blockIdx.x / (unsigned)g.H % (unsigned)g.L);
  int tile = (int)(blockIdx.x / (unsigned)g.H / (unsigned)g.L);
  // A wait that gave up in an earlier call marks the workspace; nothing runs until it is cleared.
  if (a.status && *reinterpret_cast<volatile int32_t*>(a.status + 2) != 0) return;
  // the sequence whose tile this is: 32 sequences at a time
  int b = -1;
  for (int b0 = 0; b0 < g.B; b0 += 32) {
    const int mine = b0 + lane < g.B ? (tokens_of(a.tok_off, b0 + lane, a.n_tokens).n * G + kTfRows - 1) / kTfRows : 0;
    int incl = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, incl, off);
      if (lane >= off) incl += o;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, tile < incl);
    if (hit) {
      const int who = __ffs(hit) - 1;
      tile -= __shfl_sync(0xffffffffu, incl - mine, who);
      b = b0 + who;
      break;
    }
    tile -= __shfl_sync(0xffffffffu, incl, 31);
  }
  if (b < 0) return;
  const TokRange range = tokens_of(a.tok_off, b, a.n_tokens);
  const long long bl = (long long)b * g.L + l;
  const int cur = max(0, min(a.lens.at(bl, h, g.H), min(a.max_len, g.cap(bl))));
  const int base = cur - range.n, first = tile * kTfRows, rows = min(kTfRows, range.n * G - first);
  int end = a.mask ? cur : max(0, min(cur, base + (first + rows - 1) / G + 1));
  if (end > 0 && !L2KV_BOUNDS(g.holds(bl, 0) && g.holds(bl, end - 1), a.status)) end = 0;
  const int clear = a.mask ? base : base + first / G + 1;                    // rows below it are seen by all

  for (int e = tid; e < kTfRows * D / 4; e += 128) {
    const int r = e / (D / 4), d = e % (D / 4) * 4, i = range.first + (first + r) / G;
    *reinterpret_cast<float4*>(s_q + r * D + d) =
        r < rows ? *reinterpret_cast<const float4*>(a.q.row<float>(l, i, h * G + (first + r) % G) + d) : make_float4(0, 0, 0, 0);
  }
  const float* const Ku = K + g.base(b, l, h);
  const float* const Vu = V + g.base(b, l, h);
  int limit[2];
  const uint32_t* mask[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = min(r0 + e, rows - 1), s = (first + r) / G;
    limit[e] = a.mask ? cur : min(cur, base + s + 1);
    mask[e] = a.mask + (a.mask ? (long long)(range.first + s) * 2 * a.mask_words : 0);
  }
  float m[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f}, o[2][D / 8] = {};
  for (int t0 = 0; t0 < end; t0 += kTfCols) {
    __syncthreads();                                     // the block before has been read
    for (int e = tid; e < kTfCols * D / 4; e += 128) {
      const int c = e / (D / 4), d = e % (D / 4) * 4;
      const long long at = (long long)(t0 + c) * g.st + d;
      const bool in = t0 + c < end;
      *reinterpret_cast<float4*>(s_k + c * (D + 4) + d) = in ? *reinterpret_cast<const float4*>(Ku + at) : make_float4(0, 0, 0, 0);
      *reinterpret_cast<float4*>(s_v + c * D + d) = in ? *reinterpret_cast<const float4*>(Vu + at) : make_float4(0, 0, 0, 0);
    }
    __syncthreads();
    float s[2][4] = {};
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
      const float4 qa = *reinterpret_cast<const float4*>(s_q + r0 * D + d), qb = *reinterpret_cast<const float4*>(s_q + (r0 + 1) * D + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 k = *reinterpret_cast<const float4*>(s_k + (tx + 8 * j) * (D + 4) + d);
        s[0][j] = fmaf(qa.x, k.x, fmaf(qa.y, k.y, fmaf(qa.z, k.z, fmaf(qa.w, k.w, s[0][j]))));
        s[1][j] = fmaf(qb.x, k.x, fmaf(qb.y, k.y, fmaf(qb.z, k.z, fmaf(qb.w, k.w, s[1][j]))));
      }
    }
    const bool masked = t0 + kTfCols > clear;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      bool sees[4];
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = t0 + tx + 8 * j, c = t - base;
        sees[j] = t < limit[e];
        if (a.mask && c >= 0 && sees[j]) sees[j] = c < 64 * a.mask_words && (mask[e][c >> 5] >> (c & 31) & 1u);
        s[e][j] *= a.scale_log2e;
        if (sees[j]) top = fmaxf(top, s[e][j]);
      }
#pragma unroll
      for (int off = 4; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
      const float m_new = fmaxf(m[e], top), low = m_new == -INFINITY ? 0.f : m_new;
      const float keep = exp2f(m[e] - low);              // (0 while nothing has been seen)
      m[e] = m_new;
      sum[e] *= keep;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) o[e][i] *= keep;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = sees[j] ? exp2f(s[e][j] - low) : 0.f;
        sum[e] += p;
        s_p[(r0 + e) * (kTfCols + 4) + tx + 8 * j] = p;
      }
    }
    __syncwarp();                                        // a row's eight threads are in one warp
    for (int c = 0; c < kTfCols; c += 4) {
      const float4 pa = *reinterpret_cast<const float4*>(s_p + r0 * (kTfCols + 4) + c);
      const float4 pb = *reinterpret_cast<const float4*>(s_p + (r0 + 1) * (kTfCols + 4) + c);
      const float wa[4] = {pa.x, pa.y, pa.z, pa.w}, wb[4] = {pb.x, pb.y, pb.z, pb.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const float4 v = *reinterpret_cast<const float4*>(s_v + (c + k) * D + 32 * i + 4 * tx);
          // (a value that the row does not see may be anything)
          if (!masked || wa[k] != 0.f) {
            o[0][4 * i] = fmaf(wa[k], v.x, o[0][4 * i]);
            o[0][4 * i + 1] = fmaf(wa[k], v.y, o[0][4 * i + 1]);
            o[0][4 * i + 2] = fmaf(wa[k], v.z, o[0][4 * i + 2]);
            o[0][4 * i + 3] = fmaf(wa[k], v.w, o[0][4 * i + 3]);
          }
          if (!masked || wb[k] != 0.f) {
            o[1][4 * i] = fmaf(wb[k], v.x, o[1][4 * i]);
            o[1][4 * i + 1] = fmaf(wb[k], v.y, o[1][4 * i + 1]);
            o[1][4 * i + 2] = fmaf(wb[k], v.z, o[1][4 * i + 2]);
            o[1][4 * i + 3] = fmaf(wb[k], v.w, o[1][4 * i + 3]);
          }
        }
    }
    __syncwarp();
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int off = 4; off; off >>= 1) sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], off);
    if (r0 + e >= rows) continue;
    const float inv = sum[e] == 0.f ? 0.f : 1.f / sum[e];
    const int i = range.first + (first + r0 + e) / G, j = h * G + (first + r0 + e) % G;
    float* const out = a.out.row<float>(l, i, j) + 4 * tx;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      *reinterpret_cast<float4*>(out + 32 * c) = sum[e] == 0.f ? make_float4(0, 0, 0, 0)
          : make_float4(o[e][4 * c] * inv, o[e][4 * c + 1] * inv, o[e][4 * c + 2] * inv, o[e][4 * c + 3] * inv);
    if (a.lse && tx == 0)
      a.lse[((long long)l * a.n_tokens + i) * g.Hq + j] =
          sum[e] == 0.f ? -INFINITY : (m[e] + log2f(sum[e])) * 0.6931471805599453f;
  }
}

template <int D>
static int launch_tf(const TokenAttention& a, const void* K, const void* V, cudaStream_t s) {
  const long long rows = (long long)a.n_tokens * (a.g.Hq / a.g.H);
  const long long blocks = (rows / kTfRows + std::min(a.g.B, a.n_tokens)) * a.g.H * a.g.L;
  if (blocks > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  auto kern = token_attention_fp32_kernel<D>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kTfSmem<D>) != cudaSuccess)
    return L2KV_ERR_CUDA;
  kern<<<(unsigned)blocks, 128, kTfSmem<D>, s>>>(a, static_cast<const float*>(K), static_cast<const float*>(V));
  return cudaGetLastError() == cudaSuccess ? L2KV_OK : L2KV_ERR_CUDA;
}

int launch_token_attention_fp32(const TokenAttention& a, const void* K, const void* V, cudaStream_t s) {
  return a.g.D == 128 ? launch_tf<128>(a, K, V, s) : launch_tf<64>(a, K, V, s);
}

}  // namespace l2kv
