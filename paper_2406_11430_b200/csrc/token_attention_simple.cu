// Prompt and tree attention on the CUDA cores, fp32 throughout: the path of fp32 caches, which have no
// exact tensor-core form.  One warp per (layer, token, query head), an online softmax over 32 cached
// rows at a time: for the scores a lane owns a row (its 16-byte pieces stay in L1 while the lane walks
// them), for the output it owns head_dim / 32 dimensions.  Rows that the token does not see are
// neither scored nor multiplied, whatever they hold.  Bound by instruction issue (about 2 D
// FMAs per cached row and query head, nothing shared between the heads of a group).
#include <climits>

#include "tokens.cuh"

namespace l2kv {

constexpr int kTsWarps = 4;

template <int D>
__global__ void __launch_bounds__(32 * kTsWarps)
token_attention_simple_kernel(const __grid_constant__ TokenAttention a, const float* __restrict__ K,
                              const float* __restrict__ V) {
  constexpr int DPL = D / 32;
  __shared__ __align__(16) float s_q[kTsWarps][D];
  const Geom& g = a.g;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int groups = (g.Hq + kTsWarps - 1) / kTsWarps;
  const int j = (int)(blockIdx.x % groups) * kTsWarps + warp;
  const long long il = blockIdx.x / groups;
  const int i = (int)(il % a.n_tokens), l = (int)(il / a.n_tokens);
  if (j >= g.Hq) return;
  // A wait that gave up in an earlier call marks the workspace; nothing runs until it is cleared.
  if (a.status && *reinterpret_cast<volatile int32_t*>(a.status + 2) != 0) return;
  const int b = sequence_of(a.tok_off, g.B, a.n_tokens, i);
  if (b < 0) return;
  const TokRange r = tokens_of(a.tok_off, b, a.n_tokens);
  const int h = j / (g.Hq / g.H);
  const long long bl = (long long)b * g.L + l;
  const int cur = max(0, min(a.lens.at(bl, h, g.H), min(a.max_len, g.cap(bl))));
  const int base = cur - r.n;                            // row of the sequence's first new token
  const int end = a.mask ? cur : max(0, min(cur, base + (i - r.first) + 1));

  const float* q = a.q.row<float>(l, i, j);
  for (int d = lane; d < D; d += 32) s_q[warp][d] = q[d];
  __syncwarp();
  const float* Ku = K + g.base(b, l, h);
  const float* Vu = V + g.base(b, l, h);
  float m = -INFINITY, sum = 0.f, o[DPL] = {};
  for (int t0 = 0; t0 < end; t0 += 32) {
    const int t = t0 + lane;
    bool sees = t < end;
    if (sees && a.mask && t >= base) {
      const int c = t - base;
      sees = c < 64 * a.mask_words && (a.mask[(long long)i * 2 * a.mask_words + (c >> 5)] >> (c & 31)) & 1u;
    }
    float s = -INFINITY;
    if (sees) {
      const float* row = Ku + (long long)t * g.st;
      float acc = 0.f;
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        const float4 x = *reinterpret_cast<const float4*>(row + d), y = *reinterpret_cast<const float4*>(&s_q[warp][d]);
        acc = fmaf(x.x, y.x, acc);
        acc = fmaf(x.y, y.y, acc);
        acc = fmaf(x.z, y.z, acc);
        acc = fmaf(x.w, y.w, acc);
      }
      s = acc * a.scale_log2e;
    }
    float top = s;
#pragma unroll
    for (int off = 16; off; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    const float m_new = fmaxf(m, top);
    if (m_new == -INFINITY && !__any_sync(0xffffffffu, s != s)) continue;   // nothing seen so far
    const float keep = exp2f(m - m_new);
    const float p = sees ? exp2f(s - m_new) : 0.f;
    m = m_new;
    sum = sum * keep + p;
#pragma unroll
    for (int e = 0; e < DPL; ++e) o[e] *= keep;
    unsigned who = __ballot_sync(0xffffffffu, sees);
    while (who) {
      const int k = __ffs(who) - 1;
      who &= who - 1;
      const float w = __shfl_sync(0xffffffffu, p, k);
      const float* row = Vu + (long long)(t0 + k) * g.st + lane * DPL;
#pragma unroll
      for (int e = 0; e < DPL; ++e) o[e] = fmaf(w, row[e], o[e]);
    }
  }
#pragma unroll
  for (int off = 16; off; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  float* out = a.out.row<float>(l, i, j) + lane * DPL;
#pragma unroll
  for (int e = 0; e < DPL; ++e) out[e] = sum == 0.f ? 0.f : o[e] * inv;
  if (a.lse && lane == 0)
    a.lse[((long long)l * a.n_tokens + i) * g.Hq + j] = sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f;
}

int launch_token_attention_simple(const TokenAttention& a, const void* K, const void* V, cudaStream_t s) {
  const long long blocks = (long long)a.n_tokens * a.g.L * ((a.g.Hq + kTsWarps - 1) / kTsWarps);
  if (blocks > INT_MAX) return L2KV_ERR_OUT_OF_RANGE;
  auto kern = a.g.D == 128 ? token_attention_simple_kernel<128> : token_attention_simple_kernel<64>;
  kern<<<(unsigned)blocks, 32 * kTsWarps, 0, s>>>(a, static_cast<const float*>(K), static_cast<const float*>(V));
  return cudaGetLastError() == cudaSuccess ? L2KV_OK : L2KV_ERR_CUDA;
}

}  // namespace l2kv
