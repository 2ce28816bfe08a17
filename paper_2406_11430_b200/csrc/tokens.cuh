// The packed list of new tokens: which sequence a token belongs to, and where its rows lie.
#pragma once

#include "pages.cuh"

namespace l2kv {

// Rows of tokens, [layers, n_tokens, heads, head_dim] with strides in elements.
struct TokView {
  void* p;
  long long sl, st, sh;
  template <typename T>
  __device__ __forceinline__ T* row(int l, int i, int h) const {
    return static_cast<T*>(p) + l * sl + i * st + h * sh;
  }
};

inline TokView make_view(const l2kv_tokens* t) {
  return t ? TokView{t->data, t->stride_l, t->stride_t, t->stride_h} : TokView{nullptr, 0, 0, 0};
}

// The tokens of sequence b: [first, first + n) of the list.  Offsets come from device memory and are
// brought into [0, n_tokens] whatever they hold.
struct TokRange { int first, n; };
__device__ __forceinline__ TokRange tokens_of(const int32_t* tok_off, int b, int n_tokens) {
  const int lo = max(0, min(tok_off[b], n_tokens)), hi = max(0, min(tok_off[b + 1], n_tokens));
  return {lo, max(0, hi - lo)};
}

// The sequence that token i belongs to: the number of sequences that end at or before i, counted 32
// at a time by the lanes of a warp; -1 for a token of no sequence.  Whole warps only.
__device__ __forceinline__ int sequence_of(const int32_t* tok_off, int B, int n_tokens, int i) {
  const int lane = threadIdx.x & 31;
  for (int b0 = 0; b0 < B; b0 += 32) {
    const bool past = b0 + lane < B && tok_off[b0 + lane + 1] <= i;
    const unsigned m = __ballot_sync(0xffffffffu, !past);
    if (m) {                                             // the first sequence of this group that is not over
      const int b = b0 + __ffs(m) - 1;
      if (b >= B) return -1;
      const TokRange r = tokens_of(tok_off, b, n_tokens);
      return i >= r.first && i < r.first + r.n ? b : -1;
    }
  }
  return -1;
}

// These calls follow one another step after step, most of them for a few microseconds, so a kernel may be set
// up on the SMs while the one before it in the stream runs: it is launched with launch_early, says at its start
// that the next one may do the same, and waits for everything before it -- complete, and visible -- before its first
// access to global memory.  A kernel that is launched without asking for this waits as always.  None of the early
// ones has a __restrict__ parameter: that would promise that nobody else writes the memory while the kernel lives, and
// would let the compiler read it before the wait, while the kernel before is still writing it.
__device__ __forceinline__ void next_may_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
inline int launch_early(void (*kern)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, A&&... args) {
  cudaLaunchAttribute early{};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &early;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<A&&>(args)...) == cudaSuccess ? L2KV_OK : L2KV_ERR_CUDA;
}

// A 16-byte load that leaves no line in L1.  (Not through the read-only path: q_out may be q, and
// other calls write the rows.)
__device__ __forceinline__ uint4 ld_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

template <typename... P, typename... A>
inline int launch_chained(void (*kern)(P...), long long blocks, unsigned y, unsigned threads, size_t smem, cudaStream_t s, A&&... args) {
  return launch_early(kern, dim3((unsigned)blocks, y), threads, smem, s, static_cast<A&&>(args)...);
}

int launch_rotary_write(const TokView& q, const TokView& k, const TokView& v, const TokView& q_out,
                        const int32_t* tok_off, int n_tokens, const int32_t* pos, const double* freq,
                        int rot_dim, double scale, int interleaved, void* K, void* V, int32_t* idx,
                        float* sumsq, const Geom& g, int dtype, const int32_t* start, int32_t* cur_len,
                        int per_head, int32_t* status, cudaStream_t s);
// The same with norms of queries and keys before the rotation, into pages or rows.
struct NormArgs {
  PageView pages;                                        // table == nullptr: the cache has rows of its own
  const void* q_weight;                                  // [head_dim] in the cache's dtype, or null: ones
  const void* k_weight;
  int norm_q, norm_k;
  float eps, offset;                                     // offset: what is added to the weights
};
int launch_norm_rotary_write(const TokView& q, const TokView& k, const TokView& v, const TokView& q_out,
                             const int32_t* tok_off, int n_tokens, const int32_t* pos, const double* freq,
                             int rot_dim, double scale, int interleaved, const NormArgs& norm, void* K, void* V,
                             int32_t* idx, float* sumsq, const Geom& g, int dtype, const int32_t* start,
                             int32_t* cur_len, int per_head, int32_t* status, cudaStream_t s);
int launch_tree_commit(void* K, void* V, int32_t* idx, float* sumsq, const Geom& g, int dtype,
                       const int32_t* start, const int32_t* cur, const int32_t* path, int path_cap,
                       const int32_t* n_path, int32_t* len_out, int per_head, int32_t* status, cudaStream_t s);

// Attention of packed tokens over their caches; mask == nullptr: causal, else the tree form.
struct TokenAttention {
  TokView q, out;
  const int32_t* tok_off;
  int n_tokens;
  Geom g;
  LenView lens;
  int max_len;
  float scale_log2e;
  float* lse;
  const uint32_t* mask;                                  // [n_tokens, 2 * mask_words] 32-bit halves
  int mask_words;
  int32_t* status;                                       // may be null
  PageView pages;                                        // table == nullptr: the cache has rows of its own
};
size_t token_attention_scratch(const Geom& g, int dtype, int n_tokens, int max_len, bool pages);
int launch_token_attention(const TokenAttention& a, const void* K, const void* V, int dtype, char* scratch,
                           size_t scratch_bytes, cudaStream_t s);
// The form for few tokens per sequence of a bf16 cache in pages, where that is the faster one.
bool few_tokens(const TokenAttention& a, int dtype);
size_t few_tokens_scratch(const Geom& g, int max_len);
int launch_few_tokens(const TokenAttention& a, const void* K, const void* V, char* scratch, size_t scratch_bytes, cudaStream_t s);
int launch_token_attention_fp32(const TokenAttention& a, const void* K, const void* V, cudaStream_t s);
// fp32 caches in pages, however many tokens.
size_t few_tokens_fp32_scratch(const Geom& g, int max_len);
int launch_few_tokens_fp32(const TokenAttention& a, const void* K, const void* V, char* scratch, size_t scratch_bytes, cudaStream_t s);

}  // namespace l2kv
