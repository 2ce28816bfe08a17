// The tensor map of packed new tokens' queries, and the shared-memory matrix loads of the kernels that read them.
#pragma once

#include "async_copy.cuh"
#include "tokens.cuh"

namespace l2kv {

// Rank-4 map of the queries (head_dim, head, token, layer); a box is 64 elements of the heads of a group, of box_tokens tokens.
inline bool make_query_map(CUtensorMap* map, const TokenAttention& a, int box_tokens) {
  const Geom& g = a.g;
  const int G = g.Hq / g.H;
  const long long tight = g.D;
  const cuuint64_t dims[4] = {(cuuint64_t)g.D, (cuuint64_t)g.Hq, (cuuint64_t)a.n_tokens, (cuuint64_t)g.L};
  const cuuint64_t strides[3] = {(cuuint64_t)(g.Hq > 1 ? a.q.sh : tight) * 2, (cuuint64_t)(a.n_tokens > 1 ? a.q.st : tight) * 2,
                                 (cuuint64_t)(g.L > 1 ? a.q.sl : tight) * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)G, (cuuint32_t)box_tokens, 1};
  return encode_bf16_map(map, 4, a.q.p, dims, strides, box);
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1,
                                            int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
               "[%0], [%1, {%3, %4, %5, %6}], [%2];"
               :: "r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
               : "memory");
}

}  // namespace l2kv
