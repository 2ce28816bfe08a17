// What the kernels that rotate and write new tokens' rows share.
#pragma once

#include "tokens.cuh"

namespace l2kv {

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

struct NormRotaryArgs : RotaryArgs { NormArgs norm; };
// Queries and keys in halves, all of a head rotated: the form most models have (norm_rotary.cu).
int launch_norm_rotary_halves(const NormRotaryArgs& a, void* K, void* V, int dtype, cudaStream_t s);

// Two fp32 operations in one instruction, each rounded as by itself.
__device__ __forceinline__ float2 mul_pair(float2 a, float2 b) {
  float2 d;
  asm("{ .reg .b64 x, y, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mul.rn.f32x2 w, x, y; mov.b64 {%0, %1}, w; }"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 add_pair(float2 a, float2 b) {
  float2 d;
  asm("{ .reg .b64 x, y, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 w, x, y; mov.b64 {%0, %1}, w; }"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma_pair(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{ .reg .b64 x, y, z, w; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; "
      "fma.rn.f32x2 w, x, y, z; mov.b64 {%0, %1}, w; }"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

}  // namespace l2kv
