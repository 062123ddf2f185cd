// layers.cuh -- what the kernels of a stage's layers share: element types, 16-byte
// accesses, the dropout generator.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"
#include "kernels.h"

namespace mpc {

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Elements of 16 bytes, as they lie in memory and as floats.
template <typename T>
constexpr int kVec = 16 / static_cast<int>(sizeof(T));

__device__ __forceinline__ void unpack16(const uint4& u, float (&x)[4]) {
  x[0] = __uint_as_float(u.x);
  x[1] = __uint_as_float(u.y);
  x[2] = __uint_as_float(u.z);
  x[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack16(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack16(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  uint32_t u;
  memcpy(&u, &p, 4);
  return u;
}
__device__ __forceinline__ uint4 pack16(const float (&x)[8]) {
  return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
}

// ---------------------------------------------------------------------------
// Activations and their derivatives, with one exponential each:
//   Phi(z) = (1 + erf(z / sqrt 2)) / 2,          gelu = z Phi,  gelu' = Phi + z phi(z)
//   s = 1 / (1 + exp(-v)),                     silu = z s(z)
//   (1 + tanh(v / 2)) / 2 = s(v),              gelu_tanh = z s(2 sqrt(2/pi) (z + 0.044715 z^3))
// For bf16 results the exponential and the quotient are the approximate ones (2 ulp),
// and 1 - erf is formula 7.1.26 of Abramowitz and Stegun (1.5e-7 off at most).
// ---------------------------------------------------------------------------
// 2^x and 1 / x, approximate (2 ulp), subnormal numbers as 0: one instruction each.
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float inverse_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2E = 1.4426950408889634f;
// s(v); fast: from -v log2 e.
__device__ __forceinline__ float sigmoid(float v) { return fdiv(1.0f, fadd(1.0f, expf(-v))); }
__device__ __forceinline__ float sigmoid_fast(float minus_log2) { return inverse_fast(fadd(1.0f, exp2_fast(minus_log2))); }
// Phi(z); fast: with e = exp(-z^2 / 2).
__device__ __forceinline__ float normal_cdf(float z) { return fmul(0.5f, fadd(1.0f, erff(fmul(z, 0.70710678118654752f)))); }  // 6e-8 off at most
__device__ __forceinline__ float normal_cdf_fast(float z, float e) {
  const float t = inverse_fast(__fmaf_rn(fabsf(z), 0.3275911f * 0.70710678118654752f, 1.0f));
  float q = __fmaf_rn(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f);
  q = __fmaf_rn(t, q, 0.5f * 1.421413741f);
  q = __fmaf_rn(t, q, 0.5f * -0.284496736f);
  q = __fmaf_rn(t, q, 0.5f * 0.254829592f);
  q = fmul(fmul(t, q), e);  // Phi(-|z|)
  return z < 0.0f ? q : fsub(1.0f, q);
}
__device__ __forceinline__ float bell_fast(float z) { return exp2_fast(fmul(fmul(z, z), -0.5f * kLog2E)); }
constexpr float kTanhIn = 1.5957691216057308f;  // 2 sqrt(2/pi)
template <bool FAST>
__device__ __forceinline__ float act_value(int act, float z) {
  switch (act) {
    case MPC_ACT_RELU: return z > 0.0f ? z : z != z ? z : 0.0f;
    case MPC_ACT_GELU: return fmul(z, FAST ? normal_cdf_fast(z, bell_fast(z)) : normal_cdf(z));
    case MPC_ACT_GELU_TANH: {
      const float zz = fmul(z, z);
      if (FAST) return fmul(z, sigmoid_fast(fmul(z, __fmaf_rn(zz, -kTanhIn * kLog2E * 0.044715f, -kTanhIn * kLog2E))));
      return fmul(z, sigmoid(fmul(fmul(z, kTanhIn), __fmaf_rn(zz, 0.044715f, 1.0f))));
    }
    case MPC_ACT_SILU: return fmul(z, FAST ? sigmoid_fast(fmul(z, -kLog2E)) : sigmoid(z));
    default: return z;
  }
}
template <bool FAST>
__device__ __forceinline__ float act_slope(int act, float z) {
  if (fabsf(z) > 100.0f) z = copysignf(100.0f, z);  // where every slope is its limit: no infinity times zero
  switch (act) {
    case MPC_ACT_RELU: return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
    case MPC_ACT_GELU: {
      const float e = FAST ? bell_fast(z) : expf(fmul(fmul(z, z), -0.5f));
      return __fmaf_rn(fmul(z, 0.3989422804014327f), e, FAST ? normal_cdf_fast(z, e) : normal_cdf(z));
    }
    case MPC_ACT_GELU_TANH: {
      const float zz = fmul(z, z);
      const float s = FAST ? sigmoid_fast(fmul(z, __fmaf_rn(zz, -kTanhIn * kLog2E * 0.044715f, -kTanhIn * kLog2E)))
                           : sigmoid(fmul(fmul(z, kTanhIn), __fmaf_rn(zz, 0.044715f, 1.0f)));
      // s + z s (1 - s) dv/dz
      const float dv = __fmaf_rn(zz, kTanhIn * 3.0f * 0.044715f, kTanhIn);
      return __fmaf_rn(fmul(z, dv), fmul(s, fsub(1.0f, s)), s);
    }
    case MPC_ACT_SILU: {
      const float s = FAST ? sigmoid_fast(fmul(z, -kLog2E)) : sigmoid(z);
      return fmul(s, __fmaf_rn(z, fsub(1.0f, s), 1.0f));
    }
    default: return 1.0f;
  }
}

// Dropout: entry i takes 16 bits of splitmix64 at counter i / 4 and is dropped where
// they are below `level` (65536 drops everything), else multiplied by `scale`.  16 bits
// an entry: the generator costs 20 instructions a draw, so four entries share one; p is
// met to 2^-17, and the factor is that of the p which is met.
struct Drop {
  uint64_t seed;
  const int64_t* step;  // device, or nullptr
  uint32_t level;       // 0: nothing is dropped
  float scale;
};
inline Drop make_drop(double p, uint64_t seed, const int64_t* step) {
  Drop d;
  d.seed = seed;
  d.step = step;
  d.level = static_cast<uint32_t>(p * 65536.0 + 0.5);
  d.scale = d.level < 65536 ? static_cast<float>(65536.0 / (65536.0 - d.level)) : 0.0f;
  return d;
}
__device__ __forceinline__ uint64_t drop_seed(const Drop& d) {
  return d.seed + (d.step != nullptr ? static_cast<uint64_t>(*d.step) : 0ull);
}
// Draws of neighbouring counters: the state of one is the last one's plus a constant.
struct Draws {
  uint64_t state;
  __device__ __forceinline__ Draws(uint64_t seed, uint64_t counter) : state(seed + counter * kSplitmixStep) {}
  __device__ __forceinline__ uint64_t next() { return splitmix64_of(state += kSplitmixStep); }
};
// Whether part q (0..3) of a draw keeps its entry.
__device__ __forceinline__ bool kept(uint64_t z, int q, uint32_t level) {
  const uint32_t w = static_cast<uint32_t>(q < 2 ? z : z >> 32);
  return (q & 1 ? w >> 16 : w & 0xffffu) >= level;
}
// The same of one entry by its number.
__device__ __forceinline__ bool kept_at(uint64_t seed, uint64_t i, uint32_t level) {
  return kept(splitmix64_at(seed, i >> 2), static_cast<int>(i & 3), level);
}

}  // namespace mpc
