// dropout.cu -- y = residual + drop(x) with a mask that is made where it is used and
// never stored, from splitmix64 at the entry's number (layers.cuh).
//
// What bounds it: HBM.  A draw (20 instructions) serves four entries, so an entry of bf16 costs 9
// instructions of the 23 that an SM has for the 4 bytes it moves.  Four 16-byte groups a thread
// keep enough bytes in flight.  Measured: 16384 x 4096 in fp32 with residual 107 us, without 75
// (7.5 and 7.2 TB/s: the last 120 MB are still in L2), both 190.6 us among others (7.04 TB/s); in bf16
// 57 us and 40 (7.0 and 6.8 TB/s).
#include "launch_util.h"
#include "layers.cuh"

namespace mpc {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // 16-byte groups a thread has in flight

template <bool RES>
__device__ __forceinline__ float dropped(float x, float r, bool keep, float scale) {
  const float v = keep ? fmul(x, scale) : 0.0f;
  return RES ? fadd(r, v) : v;
}

// 16-byte groups; the last n % (16 / sizeof(T)) entries by the last CTA's first threads.
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads)
    dropout_kernel(const T* x, const T* res, int64_t n, Drop d, T* y) {
  constexpr int V = kVec<T>;
  pdl_begin();
  pdl_end();
  const uint64_t seed = drop_seed(d);
  const int64_t groups = n / V;
  const int64_t g0 = static_cast<int64_t>(blockIdx.x) * (kThreads * kUnroll) + threadIdx.x;
  uint4 a[kUnroll], b[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t g = g0 + u * kThreads;
    if (g < groups) {
      a[u] = reinterpret_cast<const uint4*>(x)[g];
      if (RES) b[u] = reinterpret_cast<const uint4*>(res)[g];
    }
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int64_t g = g0 + u * kThreads;
    if (g < groups) {
      float v[V], r[V];
      unpack16(a[u], v);
      if (RES) unpack16(b[u], r);
#pragma unroll
      for (int q = 0; q < V; q += 4) {
        const uint64_t z = splitmix64_at(seed, static_cast<uint64_t>(g) * (V / 4) + q / 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[q + k] = dropped<RES>(v[q + k], RES ? r[q + k] : 0.0f, kept(z, k, d.level), d.scale);
      }
      reinterpret_cast<uint4*>(y)[g] = pack16(v);
    }
  }
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x < n - groups * V) {
    const int64_t i = groups * V + threadIdx.x;
    put(y + i, dropped<RES>(as_float(x[i]), RES ? as_float(res[i]) : 0.0f, kept_at(seed, i, d.level), d.scale));
  }
}

// Any alignment: one draw's four entries a thread.
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads)
    dropout_any_kernel(const T* x, const T* res, int64_t n, Drop d, T* y) {
  pdl_begin();
  pdl_end();
  const int64_t g = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (g * 4 >= n) return;
  const uint64_t z = splitmix64_at(drop_seed(d), g);
  float v[4], r[4];
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (g * 4 + k < n) {
      v[k] = as_float(x[g * 4 + k]);
      r[k] = RES ? as_float(res[g * 4 + k]) : 0.0f;
    }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (g * 4 + k < n) put(y + g * 4 + k, dropped<RES>(v[k], r[k], kept(z, k, d.level), d.scale));
}

template <typename T, bool RES>
cudaError_t launch(const DropoutArgs& a, const Drop& d, cudaStream_t s) {
  const T* x = static_cast<const T*>(a.x);
  const T* r = static_cast<const T*>(a.residual);
  T* y = static_cast<T*>(a.y);
  const bool wide = ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(r) | reinterpret_cast<uintptr_t>(y)) & 15) == 0;
  const int64_t each = wide ? kThreads * kUnroll * kVec<T> : kThreads * 4;
  const int64_t grid = (a.n + each - 1) / each;
  if (grid > 0x7fffffff) return cudaErrorInvalidValue;
  return launch_kernel(wide ? dropout_kernel<T, RES> : dropout_any_kernel<T, RES>, dim3(static_cast<unsigned>(grid)),
                       dim3(kThreads), 0, s, 0u, x, r, a.n, d, y);
}

}  // namespace

cudaError_t launch_dropout(const DropoutArgs& a, cudaStream_t s) {
  const Drop d = make_drop(a.p, a.seed, a.step);
  if (a.bf16) return a.residual ? launch<__nv_bfloat16, true>(a, d, s) : launch<__nv_bfloat16, false>(a, d, s);
  return a.residual ? launch<float, true>(a, d, s) : launch<float, false>(a, d, s);
}

}  // namespace mpc
