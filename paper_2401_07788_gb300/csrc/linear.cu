// linear.cu -- linear layer with bias, activation, dropout and residual, and its gradient.
//
//   z = x w^T + b;   y = r + drop(act(z))
//   dz = drop(dy) act'(z);   dx = dz w;   dw = dz^T x;   db = sum_rows dz
#include <algorithm>

#include "launch_util.h"
#include "layers.cuh"

namespace mpc {
namespace {

// C[m][n] = sum_k A[m][k] B[n][k] in 64 x 64 tiles, any strides.
struct Product {
  int64_t m, n, k;
  int64_t am, ak, bn, bk;  // strides
};
enum Out { kLayer, kGrad };

template <typename T, int OUT>
__global__ void __launch_bounds__(256)
    linear_tile_kernel(const T* a, const T* b, const Product g, const LinearArgs l, const Drop d, T* c, int64_t ldc) {
  __shared__ float as[16][65], bs[16][65];
  pdl_begin();
  const int64_t m0 = static_cast<int64_t>(blockIdx.x) * 64, n0 = static_cast<int64_t>(blockIdx.y) * 64;
  const int tm = threadIdx.x / 16 * 4, tn = threadIdx.x % 16 * 4;
  float acc[4][4] = {};
  for (int64_t k0 = 0; k0 < g.k; k0 += 16) {
    for (int i = threadIdx.x; i < 1024; i += 256) {
      const int r = i / 16, k = i % 16;
      as[k][r] = m0 + r < g.m && k0 + k < g.k ? as_float(a[(m0 + r) * g.am + (k0 + k) * g.ak]) : 0.0f;
      bs[k][r] = n0 + r < g.n && k0 + k < g.k ? as_float(b[(n0 + r) * g.bn + (k0 + k) * g.bk]) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = __fmaf_rn(as[k][tm + i], bs[k][tn + j], acc[i][j]);
    __syncthreads();
  }
  const uint64_t seed = OUT == kLayer && d.level > 0 ? drop_seed(d) : 0;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + tm + i, n = n0 + tn + j;
      if (m >= g.m || n >= g.n) continue;
      float v = acc[i][j];
      if (OUT == kLayer) {
        if (l.bias != nullptr) v = fadd(v, as_float(static_cast<const T*>(l.bias)[n]));
        if (l.z != nullptr) put(static_cast<T*>(l.z) + m * l.ldz + n, v);
        v = act_value<sizeof(T) == 2>(l.act, v);
        if (d.level > 0) v = kept_at(seed, m * l.out + n, d.level) ? fmul(v, d.scale) : 0.0f;
        if (l.residual != nullptr) v = fadd(v, as_float(static_cast<const T*>(l.residual)[m * l.ldr + n]));
      } else {
        v = fmul(v, d.scale);
      }
      put(c + m * ldc + n, v);
    }
}

// dz without dropout's factor, and its sums over 256 rows.
template <typename T>
__global__ void __launch_bounds__(256) linear_dz_kernel(const LinearArgs l, const Drop d, T* dz, float* part) {
  pdl_begin();
  const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (n >= l.out) return;
  const uint64_t seed = d.level > 0 ? drop_seed(d) : 0;
  float sum = 0.0f;
  const int64_t end = min64(l.rows, (blockIdx.y + int64_t{1}) * 256);
  for (int64_t m = blockIdx.y * int64_t{256}; m < end; ++m) {
    float v = as_float(static_cast<const T*>(l.dy)[m * l.lddy + n]);
    if (d.level > 0 && !kept_at(seed, m * l.out + n, d.level)) v = 0.0f;
    if (l.act != MPC_ACT_NONE) v = fmul(v, act_slope<sizeof(T) == 2>(l.act, as_float(static_cast<const T*>(l.z_in)[m * l.ldz + n])));
    sum = fadd(sum, v);
    put(dz + m * l.out + n, v);
  }
  part[blockIdx.y * l.out + n] = sum;
}
template <typename T>
__global__ void __launch_bounds__(256) linear_dbias_kernel(const float* part, int64_t parts, int64_t out, float scale, T* db) {
  pdl_begin();
  const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (n >= out) return;
  float v = 0.0f;
  for (int64_t p = 0; p < parts; ++p) v = fadd(v, part[p * out + n]);
  put(db + n, fmul(v, scale));
}

template <typename T, int OUT>
cudaError_t product(const T* a, const T* b, const Product& g, const LinearArgs& l, const Drop& d, void* c, int64_t ldc,
                    cudaStream_t s) {
  return launch_kernel(linear_tile_kernel<T, OUT>, dim3(static_cast<unsigned>((g.m + 63) / 64), static_cast<unsigned>((g.n + 63) / 64)),
                       dim3(256), 0, s, 0u, a, b, g, l, d, static_cast<T*>(c), ldc);
}

size_t up(size_t x) { return (x + 255) / 256 * 256; }

template <typename T>
cudaError_t forward(const LinearArgs& a, cudaStream_t s) {
  const Drop d = make_drop(a.p, a.seed, a.step);
  const Product g = {a.rows, a.out, a.in, a.ldx, 1, a.ldw, 1};
  return product<T, kLayer>(static_cast<const T*>(a.x), static_cast<const T*>(a.w), g, a, d, a.y, a.ldy, s);
}

template <typename T>
cudaError_t backward(const LinearArgs& a, cudaStream_t s) {
  const Drop d = make_drop(a.p, a.seed, a.step);
  T* dz = static_cast<T*>(a.ws);
  float* part = reinterpret_cast<float*>(static_cast<char*>(a.ws) + up(a.rows * a.out * sizeof(T)));
  const int64_t parts = (a.rows + 255) / 256;
  cudaError_t e = launch_kernel(linear_dz_kernel<T>, dim3(static_cast<unsigned>((a.out + 255) / 256), static_cast<unsigned>(parts)),
                                dim3(256), 0, s, 0u, a, d, dz, part);
  if (e == cudaSuccess && a.dbias != nullptr)
    e = launch_kernel(linear_dbias_kernel<T>, dim3(static_cast<unsigned>((a.out + 255) / 256)), dim3(256), 0, s, 0u,
                      static_cast<const float*>(part), parts, a.out, d.scale, static_cast<T*>(a.dbias));
  if (e == cudaSuccess && a.dx != nullptr)
    e = product<T, kGrad>(dz, static_cast<const T*>(a.w), Product{a.rows, a.in, a.out, a.out, 1, 1, a.ldw}, a, d, a.dx, a.lddx, s);
  if (e == cudaSuccess && a.dw != nullptr)
    e = product<T, kGrad>(dz, static_cast<const T*>(a.x), Product{a.out, a.in, a.rows, 1, a.out, 1, a.ldx}, a, d, a.dw, a.lddw, s);
  return e;
}

}  // namespace

size_t linear_workspace_bytes(int64_t rows, int64_t, int64_t out, int bf16, int pass, int64_t, int64_t, int64_t) {
  if (pass == MPC_LINEAR_FORWARD) return 0;
  return up(rows * out * (bf16 ? 2 : 4)) + up((rows + 255) / 256 * out * 4);
}
cudaError_t launch_linear_forward(const LinearArgs& a, int, cudaStream_t s) {
  return a.bf16 ? forward<__nv_bfloat16>(a, s) : forward<float>(a, s);
}
cudaError_t launch_linear_backward(const LinearArgs& a, int, cudaStream_t s) {
  return a.bf16 ? backward<__nv_bfloat16>(a, s) : backward<float>(a, s);
}

}  // namespace mpc
