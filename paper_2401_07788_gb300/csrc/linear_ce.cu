// linear_ce.cu -- softmax cross entropy of a linear head over a large
// vocabulary, with its gradient, in pieces of the vocabulary: the logits are
// never kept.
//
//   l[t][v] = <h[t], w[v]>            t over the tokens whose target counts
//   lse[t]  = log sum_v exp l[t][v];  loss[t] = lse[t] - l[t][target[t]]
//   c[t][v] = g[t] (exp(l[t][v] - lse[t]) - [v == target[t]])
//   dh = c w;   dw = c^T h
//
// Tokens that do not count (target == ignore_index) are left out from the start:
// a scan of the targets lists the others, and every kernel below works on that
// list, whose length stays on the device.  Whatever their hidden states hold
// (padding is often NaN) reaches nothing.
#include <algorithm>
#include <cuda_bf16.h>

#include "common.cuh"
#include "kernels.h"
#include "launch_util.h"

namespace mpc {
namespace {

constexpr int kTile = 64;   // tokens and vocabulary entries of a logit tile
constexpr int kStep = 16;
constexpr int kGemmThreads = 256;

struct Header {
  int valid;  // tokens that count
  float mean; // 1 / valid (0 when none counts)
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float x, float* p) { *p = x; }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16* p) { *p = __float2bfloat16_rn(x); }

// ---------------------------------------------------------------------------
// The list of tokens that count: row[i] = token, target[i], and place[t] = i
// (-1 for the others), in token order; one CTA.  A target outside [0, V) that is
// not ignore_index is reported and left out too.
// ---------------------------------------------------------------------------
__global__ void __launch_bounds__(1024)
    ce_scan_kernel(const int64_t* __restrict__ targets, int T, int64_t V, int64_t ignore,
                   Header* head, int* row, int* target, int* place, unsigned* status) {
  pdl_begin();
  __shared__ int warp_count[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int base = 0;
  for (int t0 = 0; t0 < T; t0 += 1024) {
    const int t = t0 + threadIdx.x;
    bool keep = false;
    int64_t y = 0;
    if (t < T) {
      y = targets[t];
      keep = y != ignore;
      if (keep && (y < 0 || y >= V)) {
        set_status(status, STATUS_BAD_INDEX);
        keep = false;
      }
    }
    const unsigned b = __ballot_sync(kFull, keep);
    if (lane == 0) warp_count[warp] = __popc(b);
    __syncthreads();
    int before = base, total = 0;
    for (int w = 0; w < 32; ++w) {
      if (w < warp) before += warp_count[w];
      total += warp_count[w];
    }
    const int i = before + __popc(b & lanemask_lt());
    if (t < T) place[t] = keep ? i : -1;
    if (keep) {
      row[i] = t;
      target[i] = static_cast<int>(y);
    }
    base += total;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    head->valid = base;
    head->mean = base > 0 ? fdiv(1.0f, static_cast<float>(base)) : 0.0f;
  }
}

// ---------------------------------------------------------------------------
// C[m][n] = sum_k A(m, k) B(n, k), one 64 x 64 tile a CTA, fp32.
// ---------------------------------------------------------------------------
template <class A, class B>
__device__ __forceinline__ void tile_product(const A& a, const B& b, int m0, int n0, int64_t K,
                                             float (&acc)[4][4]) {
  __shared__ float sa[kStep][kTile + 4], sb[kStep][kTile + 4];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
  for (int64_t k0 = 0; k0 < K; k0 += kStep) {
    for (int q = threadIdx.x; q < kTile * kStep; q += kGemmThreads) {
      const int r = q / kStep, k = q % kStep;
      sa[k][r] = k0 + k < K ? a(m0 + r, k0 + k) : 0.0f;
      sb[k][r] = k0 + k < K ? b(n0 + r, k0 + k) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kStep; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __fmaf_rn(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
}

struct Ce {
  const void* h;
  const void* w;
  int64_t ldh, ldw;
  int T;
  int64_t D, V;
  const Header* head;
  const int* row;
  const int* target;
  const int* place;
};

// Logits of a tile: each token's largest, the sum of exponentials over it, and
// the target's logit.  part[tile][i] = (largest, sum).
template <typename E>
__global__ void __launch_bounds__(kGemmThreads)
    ce_logits_kernel(const Ce c, float2* part, float* at_target) {
  pdl_begin();
  const int valid = c.head->valid;
  const int m0 = blockIdx.x * kTile;
  const int n0 = blockIdx.y * kTile;
  if (m0 >= valid) return;
  const E* h = static_cast<const E*>(c.h);
  const E* w = static_cast<const E*>(c.w);
  float acc[4][4];
  tile_product([&](int m, int64_t k) { return m < valid ? to_float(h[c.row[m] * c.ldh + k]) : 0.0f; },
               [&](int n, int64_t k) { return n < c.V ? to_float(w[n * c.ldw + k]) : 0.0f; },
               m0, n0, c.D, acc);
  __shared__ float s[kTile][kTile + 1];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) s[ty * 4 + i][tx * 4 + j] = acc[i][j];
  __syncthreads();
  const int m = m0 + threadIdx.x;
  if (threadIdx.x < kTile && m < valid) {
    const int n = static_cast<int>(min64(c.V - n0, kTile));
    const float* x = s[threadIdx.x];
    float top = -INFINITY, sum = 0.0f;
    for (int j = 0; j < n; ++j) top = fmaxf(top, x[j]);
    for (int j = 0; j < n; ++j) sum += expf(x[j] - top);
    part[static_cast<int64_t>(blockIdx.y) * c.T + m] = make_float2(top, sum);
    const int y = c.target[m] - n0;
    if (y >= 0 && y < n) at_target[m] = x[y];
  }
}

// lse and loss of each token from the tiles' sums; one warp a token.
__global__ void __launch_bounds__(256)
    ce_finish_kernel(const Ce c, const float2* part, int tiles, const float* at_target, float* loss,
                     float* lse) {
  pdl_begin();
  const int t = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (t >= c.T) return;
  const int m = c.place[t];
  if (m < 0) {
    if (lane == 0) loss[t] = lse[t] = 0.0f;
    return;
  }
  float top = -INFINITY;
  for (int i = lane; i < tiles; i += 32) top = fmaxf(top, part[static_cast<int64_t>(i) * c.T + m].x);
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
  float sum = 0.0f;
  for (int i = lane; i < tiles; i += 32) {
    const float2 p = part[static_cast<int64_t>(i) * c.T + m];
    sum += p.y * expf(p.x - top);
  }
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
  if (lane == 0) {
    const float l = top + logf(sum);
    lse[t] = l;
    loss[t] = l - at_target[m];
  }
}

// Coefficients c[t][v] of vocabulary entries v0.. of a piece (fp32 [valid][width]).
template <typename E>
__global__ void __launch_bounds__(kGemmThreads)
    ce_coefficients_kernel(const Ce c, const float* lse, const float* gloss, int64_t v0, int width,
                           float* coef) {
  pdl_begin();
  const int valid = c.head->valid;
  const int m0 = blockIdx.x * kTile;
  const int n0 = blockIdx.y * kTile;
  if (m0 >= valid) return;
  const E* h = static_cast<const E*>(c.h);
  const E* w = static_cast<const E*>(c.w);
  float acc[4][4];
  tile_product([&](int m, int64_t k) { return m < valid ? to_float(h[c.row[m] * c.ldh + k]) : 0.0f; },
               [&](int n, int64_t k) { return n < width ? to_float(w[(v0 + n) * c.ldw + k]) : 0.0f; },
               m0, n0, c.D, acc);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + ty * 4 + i;
    if (m >= valid) continue;
    const int t = c.row[m];
    const float g = gloss != nullptr ? gloss[t] : c.head->mean;
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + tx * 4 + j;
      if (n >= width) continue;
      const float p = expf(acc[i][j] - lse[t]);
      coef[static_cast<int64_t>(m) * width + n] = g * (v0 + n == c.target[m] ? p - 1.0f : p);
    }
  }
}

// dh of the piece added up in fp32 (first: the piece that starts the sum).
template <typename E>
__global__ void __launch_bounds__(kGemmThreads)
    ce_dh_kernel(const Ce c, const float* coef, int64_t v0, int width, int first, float* sum) {
  pdl_begin();
  const int valid = c.head->valid;
  const int m0 = blockIdx.x * kTile, n0 = blockIdx.y * kTile;
  if (m0 >= valid) return;
  const E* w = static_cast<const E*>(c.w);
  float acc[4][4];
  tile_product([&](int m, int64_t k) { return m < valid ? coef[static_cast<int64_t>(m) * width + k] : 0.0f; },
               [&](int n, int64_t k) { return n < c.D ? to_float(w[(v0 + k) * c.ldw + n]) : 0.0f; },
               m0, n0, width, acc);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m >= valid || n >= c.D) continue;
      float* s = sum + m * c.D + n;
      *s = first ? acc[i][j] : *s + acc[i][j];
    }
}

// dh in the caller's type and order; zero for tokens that do not count.
template <typename E>
__global__ void __launch_bounds__(256)
    ce_dh_out_kernel(const Ce c, const float* sum, E* dh, int64_t lddh) {
  pdl_begin();
  for (int t = blockIdx.x; t < c.T; t += gridDim.x) {
    const int m = c.place[t];
    for (int64_t d = threadIdx.x; d < c.D; d += blockDim.x)
      from_float(m < 0 ? 0.0f : sum[m * c.D + d], dh + t * lddh + d);
  }
}

template <typename E>
__global__ void __launch_bounds__(kGemmThreads)
    ce_dw_kernel(const Ce c, const float* coef, int64_t v0, int width, E* dw, int64_t lddw) {
  pdl_begin();
  const int valid = c.head->valid;
  const int m0 = blockIdx.x * kTile, n0 = blockIdx.y * kTile;
  const E* h = static_cast<const E*>(c.h);
  float acc[4][4];
  tile_product([&](int m, int64_t k) { return m < width ? coef[k * width + m] : 0.0f; },
               [&](int n, int64_t k) { return n < c.D ? to_float(h[c.row[k] * c.ldh + n]) : 0.0f; },
               m0, n0, valid, acc);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty * 4 + i, n = n0 + tx * 4 + j;
      if (m < width && n < c.D) from_float(acc[i][j], dw + (v0 + m) * lddw + n);
    }
}

// ---------------------------------------------------------------------------
// Workspace
// ---------------------------------------------------------------------------
size_t up(size_t x) { return (x + 255) / 256 * 256; }

struct Layout {
  size_t head, row, target, place, at_target, part, lse, coef, sum, total;
  int tiles;
  int64_t piece;
};

Layout layout(int64_t T, int64_t D, int64_t V, bool grad, int64_t piece) {
  Layout l = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t p = at;
    at += up(bytes);
    return p;
  };
  l.tiles = static_cast<int>((V + kTile - 1) / kTile);
  l.head = take(sizeof(Header));
  l.row = take(T * 4);
  l.target = take(T * 4);
  l.place = take(T * 4);
  l.at_target = take(T * 4);
  l.lse = take(T * 4);
  l.part = take(static_cast<size_t>(l.tiles) * T * 8);
  if (grad) {
    const int64_t most = std::max<int64_t>(kTile, (int64_t{1} << 28) / T / kTile * kTile);
    l.piece = std::min(V, piece > 0 ? piece : most);
    l.coef = take(static_cast<size_t>(T) * l.piece * 4);
    l.sum = take(static_cast<size_t>(T) * D * 4);
  }
  l.total = at;
  return l;
}

template <typename E>
cudaError_t run(const LinearCeArgs& a, cudaStream_t s) {
  const int T = static_cast<int>(a.T);
  const Layout l = layout(a.T, a.D, a.V, a.dw != nullptr, a.piece);
  char* ws = static_cast<char*>(a.ws);
  Ce c = {a.h, a.w, a.ldh, a.ldw, T, a.D, a.V, reinterpret_cast<Header*>(ws + l.head),
          reinterpret_cast<int*>(ws + l.row), reinterpret_cast<int*>(ws + l.target),
          reinterpret_cast<int*>(ws + l.place)};
  float* at_target = reinterpret_cast<float*>(ws + l.at_target);
  float2* part = reinterpret_cast<float2*>(ws + l.part);
  cudaError_t e = launch_kernel(ce_scan_kernel, dim3(1), dim3(1024), 0, s, 0, a.targets, T, a.V, a.ignore,
                                const_cast<Header*>(c.head), const_cast<int*>(c.row),
                                const_cast<int*>(c.target), const_cast<int*>(c.place), a.status);
  if (e != cudaSuccess) return e;
  const unsigned mt = static_cast<unsigned>((a.T + kTile - 1) / kTile);
  const unsigned dt = static_cast<unsigned>((a.D + kTile - 1) / kTile);
  const float* lse = a.lse_in;
  if (a.loss != nullptr) {
    float* out = a.lse != nullptr ? a.lse : reinterpret_cast<float*>(ws + l.lse);
    e = launch_kernel(ce_logits_kernel<E>, dim3(mt, l.tiles), dim3(kGemmThreads), 0, s, 0, c, part, at_target);
    if (e != cudaSuccess) return e;
    e = launch_kernel(ce_finish_kernel, dim3((T + 7) / 8), dim3(256), 0, s, 0, c, part, l.tiles, at_target,
                      a.loss, out);
    if (e != cudaSuccess) return e;
    lse = out;
  }
  if (a.dw == nullptr) return cudaSuccess;
  float* coef = reinterpret_cast<float*>(ws + l.coef);
  float* sum = reinterpret_cast<float*>(ws + l.sum);
  for (int64_t v0 = 0; v0 < a.V; v0 += l.piece) {
    const int width = static_cast<int>(std::min(l.piece, a.V - v0));
    const unsigned vt = static_cast<unsigned>((width + kTile - 1) / kTile);
    e = launch_kernel(ce_coefficients_kernel<E>, dim3(mt, vt), dim3(kGemmThreads), 0, s, 0, c, lse, a.gloss,
                      v0, width, coef);
    if (e != cudaSuccess) return e;
    e = launch_kernel(ce_dh_kernel<E>, dim3(mt, dt), dim3(kGemmThreads), 0, s, 0, c, coef, v0, width,
                      static_cast<int>(v0 == 0), sum);
    if (e != cudaSuccess) return e;
    e = launch_kernel(ce_dw_kernel<E>, dim3(vt, dt), dim3(kGemmThreads), 0, s, 0, c, coef, v0, width,
                      static_cast<E*>(a.dw), a.lddw);
    if (e != cudaSuccess) return e;
  }
  return launch_kernel(ce_dh_out_kernel<E>, dim3(static_cast<unsigned>(std::min<int64_t>(a.T, 4096))), dim3(256),
                       0, s, 0, c, sum, static_cast<E*>(a.dh), a.lddh);
}

}  // namespace

size_t linear_ce_workspace_bytes(int64_t T, int64_t D, int64_t V, int bf16, int grad, int64_t piece) {
  return layout(T, D, V, grad != 0, piece).total;
}

cudaError_t launch_linear_ce(const LinearCeArgs& a, int num_sms, cudaStream_t s) {
  return a.bf16 ? run<__nv_bfloat16>(a, s) : run<float>(a, s);
}

}  // namespace mpc
