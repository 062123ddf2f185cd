// linear_ce_few.cu -- the linear cross entropy of a few tokens (32 at most): a
// scored token of a served model, the last tokens of a batch.
//
// With so few tokens the work is one pass over w (and one over dw): T products a
// byte pair of w, under the fp32 rate of the SMs, so plain fp32 FMAs read w once at
// the memory's rate, where tiles of the matrix units would be empty rows for the
// most part (and an fp32 w would first be split into bf16 planes, 2.5 times its
// size of traffic).
//
//   ce_few_logits   a warp takes R rows of w at a time, its lanes the columns: T R
//                   sums a lane, added up over the lanes by halving exchanges, then
//                   a running (largest, sum of exponentials) for each token
//   ce_few_finish   lse and loss
//   ce_few_grad     one pass over w and dw: c of 64 rows at a time in shared
//                   memory, a thread owns a few columns, with h and the sums of dh
//                   of each token for them in registers
//   ce_few_dh       dh from the CTAs' sums
//
// Measured with w in HBM, bf16, both kernels of a call: one token x 4096 x 131072 169
// us (6.3 TB/s); x 768 x 50257 24 us, of which about 12 are start, staging of h, the
// last rows and the second launch.  With 16 tokens the FMAs show: 72 us for an fp32 w
// of 154 MB.  Rows of w off 16 bytes cost 4 to 6 us more on 77 MB.  The gradient adds
// 28 us to one token x 768 x 50257 (154 MB of w and dw, 5.4 TB/s).
//
// Tokens keep their places here; one that does not count has a zero row of h, and
// zero results.
#include <algorithm>
#include <type_traits>
#include <cuda_bf16.h>

#include "common.cuh"
#include "kernels.h"
#include "launch_util.h"

namespace mpc {
namespace {

constexpr int kFewTokens = 32;  // of a call; of a gradient, and of a pass over w, 16
constexpr int kFewGroup = 16;
constexpr int kFewThreads = 512;
constexpr int kFewWarps = kFewThreads / 32;
constexpr int kFewBytes = 200 * 1024;  // of h in fp32 in shared memory
constexpr float kL2e = 1.4426950408889634f;
constexpr float kL2 = 0.6931471805599453f;

__device__ __forceinline__ float few_float(float x) { return x; }
__device__ __forceinline__ float few_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void few_from(float x, float* p) { *p = x; }
__device__ __forceinline__ void few_from(float x, __nv_bfloat16* p) { *p = __float2bfloat16_rn(x); }

struct Few {
  const void* h;
  const void* w;
  int64_t ldh, ldw;
  const int64_t* targets;
  int T, D;
  int64_t V, ignore;
  float2* part;    // [CTA][kFewTokens] (largest logit, sum), base 2
  float* at;       // [kFewTokens] the target's logit
  float* logits;   // [T][V] for the gradient, or nullptr
  float* lse;      // [T]
  float* loss;     // [T], or nullptr
  const float* gloss;
  float* weight;   // [kFewTokens] g, 0 for tokens that do not count
  float* sums;     // [CTA][T][D] of dh
  void* dh;
  void* dw;
  int64_t lddh, lddw;
  int parts;
  unsigned* status;
};

__device__ __forceinline__ int few_target(const Few& f, int t) {
  if (t >= f.T) return -1;
  const int64_t y = f.targets[t];
  return y != f.ignore && y >= 0 && y < f.V ? static_cast<int>(y) : -1;
}

// V elements from p on as floats.
template <int N>
__device__ __forceinline__ void few_load(const float* p, float (&x)[N]) {
  if (N == 1) {
    x[0] = p[0];
    return;
  }
  if (N == 2) {
    const float2 v = *reinterpret_cast<const float2*>(p);
    x[0] = v.x; x[1] = v.y;
    return;
  }
#pragma unroll
  for (int j = 0; j + 4 <= N; j += 4) {
    const float4 v = *reinterpret_cast<const float4*>(p + j);
    x[j] = v.x; x[j + 1] = v.y; x[j + 2] = v.z; x[j + 3] = v.w;
  }
}
template <int N>
__device__ __forceinline__ void few_load(const __nv_bfloat16* p, float (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = __bfloat162float(p[0]);
  } else {
  uint32_t u[N / 2];
  if (N == 8) *reinterpret_cast<uint4*>(u) = *reinterpret_cast<const uint4*>(p);
  else if (N == 4) *reinterpret_cast<uint2*>(u) = *reinterpret_cast<const uint2*>(p);
  else u[0] = *reinterpret_cast<const uint32_t*>(p);
#pragma unroll
  for (int j = 0; j < N / 2; ++j) {
    x[2 * j] = __uint_as_float(u[j] << 16);
    x[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
  }
  }
}

// The rows of h of TT tokens in shared memory, fp32.  Columns of a 16-byte group
// of 8 bf16 are kept in two halves of 4, so that 128-bit reads of neighbouring
// lanes do not meet in a bank.
template <typename E, int W>
__device__ __forceinline__ int few_place(int d, int Dp) {
  if (W * sizeof(E) < 16 || sizeof(E) == 4) return d;
  return (d >> 2 & 1) * (Dp / 2) + (d >> 3) * 4 + (d & 3);
}

// W elements of w an access: 16 bytes where its rows start on 16, else pairs of
// bf16 where they start on 4, else one element; neighbouring lanes neighbouring
// accesses.  Tokens t0 .. t0 + TT - 1.
template <typename E, int TT, int W>
__global__ void __launch_bounds__(kFewThreads, 1) ce_few_logits_kernel(const Few f, int t0) {
  constexpr int VEC = W;
  constexpr bool WIDE = W * sizeof(E) == 16;
  constexpr int R = TT == 1 ? 8 : 4;  // rows a warp takes at a time
  constexpr int N = R * TT;
  pdl_begin();
  extern __shared__ float sh[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int Dp = (f.D + 7) / 8 * 8;
  const E* h = static_cast<const E*>(f.h);
  const E* w = static_cast<const E*>(f.w);
  // 16-byte reads run one step (of 32 groups of a warp's rows) ahead of the products,
  // into the next rows where these end, the first one before h is staged
  const int64_t groups = (f.V + R - 1) / R, stride = static_cast<int64_t>(gridDim.x) * kFewWarps;
  const int64_t g0 = blockIdx.x * kFewWarps + warp;
  const int whole = f.D / VEC * VEC;
  uint4 ahead[WIDE ? R : 1];
  auto read = [&](int64_t g, int d) {
    if (g < groups && d < whole) {
#pragma unroll
      for (int r = 0; r < (WIDE ? R : 1); ++r)
        ahead[r] = *reinterpret_cast<const uint4*>(w + min64(g * R + r, f.V - 1) * f.ldw + d);
    } else {
#pragma unroll
      for (int r = 0; r < (WIDE ? R : 1); ++r) ahead[r] = make_uint4(0, 0, 0, 0);
    }
  };
  if constexpr (WIDE) read(g0, lane * VEC);
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const bool live = few_target(f, t0 + t) >= 0;
    for (int d = threadIdx.x; d < Dp; d += kFewThreads)
      sh[t * Dp + few_place<E, W>(d, Dp)] = live && d < f.D ? few_float(h[(t0 + t) * f.ldh + d]) : 0.0f;
  }
  if (blockIdx.x == 0 && t0 == 0 && threadIdx.x < f.T) {
    const int64_t y = f.targets[threadIdx.x];
    if (y != f.ignore && (y < 0 || y >= f.V)) set_status(f.status, STATUS_BAD_INDEX);
  }
  __syncthreads();

  // this lane's sums after the exchange: indices idx .. idx + C - 1 of r * TT + t
  constexpr int C = N > 32 ? N / 32 : 1;
  int idx = 0;
  bool counts = true;  // the one lane of those that hold the same sum
  {
    int c = N;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      if (c > 1) {
        c /= 2;
        if (lane & o) idx += c;
      } else if (lane & o) {
        counts = false;
      }
    }
  }
  float top[C], sum[C];
  int target[C];
#pragma unroll
  for (int i = 0; i < C; ++i) {
    top[i] = -INFINITY;
    sum[i] = 0.0f;
    target[i] = few_target(f, t0 + (idx + i) % TT);
  }
  for (int64_t g = g0; g < groups; g += stride) {
    const int64_t v0 = g * R;
    float acc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = 0.0f;
    const E* rows[R];  // (dead in the first form but for the columns after the last whole group)
#pragma unroll
    for (int r = 0; r < R; ++r) rows[r] = w + min64(v0 + r, f.V - 1) * f.ldw;
    if constexpr (WIDE) {
      for (int d = lane * VEC; d - lane * VEC < whole; d += 32 * VEC) {
        uint4 u[R];
#pragma unroll
        for (int r = 0; r < R; ++r) u[r] = ahead[r];
        if (d - lane * VEC + 32 * VEC < whole) read(g, d + 32 * VEC);
        else read(g + stride, lane * VEC);
        if (d >= whole) continue;
#pragma unroll
        for (int q = 0; q < VEC; q += 4) {
          float x[R][4];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if constexpr (sizeof(E) == 4) {
              x[r][0] = __uint_as_float(u[r].x); x[r][1] = __uint_as_float(u[r].y);
              x[r][2] = __uint_as_float(u[r].z); x[r][3] = __uint_as_float(u[r].w);
            } else {
              const uint32_t lo = q == 0 ? u[r].x : u[r].z, hi = q == 0 ? u[r].y : u[r].w;
              x[r][0] = __uint_as_float(lo << 16); x[r][1] = __uint_as_float(lo & 0xffff0000u);
              x[r][2] = __uint_as_float(hi << 16); x[r][3] = __uint_as_float(hi & 0xffff0000u);
            }
          }
#pragma unroll
          for (int t = 0; t < TT; ++t) {
            const float4 y = *reinterpret_cast<const float4*>(&sh[t * Dp + few_place<E, W>(d + q, Dp)]);
#pragma unroll
            for (int r = 0; r < R; ++r) {
              float& to = acc[r * TT + t];
              to = __fmaf_rn(x[r][0], y.x, to);
              to = __fmaf_rn(x[r][1], y.y, to);
              to = __fmaf_rn(x[r][2], y.z, to);
              to = __fmaf_rn(x[r][3], y.w, to);
            }
          }
        }
      }
    } else {
      // enough narrow loads in flight (pairs at 4 x 1854 x 92484: 118 -> 88 us from two)
#pragma unroll (W == 1 ? (TT <= 4 ? 8 : 4) : (TT <= 8 ? 4 : 2))
      for (int d = lane * W; d < whole; d += 32 * W) {
        float x[R][W];
#pragma unroll
        for (int r = 0; r < R; ++r) few_load<W>(rows[r] + d, x[r]);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
#pragma unroll
          for (int j = 0; j < W; ++j) {
            const float y = sh[t * Dp + d + j];
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r * TT + t] = __fmaf_rn(x[r][j], y, acc[r * TT + t]);
          }
        }
      }
    }
    if (W > 1 && whole + lane < f.D) {  // the columns after the last whole group
      const int d = whole + lane;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float x = few_float(rows[r][d]);
#pragma unroll
        for (int t = 0; t < TT; ++t)
          acc[r * TT + t] = __fmaf_rn(x, sh[t * Dp + few_place<E, W>(d, Dp)], acc[r * TT + t]);
      }
    }
    // sums over the lanes: halve the list and the lanes' share of it at each step
    {
      int c = N;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        if (c > 1) {
          c /= 2;
#pragma unroll
          for (int i = 0; i < N / 2; ++i) {
            if (i < c) {
              const bool up = lane & o;
              const float give = up ? acc[i] : acc[i + c];
              const float keep = up ? acc[i + c] : acc[i];
              acc[i] = fadd(keep, __shfl_xor_sync(kFull, give, o));
            }
          }
        } else {
          acc[0] = fadd(acc[0], __shfl_xor_sync(kFull, acc[0], o));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int t = t0 + (idx + i) % TT;
      const int64_t v = v0 + (idx + i) / TT;
      if (v < f.V && counts) {
        if (f.logits != nullptr && t < f.T) f.logits[t * f.V + v] = acc[i];
        if (v == target[i]) {  // out of the sum: a small loss is the logarithm of 1 + the others
          f.at[t] = acc[i];
          continue;
        }
        const float l = fmul(acc[i], kL2e);
        const float up = fmaxf(top[i], l);
        if (up != -INFINITY) {
          // (a sum without a largest value is 0, or NaN where a NaN logit came first)
          const float old = top[i] == -INFINITY ? sum[i] : fmul(sum[i], exp2f(fsub(top[i], up)));
          // one rounding in the exponent, as in the loss
          sum[i] = fadd(old, exp2f(__fmaf_rn(acc[i], kL2e, -up)));
          top[i] = up;
        } else if (acc[i] != acc[i]) {
          sum[i] = acc[i];
        }
      }
    }
  }
  __shared__ float2 all[kFewWarps][N];
  if (counts) {
#pragma unroll
    for (int i = 0; i < C; ++i) all[warp][idx + i] = make_float2(top[i], sum[i]);
  }
  __syncthreads();
  if (threadIdx.x < TT) {
    const int t = threadIdx.x;
    float m = -INFINITY, s = 0.0f;
    for (int q = 0; q < kFewWarps; ++q)
      for (int r = 0; r < R; ++r) m = fmaxf(m, all[q][r * TT + t].x);
    for (int q = 0; q < kFewWarps; ++q)
      for (int r = 0; r < R; ++r) {
        const float2 p = all[q][r * TT + t];
        if (p.x != -INFINITY) s = fadd(s, fmul(p.y, exp2f(fsub(p.x, m))));
        else if (p.y != p.y) s = p.y;
      }
    f.part[blockIdx.x * kFewTokens + t0 + t] = make_float2(m, s);
  }
}

// lse and loss, one warp a token; the weights of a gradient.
__global__ void __launch_bounds__(kFewTokens * 32) ce_few_finish_kernel(const Few f, int given) {
  pdl_begin();
  const int t = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned counted = __ballot_sync(kFull, few_target(f, lane) >= 0);
  const int n = __popc(counted);
  const bool live = counted >> t & 1;
  if (lane == 0 && f.weight != nullptr) {
    const float mean = n > 0 ? fdiv(1.0f, static_cast<float>(n)) : 0.0f;
    f.weight[t] = !live ? 0.0f : f.gloss != nullptr ? f.gloss[t] : mean;
  }
  if (t >= f.T || given) return;
  float m = -INFINITY, s = 0.0f;
  for (int i = lane; i < f.parts; i += 32) m = fmaxf(m, f.part[i * kFewTokens + t].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, o));
  for (int i = lane; i < f.parts; i += 32) {
    const float2 p = f.part[i * kFewTokens + t];
    if (p.x != -INFINITY) s = fadd(s, fmul(p.y, exp2f(fsub(p.x, m))));
    else if (p.y != p.y) s = p.y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s = fadd(s, __shfl_xor_sync(kFull, s, o));
  if (lane == 0) {
    const float l = f.at[t], d = __fmaf_rn(l, kL2e, -m), ratio = fmul(s, exp2f(-d));
    float loss = ratio < 1e6f ? log1pf(ratio) : fmul(fsub(log2f(s), d), kL2);
    float lse = fadd(l, loss);
    if (l == INFINITY) {  // inf - inf (an infinite d alone would make it 0)
      loss = __int_as_float(0x7fffffff);
      lse = fadd(l, s);
    } else if (l == -INFINITY) {  // of l + loss nothing is left: that of the others
      lse = fmul(fadd(log2f(s), m), kL2);
    }
    f.lse[t] = live ? lse : 0.0f;
    if (f.loss != nullptr) f.loss[t] = live ? loss : 0.0f;
  }
}

// Columns that a thread of the gradient kernel owns: h and dh's sums of TT tokens
// for each are 2 TT registers.
__host__ __device__ constexpr int few_cols(int tt) { return tt >= 16 ? 2 : 4; }
// CTAs of the gradient kernel on an SM, as its registers allow.
__host__ __device__ constexpr int few_resident(int tt) { return tt <= 2 ? 4 : tt == 4 ? 3 : 2; }
constexpr int kGradThreads = 256;
template <int BYTES> struct FewWord;
template <> struct FewWord<2> { using type = uint16_t; };
template <> struct FewWord<4> { using type = uint32_t; };
template <> struct FewWord<8> { using type = uint2; };
template <> struct FewWord<16> { using type = uint4; };

// dw rows of this CTA's range and its sums of dh.  Threads: G column groups of
// few_cols(TT), in accesses of A neighbouring columns that lie G accesses apart, by
// RL rows at a time; a CTA takes the columns of blockIdx.y.  D is a multiple of A;
// dw_words: dw's rows suit accesses of A.
template <typename E, int TT, int W>
__global__ void __launch_bounds__(kGradThreads, few_resident(TT)) ce_few_grad_kernel(const Few f, int G, int RL, int with_loss, int dw_words) {
  constexpr int kRows = 64, CP = few_cols(TT), A = W < CP ? W : CP, U = A == 1 && sizeof(E) == 4 && (TT == 4 || TT == 8) ? 2 : 4;
  constexpr bool kAhead = TT >= 8 || A == 4 || U == 2;
  pdl_begin();
  __shared__ __align__(16) float c[kRows][TT];
  __shared__ float lse_of[TT], weight_of[TT], minus_loss[TT];
  __shared__ int target_of[TT];
  extern __shared__ float red[];
  const E* h = static_cast<const E*>(f.h);
  const E* w = static_cast<const E*>(f.w);
  E* dw = static_cast<E*>(f.dw);
  const int group = threadIdx.x % G, rl = threadIdx.x / G;
  const int d0 = blockIdx.y * G * CP + group * A;
  auto col = [&](int j) { return d0 + j / A * G * A + j % A; };
  int at[CP / A];  // where each access reads, within the row
#pragma unroll
  for (int k = 0; k < CP / A; ++k) at[k] = min(col(k * A), f.D - A);
  if (threadIdx.x < TT) {
    const int t = threadIdx.x;
    target_of[t] = few_target(f, t);
    weight_of[t] = f.weight[t];
    lse_of[t] = t < f.T ? f.lse[t] : 0.0f;
    minus_loss[t] = t < f.T && target_of[t] >= 0
                        ? (with_loss ? -f.loss[t] : fsub(f.logits[t * f.V + target_of[t]], f.lse[t]))
                        : 0.0f;
  }
  float x[TT][CP], sum[TT][CP];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const bool live = few_target(f, t) >= 0;
#pragma unroll
    for (int j = 0; j < CP; ++j) {
      x[t][j] = live && col(j) < f.D ? few_float(h[t * f.ldh + col(j)]) : 0.0f;
      sum[t][j] = 0.0f;
    }
  }
  const int64_t first = f.V * blockIdx.x / gridDim.x, last = f.V * (blockIdx.x + 1) / gridDim.x;
  // U rows at a time, all their loads before the first store (which could be to what
  // the next row loads, for all the compiler knows) and without conditions: past the
  // end the last row and group are read again, with nothing done for them.  Where
  // registers allow, the loads run one step ahead, over the fill of c too (4096 x
  // 131072 fp32, 16 tokens 2310 -> 1976 us, 8 1224 -> 1092, 4 1027 -> 1018); loads of
  // single elements spill then.  2075 x 98787, four rows, four ahead, two ahead: fp32,
  // 8 tokens 764, 793, 695 us, 4 tokens 566, 869, 557, 2 tokens 492, 856, 532; bf16, 8
  // tokens 810, 756, 841, 4 tokens 564, 572, 591.
  float next[U][CP];
  auto read = [&](int64_t v) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const E* from = w + min64(v + rl + u * RL, last - 1) * f.ldw;
#pragma unroll
      for (int k = 0; k < CP; k += A) {
        float part[A];
        few_load<A>(from + at[k / A], part);
#pragma unroll
        for (int j = 0; j < A; ++j) next[u][k + j] = part[j];
      }
    }
  };
  if (kAhead) read(first);
  for (int64_t v0 = first; v0 < last; v0 += kRows) {
    const int rows = static_cast<int>(min64(last - v0, kRows));
    __syncthreads();
    for (int q = threadIdx.x; q < rows * TT; q += blockDim.x) {
      const int r = q % rows, t = q / rows;  // neighbouring threads read neighbouring logits
      float p = 0.0f;
      if (target_of[t] >= 0)
        p = fmul(weight_of[t], target_of[t] == v0 + r ? expm1f(minus_loss[t])
                                                      : expf(fsub(f.logits[t * f.V + v0 + r], lse_of[t])));
      c[r][t] = p;
    }
    __syncthreads();
    for (int b = 0; b < rows; b += RL * U) {
      float y[U][CP];
      if (!kAhead) read(v0 + b);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < CP; ++k) y[u][k] = next[u][k];
      if (kAhead) read(b + RL * U < rows ? v0 + b + RL * U : v0 + kRows);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = b + rl + u * RL;
        if (r < rows) {
          float z[CP] = {}, a[TT];
          if constexpr (TT >= 4) {
#pragma unroll
            for (int t = 0; t < TT; t += 4) {
              const float4 q = *reinterpret_cast<const float4*>(&c[r][t]);
              a[t] = q.x; a[t + 1] = q.y; a[t + 2] = q.z; a[t + 3] = q.w;
            }
          } else {
#pragma unroll
            for (int t = 0; t < TT; ++t) a[t] = c[r][t];
          }
#pragma unroll
          for (int t = 0; t < TT; ++t) {
#pragma unroll
            for (int j = 0; j < CP; ++j) {
              sum[t][j] = __fmaf_rn(a[t], y[u][j], sum[t][j]);
              z[j] = __fmaf_rn(a[t], x[t][j], z[j]);
            }
          }
          E* to = dw + (v0 + r) * f.lddw;
#pragma unroll
          for (int k = 0; k < CP; k += A) {
            E out[A];
#pragma unroll
            for (int j = 0; j < A; ++j) few_from(z[k + j], &out[j]);
            if (col(k) < f.D) {
              if (A == 1 || dw_words) {
                using U_ = typename FewWord<A * sizeof(E)>::type;
                U_ word;
                memcpy(&word, out, sizeof(word));
                *reinterpret_cast<U_*>(to + col(k)) = word;
              } else {
#pragma unroll
                for (int j = 0; j < A; ++j) to[col(k) + j] = out[j];
              }
            }
          }
        }
      }
    }
  }
  // the row lanes' sums, in their order
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    if (t < f.T) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < CP; ++j) red[(rl * CP + j) * G + group] = sum[t][j];
      __syncthreads();
      if (rl == 0) {
#pragma unroll
        for (int j = 0; j < CP; ++j) {
          float s = 0.0f;
          for (int q = 0; q < RL; ++q) s = fadd(s, red[(q * CP + j) * G + group]);
          if (col(j) < f.D) f.sums[(static_cast<int64_t>(blockIdx.x) * f.T + t) * f.D + col(j)] = s;
        }
      }
    }
  }
}

// dh: the sums of the CTAs, four interleaved running sums.
template <typename E>
__global__ void __launch_bounds__(256) ce_few_dh_kernel(const Few f, int ranges) {
  pdl_begin();
  __shared__ float part[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t q = blockIdx.x * int64_t{32} + lane, n = static_cast<int64_t>(f.T) * f.D;
  float s = 0.0f;
  if (q < n)
    for (int i = warp; i < ranges; i += 8) s = fadd(s, f.sums[i * n + q]);
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && q < n) {
    for (int i = 1; i < 8; ++i) s = fadd(s, part[i][lane]);
    const int t = static_cast<int>(q / f.D), d = static_cast<int>(q - static_cast<int64_t>(t) * f.D);
    few_from(few_target(f, t) >= 0 ? s : 0.0f, static_cast<E*>(f.dh) + t * f.lddh + d);
  }
}

int few_tokens_up(int64_t T) {
  int tt = 1;
  while (tt < T) tt *= 2;
  return tt;
}
// The gradient kernel's shape: G column groups by RL rows a CTA, `columns` CTAs
// across and `ranges` parts of the vocabulary, as many as are resident.
struct FewShape {
  int G, RL, columns, ranges;
};
FewShape few_shape(int64_t T, int64_t D, int64_t V, int num_sms) {
  const int tt = few_tokens_up(T), cp = few_cols(tt);
  FewShape p;
  p.G = static_cast<int>(std::min<int64_t>((D + cp - 1) / cp, kGradThreads));
  p.RL = kGradThreads / p.G;
  p.columns = static_cast<int>((D + cp * p.G - 1) / (cp * p.G));
  const int resident = num_sms * few_resident(tt);
  p.ranges = static_cast<int>(std::min<int64_t>(std::max(resident / p.columns, 1), (V + 15) / 16));
  return p;
}
constexpr int kMostSms = 160;

size_t few_up(size_t x) { return (x + 255) / 256 * 256; }

// Tokens that the logits kernel takes at a time: h of them in shared memory.
int few_group(int64_t T, int64_t D) {
  int tt = std::min(few_tokens_up(T), kFewGroup);
  while (tt > 1 && tt * ((D + 7) / 8 * 8) * 4 > kFewBytes) tt /= 2;
  return tt;
}

template <typename E, int TT, int W>
cudaError_t few_logits(const Few& f, int t0, int num_sms, cudaStream_t s) {
  auto kernel = ce_few_logits_kernel<E, TT, W>;
  cudaError_t e = ensure_dynamic_smem(kernel, kFewBytes);
  if (e != cudaSuccess) return e;
  return launch_kernel(kernel, dim3(num_sms), dim3(kFewThreads), TT * ((f.D + 7) / 8 * 8) * 4, s, 0, f, t0);
}

template <typename E, int TT, int W>
cudaError_t few_grad(const Few& f, int num_sms, bool with_loss, cudaStream_t s) {
  constexpr int CP = few_cols(TT), A = W < CP ? W : CP;
  const FewShape p = few_shape(f.T, f.D, f.V, num_sms);
  const bool words = reinterpret_cast<uintptr_t>(f.dw) % (A * sizeof(E)) == 0 && f.lddw % A == 0;
  cudaError_t e = launch_kernel(ce_few_grad_kernel<E, TT, W>, dim3(p.ranges, p.columns), dim3(p.G * p.RL),
                                p.G * p.RL * CP * 4, s, 0, f, p.G, p.RL, with_loss ? 1 : 0, words ? 1 : 0);
  if (e != cudaSuccess) return e;
  const int64_t n = static_cast<int64_t>(f.T) * f.D;
  return launch_kernel(ce_few_dh_kernel<E>, dim3(static_cast<unsigned>((n + 31) / 32)), dim3(256), 0, s, 0, f, p.ranges);
}

// Calls fn with the token count as a compile-time constant.
template <class F>
cudaError_t few_tokens(int tt, F fn) {
  switch (tt) {
    case 1: return fn(std::integral_constant<int, 1>{});
    case 2: return fn(std::integral_constant<int, 2>{});
    case 4: return fn(std::integral_constant<int, 4>{});
    case 8: return fn(std::integral_constant<int, 8>{});
    default: return fn(std::integral_constant<int, 16>{});
  }
}

template <typename E, int W>
cudaError_t few_run(const LinearCeArgs& a, Few f, int num_sms, cudaStream_t s) {
  const bool grad = a.dw != nullptr, given = a.loss == nullptr;
  f.parts = num_sms;
  const int most = few_group(f.T, f.D);
  cudaError_t e = cudaSuccess;
  for (int t0 = 0; t0 < f.T; t0 += most) {
    e = few_tokens(std::min(most, few_tokens_up(f.T - t0)),
                   [&](auto tt) { return few_logits<E, tt.value, W>(f, t0, num_sms, s); });
    if (e != cudaSuccess) return e;
  }
  e = launch_kernel(ce_few_finish_kernel, dim3(1), dim3(kFewTokens * 32), 0, s, 0, f, given ? 1 : 0);
  if (e != cudaSuccess || !grad) return e;
  return few_tokens(few_tokens_up(f.T), [&](auto tt) {
    constexpr int CP = few_cols(tt.value), A = W < CP ? W : CP;
    if (f.D % A == 0) return few_grad<E, tt.value, W>(f, num_sms, !given, s);
    return few_grad<E, tt.value, 1>(f, num_sms, !given, s);
  });
}

template <typename E>
cudaError_t few_typed(const LinearCeArgs& a, const Few& f, int num_sms, cudaStream_t s) {
  auto starts_on = [&](uintptr_t bytes) {
    return reinterpret_cast<uintptr_t>(a.w) % bytes == 0 && a.ldw * sizeof(E) % bytes == 0;
  };
  if (starts_on(16)) return few_run<E, 16 / sizeof(E)>(a, f, num_sms, s);
  if constexpr (sizeof(E) == 2) {
    if (starts_on(4)) return few_run<E, 2>(a, f, num_sms, s);
  }
  return few_run<E, 1>(a, f, num_sms, s);
}

struct FewLayout {
  size_t part, at, weight, lse, logits, sums, total;
};
FewLayout few_layout(int64_t T, int64_t D, int64_t V, bool grad) {
  FewLayout l = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t p = at;
    at += few_up(bytes);
    return p;
  };
  l.part = take(kMostSms * kFewTokens * 8);
  l.at = take(kFewTokens * 4);
  l.weight = take(kFewTokens * 4);
  l.lse = take(kFewTokens * 4);
  if (grad) {
    l.logits = take(static_cast<size_t>(T) * V * 4);
    l.sums = take(static_cast<size_t>(few_shape(T, D, V, kMostSms).ranges) * T * D * 4);
  }
  l.total = at;
  return l;
}

}  // namespace

// Whether a call goes this way, or by the matrix units, whose time hardly depends on
// so few tokens while a pass over w here takes 16 FMAs or less an element at no more
// than the memory's rate.  Measured, this way against the other:
//   fp32, loss       32 x 768 x 50257 145 us against 141, 17 tokens 110; 32 x 2075 x
//                    98787 460 against 780; 32 x 4096 x 131072 1517 against 1640
//   fp32, gradient   16 x 768 x 50257 207 us against 316, 16 x 4096 x 131072 1976
//                    against 3150; with sums for 32 tokens in registers 383 and 4548
//                    (one step behind in its loads)
//   bf16, loss       8 x 768 x 50257 40 us against 46, 8 x 4096 x 131072 258 against
//                    360, 16 of them 70 and 504; rows off 16 bytes, which the other
//                    way copies first: 16 x 2075 x 98787 225 against 332
//   bf16, gradient   8 x 2075 x 98787 756 us against 804, 8 x 4096 x 131072 1025
//                    against 1144, 16 of them 2028 and 1146 (as above)
// Small heads are bound by launches, of which this way has fewer: 16 x 300 x 5000 in
// bf16 42 us against 67, 16 x 1001 x 30000 195 against 187.  Wide rows take several
// passes: four over an fp32 w cost what the other way does, two over a bf16 one.
// ldw: 0 for a w that does not start on 16 bytes, as for the workspace.
bool linear_ce_few_fits(int64_t T, int64_t D, int64_t V, int64_t ldw, bool bf16, bool grad) {
  if (T > (bf16 || grad ? kFewGroup : kFewTokens) || (D + 7) / 8 * 8 * 4 > kFewBytes) return false;
  if (T > few_group(T, D) * (bf16 ? 1 : 4)) return false;
  const bool copied = ldw == 0 || ldw % 8 != 0;  // a bf16 w by the other way
  return !bf16 || T <= 8 || D * V < int64_t{1} << 24 || (!grad && copied);
}

size_t linear_ce_few_workspace_bytes(int64_t T, int64_t D, int64_t V, int grad) {
  return few_layout(T, D, V, grad != 0).total;
}

cudaError_t launch_linear_ce_few(const LinearCeArgs& a, int num_sms, cudaStream_t s) {
  const bool grad = a.dw != nullptr;
  const FewLayout l = few_layout(a.T, a.D, a.V, grad);
  char* ws = static_cast<char*>(a.ws);
  auto floats = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
  Few f = {};
  f.h = a.h;
  f.w = a.w;
  f.ldh = a.ldh;
  f.ldw = a.ldw;
  f.targets = a.targets;
  f.T = static_cast<int>(a.T);
  f.D = static_cast<int>(a.D);
  f.V = a.V;
  f.ignore = a.ignore;
  f.part = reinterpret_cast<float2*>(ws + l.part);
  f.at = floats(l.at);
  f.logits = grad ? floats(l.logits) : nullptr;
  f.lse = a.loss == nullptr ? const_cast<float*>(a.lse_in) : a.lse != nullptr ? a.lse : floats(l.lse);
  f.loss = a.loss;
  f.gloss = a.gloss;
  f.weight = grad ? floats(l.weight) : nullptr;
  f.sums = floats(l.sums);
  f.dh = a.dh;
  f.dw = a.dw;
  f.lddh = a.lddh;
  f.lddw = a.lddw;
  f.status = a.status;
  num_sms = std::min(num_sms, kMostSms);
  return a.bf16 ? few_typed<__nv_bfloat16>(a, f, num_sms, s) : few_typed<float>(a, f, num_sms, s);
}

}  // namespace mpc
