// linear_few.cu -- the linear layer's forward pass of a few rows: the tokens of a served
// batch.
//
//   y[m][n] = layer(sum_k x[m][k] w[n][k]),  up to 64 rows m (bf16) or 8
//
// What bounds it is one pass over w: a tile of the matrix units would be empty rows for the most
// part, and its start, its accumulators' way through tensor memory and the parts along K with
// a launch to add them cost more than the pass itself (24 x 4096 x 4096 in bf16: 17 + 4.5
// us; 5.0 us is what 33.5 MB of w take).
//
// bf16 rows on 16 bytes, up to 64 rows of x: linear_few_mma_kernel.  A CTA of four or eight
// warps takes 16 or 32 rows of w, its warps a stretch of K each.  A lane reads 32 (or 16) bytes of a row
// of w and as many of a row of x and feeds them to warp-level products as they lie: the sum over K
// may run in any order, so the k that a lane of the fragment stands for is that of its own
// bytes, the same in both operands.  The warps' sums are added in shared memory in a
// fixed order, and every thread finishes some of the CTA's results.
//
// fp32, and rows on any alignment, up to 8 rows: linear_few_kernel, the same with plain fp32 FMAs, a
// warp 4 rows of w and all of K.
//
// Measured with w in HBM, launches in a graph: bf16 1 x 1024 x 4096 3.3 us, 1 x 4096 x 4096 7.0 (4.8
// TB/s), 8 x 4096 x 16384 27 (4.9 TB/s), 24 x 4096 x 4096 10.9, 64 x 4096 x 4096 17.9 (x comes from
// L2 once for every 16 rows of w: 50 MB with 24 rows, 134 with 64, beside 34 MB of w); fp32 1 x 4096 x 4096 14 us (4.8 TB/s), 8 rows 36; bf16
// rows on 2 bytes 38 us.  16-byte accesses (64 bytes of a row a time) took 10.2 for 7.0.
#include <algorithm>
#include <type_traits>

#include "launch_util.h"
#include "layers.cuh"

namespace mpc {
namespace {

struct Few {
  LinearArgs a;
  Drop drop;
};

// The end of one result: z (summed, without bias) to y.
template <typename T>
__device__ __forceinline__ void finish_one(const Few& f, uint64_t seed, int64_t m, int64_t n, float v) {
  const LinearArgs& a = f.a;
  if (a.bias != nullptr) v = fadd(v, as_float(static_cast<const T*>(a.bias)[n]));
  if (a.z != nullptr) put(static_cast<T*>(a.z) + m * a.ldz + n, v);
  v = act_value<sizeof(T) == 2>(a.act, v);
  if (f.drop.level > 0) v = kept_at(seed, static_cast<uint64_t>(m) * a.out + n, f.drop.level) ? fmul(v, f.drop.scale) : 0.0f;
  if (a.residual != nullptr) v = fadd(as_float(static_cast<const T*>(a.residual)[m * a.ldr + n]), v);
  put(static_cast<T*>(a.y) + m * a.ldy + n, v);
}

// D += A B for A 16 x 16, B 16 x 8 of bf16: lane 4 i + j holds of A rows i and i + 8, of B column i,
// the k of its j; of D rows i and i + 8, columns 2 j and 2 j + 1.
__device__ __forceinline__ void warp_product(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// B bytes of a lane: k of a step.
template <int B>
struct Bytes {
  uint32_t u[B / 4];
};
template <int B>
__device__ __forceinline__ void load_bytes(Bytes<B>& v, const void* p, bool there) {
  if (!there) {
#pragma unroll
    for (int i = 0; i < B / 4; ++i) v.u[i] = 0;
  } else if constexpr (B == 32) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v.u[0]), "=r"(v.u[1]), "=r"(v.u[2]), "=r"(v.u[3]), "=r"(v.u[4]), "=r"(v.u[5]), "=r"(v.u[6]), "=r"(v.u[7])
                 : "l"(p));
  } else {
    const uint4 x = *static_cast<const uint4*>(p);
    v.u[0] = x.x, v.u[1] = x.y, v.u[2] = x.z, v.u[3] = x.w;
  }
}

// NT: groups of 8 rows of x; RT: groups of 16 rows of w; B: bytes of an access.
template <int NT, int RT, int B, int kMmaWarps>
__global__ void __launch_bounds__(kMmaWarps * 32) linear_few_mma_kernel(const Few f) {
  constexpr int kRows = 16 * RT, kTokens = 8 * NT;
  __shared__ float sums[kMmaWarps][kRows][kTokens + 1];
  pdl_begin();
  pdl_end();
  const LinearArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i = lane >> 2, j = lane & 3;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kRows;
  const int K = static_cast<int>(a.in), M = static_cast<int>(a.rows);
  const __nv_bfloat16* w = static_cast<const __nv_bfloat16*>(a.w);
  const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(a.x);
  // rows that do not exist are read as the last one; their sums are not used
  const __nv_bfloat16* wr[2 * RT];
  const __nv_bfloat16* xr[NT];
#pragma unroll
  for (int r = 0; r < 2 * RT; ++r) wr[r] = w + min64(n0 + r * 8 + i, a.out - 1) * a.ldw;
#pragma unroll
  for (int r = 0; r < NT; ++r) xr[r] = x + static_cast<int64_t>(min(r * 8 + i, M - 1)) * a.ldx;
  constexpr int kEach = B / 2, kStep = 4 * kEach;  // k of a lane, of a step
  const int steps = (K + kStep - 1) / kStep;
  const int first = static_cast<int>(static_cast<int64_t>(steps) * warp / kMmaWarps);
  const int last = static_cast<int>(static_cast<int64_t>(steps) * (warp + 1) / kMmaWarps);
  float d[RT][NT][4] = {};
  // a ring of steps whose loads are in flight
  constexpr int kLoads = (2 * RT + NT) * (B / 16), kAhead = kLoads <= 3 ? 8 : kLoads <= 6 ? 4 : kLoads <= 12 ? 2 : 1;
  Bytes<B> wa[kAhead][2 * RT], xb[kAhead][NT];
  auto load = [&](int u, int s) {
    const int k = s * kStep + j * kEach;  // K is a multiple of kEach: all of a lane's exist, or none
    const bool there = s < last && k < K;
#pragma unroll
    for (int r = 0; r < 2 * RT; ++r) load_bytes<B>(wa[u][r], wr[r] + k, there);
#pragma unroll
    for (int r = 0; r < NT; ++r) load_bytes<B>(xb[u][r], xr[r] + k, there);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) load(u, first + u);
  for (int s = first; s < last; s += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int q = 0; q < B / 4; q += 2) {
            const uint32_t *lo = wa[u][2 * r].u + q, *hi = wa[u][2 * r + 1].u + q, *b = xb[u][t].u + q;
            warp_product(d[r][t], lo[0], hi[0], lo[1], hi[1], b[0], b[1]);
          }
      load(u, s + u + kAhead);
    }
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int q = 0; q < 4; ++q) sums[warp][r * 16 + (q >> 1) * 8 + i][t * 8 + 2 * j + (q & 1)] = d[r][t][q];
  __syncthreads();
  const uint64_t seed = f.drop.level > 0 ? drop_seed(f.drop) : 0;
  for (int q = threadIdx.x; q < kRows * kTokens; q += kMmaWarps * 32) {
    const int r = q % kRows, t = q / kRows;  // neighbouring threads neighbouring columns of y
    if (t >= M || n0 + r >= a.out) continue;
    float v = sums[0][r][t];
#pragma unroll
    for (int p = 1; p < kMmaWarps; ++p) v = fadd(v, sums[p][r][t]);
    finish_one<__nv_bfloat16>(f, seed, t, n0 + r, v);
  }
}

// W elements of a row an access.
template <typename T, int W>
__device__ __forceinline__ void few_load(const T* p, float (&v)[W]) {
  if constexpr (W == 1) {
    v[0] = as_float(*p);
  } else if constexpr (W * sizeof(T) == 16) {
    unpack16(*reinterpret_cast<const uint4*>(p), v);
  } else {  // a pair of bf16
    const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
    v[0] = __uint_as_float(u << 16);
    v[1] = __uint_as_float(u & 0xffff0000u);
  }
}


// M rows of x; accesses of W elements, of which K is a multiple. A warp takes four
// rows of w: x is read once for all of them.
template <typename T, int M, int W>
__global__ void __launch_bounds__(128) linear_few_kernel(const Few f) {
  constexpr int kFmaRows = 4;
  pdl_begin();
  pdl_end();
  const LinearArgs& a = f.a;
  const int lane = threadIdx.x & 31;
  const int64_t n0 = (static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5)) * kFmaRows;
  if (n0 >= a.out) return;
  const T* x = static_cast<const T*>(a.x);
  const int K = static_cast<int>(a.in), rows = static_cast<int>(a.rows);
  const T* wr[kFmaRows];
#pragma unroll
  for (int r = 0; r < kFmaRows; ++r) wr[r] = static_cast<const T*>(a.w) + min64(n0 + r, a.out - 1) * a.ldw;
  float acc[kFmaRows][M] = {};
  constexpr int kAhead = W == 1 ? 8 : 4;
  for (int k0 = lane * W; k0 < K; k0 += 32 * W * kAhead) {
    float wv[kAhead][kFmaRows][W];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int r = 0; r < kFmaRows; ++r) {
        const int k = k0 + u * 32 * W;
        if (k < K) {
          few_load<T, W>(wr[r] + k, wv[u][r]);
        } else {
#pragma unroll
          for (int e = 0; e < W; ++e) wv[u][r][e] = 0.0f;
        }
      }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int k = k0 + u * 32 * W;
      if (k < K) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
          float xv[W];
          few_load<T, W>(x + static_cast<int64_t>(min(m, rows - 1)) * a.ldx + k, xv);
#pragma unroll
          for (int r = 0; r < kFmaRows; ++r)
#pragma unroll
            for (int e = 0; e < W; ++e) acc[r][m] = __fmaf_rn(xv[e], wv[u][r][e], acc[r][m]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kFmaRows; ++r)
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[r][m] = fadd(acc[r][m], __shfl_xor_sync(kFull, acc[r][m], o));
  const uint64_t seed = f.drop.level > 0 ? drop_seed(f.drop) : 0;
  // result r M + m by lane r M + m
#pragma unroll
  for (int r = 0; r < kFmaRows; ++r)
#pragma unroll
    for (int m = 0; m < M; ++m)
      if (lane == r * M + m && m < rows && n0 + r < a.out) finish_one<T>(f, seed, m, n0 + r, acc[r][m]);
}

template <int NT, int RT, int B, int WARPS>
cudaError_t launch_mma(const Few& f, cudaStream_t s) {
  const unsigned grid = static_cast<unsigned>((f.a.out + 16 * RT - 1) / (16 * RT));
  return launch_kernel(linear_few_mma_kernel<NT, RT, B, WARPS>, dim3(grid), dim3(WARPS * 32), 0, s, 0u, f);
}
// 32 rows of w a CTA read x half as often, where enough CTAs are left and the loads in flight
// fit the registers; eight warps along K where a warp's stretch stays long and little of x is
// read (1 x 4096 x 4096 in bf16 7.1 us, with four 7.7; 24 x 4096 x 4096 12.6 and 10.9).
template <int NT, int B>
cudaError_t launch_mma(const Few& f, int num_sms, cudaStream_t s) {
  if constexpr (NT <= 2) {
    const bool wide = f.a.out >= int64_t{32} * 2 * num_sms;
    if (NT == 1 && f.a.in >= 2048)
      return wide ? launch_mma<NT, 2, B, 8>(f, s) : launch_mma<NT, 1, B, 8>(f, s);
    if (wide) return launch_mma<NT, 2, B, 4>(f, s);
  }
  return launch_mma<NT, 1, B, 4>(f, s);
}
template <int B>
cudaError_t launch_mma(const Few& f, int num_sms, cudaStream_t s) {
  switch ((f.a.rows + 7) / 8) {
    case 1: return launch_mma<1, B>(f, num_sms, s);
    case 2: return launch_mma<2, B>(f, num_sms, s);
    case 3: return launch_mma<3, B>(f, num_sms, s);
    case 4: return launch_mma<4, B>(f, num_sms, s);
    default: return launch_mma<8, B>(f, num_sms, s);
  }
}

template <typename T, int W>
cudaError_t launch_fma(const Few& f, cudaStream_t s) {
  const int64_t m = f.a.rows, each = 16;
  const unsigned grid = static_cast<unsigned>((f.a.out + each - 1) / each);
  auto* kernel = m <= 1 ? linear_few_kernel<T, 1, W> : m <= 2 ? linear_few_kernel<T, 2, W> : m <= 4 ? linear_few_kernel<T, 4, W>
                                                                                         : linear_few_kernel<T, 8, W>;
  return launch_kernel(kernel, dim3(grid), dim3(128), 0, s, 0u, f);
}

}  // namespace

bool linear_few_fits(int64_t rows, int64_t in, int bf16, int64_t ldx, int64_t ldw) {
  const bool mma = bf16 && in % 8 == 0 && ldx >= in && ldw >= in && ldx % 8 == 0 && ldw % 8 == 0;
  return rows <= (mma ? 64 : 8);
}

cudaError_t launch_linear_few(const LinearArgs& a, int num_sms, cudaStream_t s) {
  const Few f = {a, make_drop(a.p, a.seed, a.step)};
  auto on = [&](uintptr_t bytes) {
    const int64_t size = a.bf16 ? 2 : 4;
    return ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w) | static_cast<uintptr_t>(a.ldx * size) |
             static_cast<uintptr_t>(a.ldw * size) | static_cast<uintptr_t>(a.in * size)) % bytes) == 0;
  };
  if (a.bf16) {
    if (on(32)) return launch_mma<32>(f, num_sms, s);
    if (on(16)) return launch_mma<16>(f, num_sms, s);
    return on(4) ? launch_fma<__nv_bfloat16, 2>(f, s) : launch_fma<__nv_bfloat16, 1>(f, s);
  }
  return on(16) ? launch_fma<float, 4>(f, s) : launch_fma<float, 1>(f, s);
}

}  // namespace mpc
