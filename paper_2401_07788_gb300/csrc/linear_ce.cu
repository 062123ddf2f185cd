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

#include "kernels.h"
#include "launch_util.h"
#include "tcgen05.cuh"

namespace mpc {
namespace {

constexpr int kM = 128;        // rows of a CTA's output tile (lanes of tensor memory)
constexpr int kPair = 2 * kM;  // rows of a CTA pair's output tile
constexpr int kN = 256;        // columns of an output tile
constexpr int kK = 64;         // K elements of a stage: 128 bytes, one swizzle row
constexpr int kStages = 6;
constexpr int kBytesA = kM * kK * 2;
constexpr int kBytesB = kN / 2 * kK * 2;
constexpr int kStageBytes = kBytesA + kBytesB;
constexpr int kEpiWarps = 8;
constexpr int kGemmThreads = (2 + kEpiWarps) * 32;
constexpr int kHalf = kN / 2;  // columns an epilogue warp takes
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Header {
  int valid;  // tokens that count
  float mean; // 1 / valid (0 when none counts)
};

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
// Operands in bf16 planes.  A bf16 tensor is one plane.  An fp32 x is the sum of
// three, x0 = bf16(x), x1 = bf16(x - x0), x2 = bf16(x - x0 - x1) (24 bits), and a
// product of two fp32 tensors the sum of the plane products i + j <= 2, six of
// them: what is left out is below 2^-24 of a term.  One kernel so serves both
// types, an fp32 product being a bf16 one with six times the K steps.
// ---------------------------------------------------------------------------
__device__ __forceinline__ void split(float x, uint16_t (&p)[3]) {
  const __nv_bfloat16 a = __float2bfloat16_rn(x);
  const float r = fsub(x, __bfloat162float(a));
  const __nv_bfloat16 b = __float2bfloat16_rn(r);
  const __nv_bfloat16 c = __float2bfloat16_rn(fsub(r, __bfloat162float(b)));
  p[0] = __bfloat16_as_ushort(a);
  p[1] = __bfloat16_as_ushort(b);
  p[2] = __bfloat16_as_ushort(c);
}

template <typename E>
__device__ __forceinline__ void planes_of(E x, uint16_t (&p)[3]);
template <>
__device__ __forceinline__ void planes_of<float>(float x, uint16_t (&p)[3]) { split(x, p); }
template <>
__device__ __forceinline__ void planes_of<__nv_bfloat16>(__nv_bfloat16 x, uint16_t (&p)[3]) {
  p[0] = __bfloat16_as_ushort(x);
}

// out[plane][r][0..Dp) of `rows` rows: row r is x's row list[r] (r itself without
// a list); zeros for r >= *count and for columns >= D.
template <typename E, int P>
__global__ void __launch_bounds__(256)
    ce_pack_kernel(const E* __restrict__ x, int64_t ld, const int* __restrict__ list, const int* count, int64_t rows,
                   int64_t padded, int D, int Dp, uint16_t* __restrict__ out) {
  pdl_begin();
  const int64_t n = count != nullptr ? *count : rows;
  const int64_t need = min64((n + kPair - 1) / kPair * kPair, padded);  // rows that a product may touch
  const int groups = Dp / 8;
  const int64_t plane = padded * Dp;
  for (int64_t q = blockIdx.x * int64_t{256} + threadIdx.x; q < need * groups; q += gridDim.x * int64_t{256}) {
    const int64_t r = q / groups;
    const int d0 = static_cast<int>(q % groups) * 8;
    uint16_t p[8][3];
    const E* src = r < n ? x + (list != nullptr ? list[r] : r) * ld + d0 : nullptr;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (src != nullptr && d0 + j < D) planes_of<E>(src[j], p[j]);
      else p[j][0] = p[j][1] = p[j][2] = 0;
    }
#pragma unroll
    for (int k = 0; k < P; ++k) {
      uint4 u;
      u.x = p[0][k] | static_cast<uint32_t>(p[1][k]) << 16;
      u.y = p[2][k] | static_cast<uint32_t>(p[3][k]) << 16;
      u.z = p[4][k] | static_cast<uint32_t>(p[5][k]) << 16;
      u.w = p[6][k] | static_cast<uint32_t>(p[7][k]) << 16;
      *reinterpret_cast<uint4*>(out + k * plane + r * Dp + d0) = u;
    }
  }
}

// ---------------------------------------------------------------------------
// The matrix products: C[m][n] = sum_k A[m][k] B[n][k] in 256 x 256 tiles.
//
// A persistent pair of CTAs on two SMs per tile, 128 rows each: every CTA copies
// its rows of A and half the rows of B, so an SM reads 32 KB from L2 for 2^20
// products (48 KB with a tile of its own).  Warp 0 copies operand tiles through
// tensor maps (kStages stages of 32 KB a CTA), one thread of the first CTA's warp
// 1 issues the products of both, eight warps a CTA take the finished tile from
// tensor memory.  Two
// accumulators of 256 columns fill the tensor memory, so a tile's epilogue runs
// under the next tile's products.
//
// kLoss   A = h [valid][D],  B = w [V][D]: a tile's logits become, for each token
//         and half tile, their largest and the sum of exponentials over it.
// kCoef   the same products again: the coefficients c of a piece of the vocabulary,
//         rounded to bf16 planes.
// kDh     A = c [valid][piece], B = w^T [D][piece]: dh, K split over several CTAs
//         where there are few tiles, each split's sum kept in fp32.
// kDw     A = c^T [piece][valid], B = h^T [D][valid]: dw of the piece.
//
// An accumulator adds each product step with truncation: about 5e-9 of its value
// a step of 16, always towards zero (measured: dh over 50257 entries 9e-5 off).
// Where fp32 results depend on it, an accumulator sums a chunk of K blocks only,
// the smallest plane products first, and the epilogue adds the chunks in fp32
// with rounding to nearest; two accumulators in turn keep the products running.
// Operands whose K is not the contiguous axis (w^T, c^T, h^T) are read as they
// are: rows of 64 M/N-elements, and the product's descriptors say so.
// ---------------------------------------------------------------------------
enum Mode { kLoss, kCoef, kDh, kDw };

struct Gemm {
  const Header* head;
  const int* row;       // token of a listed row
  const int* target;
  int T;                // tokens (upper bound of the list)
  int D;
  int width;            // vocabulary entries of the piece
  int64_t v0;           // its first one
  int terms;            // 1 (bf16) or 6 (fp32 in three planes)
  int chunk;            // K blocks that one accumulator sums (see ce_gemm_kernel)
  int splits;           // kDh: parts of K
  int first;            // kDh: the piece that starts the sums
  float2* part;         // kLoss: [half tile][T] (largest logit, sum), base 2
  float* at_target;     // kLoss: [T]
  const float* lse;     // kCoef: [T] by token
  const float* gloss;   // kCoef: [T] by token, or nullptr for the mean
  uint16_t* coef;       // kCoef: [plane][rows][ldc]
  int64_t ldc, coef_plane;
  float* sum;           // kDh: [split][rows][lds]
  int64_t lds, sum_split;
  void* dw;             // kDw
  int64_t lddw;
  int dw_bf16, dw_wide; // type; rows and base suit 32-byte stores
  uint32_t spin_limit;
  unsigned* status;
};

// Plane pair of a term, smallest products first.
__device__ __forceinline__ void term_planes(int terms, int t, int* a, int* b) {
  if (terms == 1) {
    *a = *b = 0;
  } else {  // (2,0) (0,2) (1,1) (1,0) (0,1) (0,0), two bits each
    *a = (0x052 >> (2 * t)) & 3;
    *b = (0x118 >> (2 * t)) & 3;
  }
}

struct Tile {
  int m0, n0, split, k0, k1;  // K blocks [k0, k1)
};

struct Shape {
  int m_tiles, n_tiles, blocks, splits;
  __device__ int total() const { return m_tiles * n_tiles * splits; }
};

template <int MODE>
__device__ __forceinline__ Shape shape_of(const Gemm& g, int valid) {
  Shape s;
  const int m = MODE == kDw ? g.width : valid;
  const int n = MODE == kDh || MODE == kDw ? g.D : g.width;
  const int k = MODE == kDh ? g.width : MODE == kDw ? valid : g.D;
  s.m_tiles = (m + kPair - 1) / kPair;
  s.n_tiles = (n + kN - 1) / kN;
  s.blocks = (k + kK - 1) / kK;
  s.splits = MODE == kDh ? g.splits : 1;
  return s;
}

// Order of the tiles: those that run at the same time share operands in L2.  For
// the logits all tokens pass one stretch of the vocabulary; for dh and dw the
// columns of one row tile of c run together, so that c is read from HBM once.
template <int MODE>
__device__ __forceinline__ Tile tile_of(const Shape& s, int i) {
  Tile t;
  if (MODE == kLoss || MODE == kCoef) {
    t.m0 = i % s.m_tiles * kPair;
    t.n0 = i / s.m_tiles * kN;
    t.split = 0;
  } else {
    t.n0 = i % s.n_tiles * kN;
    i /= s.n_tiles;
    t.m0 = i % s.m_tiles * kPair;
    t.split = i / s.m_tiles;
  }
  t.k0 = static_cast<int>(static_cast<int64_t>(s.blocks) * t.split / s.splits);
  t.k1 = static_cast<int>(static_cast<int64_t>(s.blocks) * (t.split + 1) / s.splits);
  return t;
}

__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  uint32_t u;
  memcpy(&u, &p, 4);
  return u;
}

// One lane's row of a half tile: x[j] = C[m][n0 + j], j < 128.
template <int MODE>
__device__ __forceinline__ void epilogue(const Gemm& g, int valid, const Tile& t, int m, int n0, float (&x)[kHalf]) {
  if (MODE == kLoss) {
    const int cols = min(g.width - n0, kHalf);
    if (cols <= 0 || m >= valid) return;
    const int y = static_cast<int>(g.target[m] - n0);
    if (cols < kHalf) {
#pragma unroll
      for (int j = 0; j < kHalf; ++j)
        if (j >= cols) x[j] = -INFINITY;
    }
    if (y >= 0 && y < cols) {
      float v = x[0];
#pragma unroll
      for (int j = 1; j < kHalf; ++j) v = j == y ? x[j] : v;
      g.at_target[m] = v;
    }
    // base 2 throughout: exp(l - top) = 2^(l log2e - top log2e), one rounding in the exponent
    float top = x[0];
#pragma unroll
    for (int j = 1; j < kHalf; ++j) top = fmaxf(top, x[j]);
    const float base = fmul(top, kLog2e);
    const float shift = base == -INFINITY ? 0.0f : -base;
    float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
    for (int j = 0; j < kHalf; j += 4) {
      s0 = fadd(s0, exp2_approx(__fmaf_rn(x[j], kLog2e, shift)));
      s1 = fadd(s1, exp2_approx(__fmaf_rn(x[j + 1], kLog2e, shift)));
      s2 = fadd(s2, exp2_approx(__fmaf_rn(x[j + 2], kLog2e, shift)));
      s3 = fadd(s3, exp2_approx(__fmaf_rn(x[j + 3], kLog2e, shift)));
    }
    g.part[static_cast<int64_t>(n0 / kHalf) * g.T + m] = make_float2(base, fadd(fadd(s0, s1), fadd(s2, s3)));
  } else if (MODE == kCoef) {
    if (n0 >= g.ldc) return;
    const bool live = m < valid;
    float shift = 0.0f, weight = 0.0f, scale = 0.0f;
    int y = -1;
    if (live) {
      const int token = g.row[m];
      const float lse = g.lse[token];
      weight = g.gloss != nullptr ? g.gloss[token] : g.head->mean;
      // what the rounding of lse log2e leaves out goes into the factor
      shift = fmul(lse, -kLog2e);
      scale = fmul(weight, exp2f(-__fmaf_rn(lse, kLog2e, shift)));
      y = static_cast<int>(g.target[m] - g.v0 - n0);
    }
#pragma unroll
    for (int j = 0; j < kHalf; ++j)
      x[j] = live ? fmul(scale, exp2_approx(__fmaf_rn(x[j], kLog2e, shift))) : 0.0f;
    if (y >= 0 && y < kHalf) {
#pragma unroll
      for (int j = 0; j < kHalf; ++j)
        if (j == y) x[j] = fsub(x[j], weight);
    }
    uint16_t* out = g.coef + m * g.ldc + n0;
    if (g.terms == 1) {
#pragma unroll
      for (int j = 0; j < kHalf; j += 16) {
        uint32_t u[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) u[q] = pack_bf16(x[j + 2 * q], x[j + 2 * q + 1]);
        st_v8(out + j, u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kHalf; j += 16) {
        uint32_t u[3][8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          uint16_t a[3], b[3];
          split(x[j + 2 * q], a);
          split(x[j + 2 * q + 1], b);
#pragma unroll
          for (int k = 0; k < 3; ++k) u[k][q] = a[k] | static_cast<uint32_t>(b[k]) << 16;
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) st_v8(out + k * g.coef_plane + j, u[k]);
      }
    }
  } else if (MODE == kDh) {
    if (m >= valid) return;
    float* out = g.sum + t.split * g.sum_split + m * g.lds + n0;
#pragma unroll
    for (int j = 0; j < kHalf; j += 8) {
      if (n0 + j < g.lds) {
        uint32_t u[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if (!g.first) x[j + q] = fadd(x[j + q], out[j + q]);
          u[q] = __float_as_uint(x[j + q]);
        }
        st_v8(out + j, u);
      }
    }
  } else {
    if (m >= g.width) return;
    const int64_t at = (g.v0 + m) * g.lddw + n0;
    if (g.dw_bf16) {
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(g.dw) + at;
#pragma unroll
      for (int j = 0; j < kHalf; j += 16) {
        if (g.dw_wide && n0 + j + 16 <= g.D) {
          uint32_t u[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) u[q] = pack_bf16(x[j + 2 * q], x[j + 2 * q + 1]);
          st_v8(out + j, u);
        } else {
#pragma unroll
          for (int q = 0; q < 16; ++q)
            if (n0 + j + q < g.D) out[j + q] = __float2bfloat16_rn(x[j + q]);
        }
      }
    } else {
      float* out = static_cast<float*>(g.dw) + at;
#pragma unroll
      for (int j = 0; j < kHalf; j += 8) {
        if (g.dw_wide && n0 + j + 8 <= g.D) {
          uint32_t u[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) u[q] = __float_as_uint(x[j + q]);
          st_v8(out + j, u);
        } else {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            if (n0 + j + q < g.D) out[j + q] = x[j + q];
        }
      }
    }
  }
}

// Columns of a tile that the product forms: a multiple of 16.  Each CTA of the
// pair holds half of them as rows of B.
__device__ __forceinline__ int tile_cols(int cols, int n0) { return min((cols - n0 + 15) / 16 * 16, kN); }

template <int MODE>
__global__ void __launch_bounds__(kGemmThreads, 1)
    ce_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ Gemm g) {
  constexpr bool A_MN = MODE == kDw, B_MN = MODE == kDh || MODE == kDw;
  extern __shared__ uint8_t raw[];
  // full and taken are used in the first CTA, for both; empty and done in each
  __shared__ uint64_t full[kStages], empty[kStages], done[2], taken[2], drain;
  __shared__ uint32_t tmem;
  uint8_t* stage0 = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_rank());
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&done[i], 1);
      mbar_init(&taken[i], 2 * kEpiWarps);
    }
    mbar_init(&drain, 1);
    fence_mbar_init();
    prefetch_map(&map_a);
    prefetch_map(&map_b);
  }
  if (warp == 1) tmem_alloc(&tmem, 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t acc = tmem;
  pdl_begin();
  const int valid = g.head->valid;
  const Shape s = shape_of<MODE>(g, valid);
  const int total = s.total();
  const int cols = MODE == kDh || MODE == kDw ? g.D : g.width;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (warp == 0) {
    if (lane == 0) {
      fence_proxy_async_all();  // operands that earlier kernels wrote
      uint32_t it = 0;
      bool ok = true;
      for (int i = pair; i < total && ok; i += pairs) {
        const Tile t = tile_of<MODE>(s, i);
        const int m0 = t.m0 + rank * kM, n0 = t.n0 + rank * (tile_cols(cols, t.n0) / 2);
        for (int c = t.k0; c < t.k1 && ok; c += g.chunk) {
          const int blocks = min(g.chunk, t.k1 - c);
          for (int j = 0; j < blocks * g.terms; ++j, ++it) {
            const int kb = c + j % blocks;
            const int st = it % kStages;
            ok = mbar_wait_bounded(&empty[st], (it / kStages & 1) ^ 1, g.spin_limit, g.status);
            if (!ok) break;
            int pa, pb;
            term_planes(g.terms, j / blocks, &pa, &pb);
            uint8_t* a = stage0 + st * kStageBytes;
            uint8_t* b = a + kBytesA;
            const uint32_t bar = dsmem_addr(&full[st], 0);
            if (rank == 0) mbar_arrive_expect_tx(&full[st], 2 * kStageBytes);
            if (A_MN) {
#pragma unroll
              for (int q = 0; q < kM / 64; ++q) tensor_g2s(a + q * kK * 128, &map_a, m0 + q * 64, kb * kK, pa, bar);
            } else {
              tensor_g2s(a, &map_a, kb * kK, m0, pa, bar);
            }
            if (B_MN) {
              const int k_at = kb * kK + (MODE == kDh ? static_cast<int>(g.v0) : 0);
#pragma unroll
              for (int q = 0; q < kN / 128; ++q) tensor_g2s(b + q * kK * 128, &map_b, n0 + q * 64, k_at, pb, bar);
            } else {
              tensor_g2s(b, &map_b, kb * kK, static_cast<int>(g.v0) + n0, pb, bar);
            }
          }
        }
      }
      // Copies in flight must land before either CTA leaves (the cluster barrier
      // below).  The first CTA sees both CTAs' copies arrive; where a wait gave up,
      // the second one may have sent some that the first no longer counts, and
      // gives them a millisecond.
      if (rank == 0) {
        for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i)
          mbar_wait_bounded(&full[i % kStages], i / kStages & 1, kDrainPolls, g.status);
      } else if (!ok) {
        const uint64_t until = global_ns() + 1000000;
        while (global_ns() < until) __nanosleep(1000);
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, n = 0;
      bool ok = true;
      for (int i = pair; i < total && ok; i += pairs) {
        const Tile t = tile_of<MODE>(s, i);
        const uint32_t idesc = mma_desc(kPair, tile_cols(cols, t.n0), A_MN, B_MN);
        for (int c = t.k0; c < t.k1 && ok; c += g.chunk, ++n) {
          ok = mbar_wait_bounded(&taken[n & 1], (n / 2 & 1) ^ 1, g.spin_limit, g.status);
          tc_fence_after();
          const uint32_t d = acc + (n & 1) * kN;
          bool fresh = true;
          const int steps = min(g.chunk, t.k1 - c) * g.terms;
          for (int k = 0; k < steps && ok; ++k, ++it) {
            const int st = it % kStages;
            ok = mbar_wait_bounded(&full[st], it / kStages & 1, g.spin_limit, g.status);
            if (!ok) break;
            tc_fence_after();
            const uint32_t a = smem_addr(stage0 + st * kStageBytes), b = a + kBytesA;
#pragma unroll
            for (int q = 0; q < kK / 16; ++q) {
              // 16 K-elements on: 32 bytes along a row, or 16 rows of 128 bytes
              const uint64_t da = A_MN ? smem_desc(a + q * 2048, kK * 128, 1024) : smem_desc(a + q * 32, 16, 1024);
              const uint64_t db = B_MN ? smem_desc(b + q * 2048, kK * 128, 1024) : smem_desc(b + q * 32, 16, 1024);
              mma_bf16(d, da, db, idesc, fresh);
              fresh = false;
            }
            mma_commit_pair(&empty[st]);
          }
          if (ok) mma_commit_pair(&done[n & 1]);
        }
      }
      if (!ok) {  // products in flight must end before the tensor memory is given back
        mma_commit(&drain);
        mbar_wait_bounded(&drain, 0, kDrainPolls, g.status);
      }
    }
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    uint32_t n = 0;
    bool ok = true;
    for (int i = pair; i < total; i += pairs) {
      const Tile t = tile_of<MODE>(s, i);
      float x[kHalf];
#pragma unroll
      for (int q = 0; q < kHalf; ++q) x[q] = 0.0f;
      for (int c = t.k0; c < t.k1; c += g.chunk, ++n) {
        ok = mbar_wait_bounded(&done[n & 1], n / 2 & 1, g.spin_limit, g.status);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t at = acc + (n & 1) * kN + half * kHalf + (static_cast<uint32_t>(quad * 32) << 16);
#pragma unroll
        for (int q = 0; q < kHalf; q += 64) {
          float y[64];
          tmem_ld32(at + q, y);
          tmem_ld32(at + q + 32, y + 32);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 64; ++j) {
            asm volatile("" : "+f"(y[j]));  // nothing uses y before the wait
            x[q + j] = fadd(x[q + j], y[j]);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(dsmem_addr(&taken[n & 1], 0));
      }
      if (!ok) break;
      epilogue<MODE>(g, valid, t, t.m0 + rank * kM + quad * 32 + lane, t.n0 + half * kHalf, x);
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // nothing signals or reads the other CTA's shared memory any more
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(acc, 512);
  }
}

// lse and loss of each token from its half tiles' sums; one warp a token.
__global__ void __launch_bounds__(256)
    ce_finish_kernel(int T, const int* place, const float2* part, int parts, const float* at_target, float* loss,
                     float* lse) {
  pdl_begin();
  const int t = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (t >= T) return;
  const int m = place[t];
  if (m < 0) {
    if (lane == 0) loss[t] = lse[t] = 0.0f;
    return;
  }
  float top = -INFINITY;
  for (int i = lane; i < parts; i += 32) top = fmaxf(top, part[static_cast<int64_t>(i) * T + m].x);
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
  float sum = 0.0f;
  for (int i = lane; i < parts; i += 32) {
    const float2 p = part[static_cast<int64_t>(i) * T + m];
    sum = fadd(sum, fmul(p.y, exp2f(fsub(p.x, top))));
  }
  for (int o = 16; o > 0; o >>= 1) sum = fadd(sum, __shfl_xor_sync(kFull, sum, o));
  if (lane == 0) {
    const float l = __fmaf_rn(top, kLn2, logf(sum));
    lse[t] = l;
    loss[t] = fsub(l, at_target[m]);
  }
}

// dh in the caller's type and order from the splits' sums; zero for tokens that
// do not count.
template <typename E>
__global__ void __launch_bounds__(256)
    ce_dh_out_kernel(int T, int64_t D, const int* place, const float* sum, int64_t lds, int splits, int64_t sum_split,
                     E* dh, int64_t lddh) {
  pdl_begin();
  for (int t = blockIdx.x; t < T; t += gridDim.x) {
    const int m = place[t];
    for (int64_t d = threadIdx.x; d < D; d += blockDim.x) {
      float x = 0.0f;
      if (m >= 0)
        for (int i = 0; i < splits; ++i) x = fadd(x, sum[i * sum_split + m * lds + d]);
      from_float(x, dh + t * lddh + d);
    }
  }
}

// ---------------------------------------------------------------------------
// Workspace and launches
// ---------------------------------------------------------------------------
size_t up(size_t x) { return (x + 255) / 256 * 256; }
int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The coefficients of a piece take 1 GiB at most (0.4 % of the memory; a shorter
// vocabulary piece makes smaller products and more launches).
constexpr int64_t kPieceBytes = int64_t{1} << 30;
constexpr int kMaxSplits = 8;

struct Layout {
  size_t head, row, target, place, at_target, part, lse, h, w, coef, sum, total;
  int parts, planes, splits;
  bool pack_w;
  int64_t piece, padded, Dp, lds, ldc;
};

// Parts of K for dh: full waves of the SMs for the least part sums.
int splits_for(int64_t T, int64_t D, int64_t piece) {
  constexpr int pairs = 76;  // of the 152 SMs
  const int64_t tiles = (T + kPair - 1) / kPair * ((D + kN - 1) / kN);
  const int64_t blocks = (piece + kK - 1) / kK;
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= kMaxSplits && s * 8 <= std::max<int64_t>(blocks, 8); ++s) {
    const double waves = static_cast<double>((tiles * s + pairs - 1) / pairs) / s * (1.0 + 0.02 * s);
    if (waves < least) {
      least = waves;
      best = s;
    }
  }
  return best;
}

Layout layout(int64_t T, int64_t D, int64_t V, bool bf16, bool grad, int64_t piece, int64_t ldw) {
  Layout l = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t p = at;
    at += up(bytes);
    return p;
  };
  l.planes = bf16 ? 1 : 3;
  l.pack_w = !bf16 || ldw < D || ldw % 8 != 0;
  l.padded = round_up(T, kPair);
  l.Dp = round_up(D, 8);
  l.parts = static_cast<int>((V + kHalf - 1) / kHalf);
  l.head = take(sizeof(Header));
  l.row = take(T * 4);
  l.target = take(T * 4);
  l.place = take(T * 4);
  l.at_target = take(T * 4);
  l.lse = take(T * 4);
  l.part = take(static_cast<size_t>(l.parts) * T * 8);
  l.h = take(static_cast<size_t>(l.planes) * l.padded * l.Dp * 2);
  l.w = take(l.pack_w ? static_cast<size_t>(l.planes) * V * l.Dp * 2 : 0);
  if (grad) {
    const int64_t most = std::max<int64_t>(kN, kPieceBytes / (l.padded * 2 * l.planes) / kN * kN);
    l.piece = std::min(V, piece > 0 ? piece : most);
    l.ldc = round_up(l.piece, kN);
    l.lds = round_up(D, 8);
    l.splits = kMaxSplits;
    l.coef = take(static_cast<size_t>(l.planes) * l.padded * l.ldc * 2);
    l.sum = take(static_cast<size_t>(splits_for(T, D, l.piece)) * l.padded * l.lds * 4);
  }
  l.total = at;
  return l;
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder() {
  static EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

// A map over [planes][rows][cols] bf16 with rows ld elements apart, read in boxes
// of 64 columns x box_rows rows; what lies outside reads as zero.
cudaError_t make_map(CUtensorMap* map, const void* base, int64_t cols, int64_t rows, int planes, int64_t ld,
                     int64_t plane, int box_rows) {
  const cuuint64_t size[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows),
                              static_cast<cuuint64_t>(planes)};
  const cuuint64_t stride[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(plane) * 2};
  const cuuint32_t box[3] = {kK, static_cast<cuuint32_t>(box_rows), 1}, step[3] = {1, 1, 1};
  const EncodeFn fn = encoder();
  if (fn == nullptr) return cudaErrorNotSupported;
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), size, stride, box, step,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? cudaSuccess
             : cudaErrorInvalidValue;
}

template <int MODE>
cudaError_t launch_gemm(const CUtensorMap& a, const CUtensorMap& b, const Gemm& g, int64_t tiles, int num_sms,
                        cudaStream_t s) {
  constexpr int smem = kStages * kStageBytes + 1024;
  const cudaError_t e = ensure_dynamic_smem(ce_gemm_kernel<MODE>, smem);
  if (e != cudaSuccess) return e;
  const unsigned grid = static_cast<unsigned>(2 * std::min<int64_t>(tiles, num_sms / 2));
  return launch_kernel(ce_gemm_kernel<MODE>, dim3(grid), dim3(kGemmThreads), smem, s, 2, a, b, g);
}

#define CE_TRY(expr)                      \
  do {                                    \
    const cudaError_t e_ = (expr);        \
    if (e_ != cudaSuccess) return e_;     \
  } while (0)

template <typename E>
cudaError_t run(const LinearCeArgs& a, int num_sms, cudaStream_t s) {
  constexpr bool bf16 = sizeof(E) == 2;
  constexpr int P = bf16 ? 1 : 3;
  const int T = static_cast<int>(a.T), D = static_cast<int>(a.D);
  const int64_t ldw = (reinterpret_cast<uintptr_t>(a.w) & 15) == 0 ? a.ldw : 0;
  const Layout l = layout(a.T, a.D, a.V, bf16, a.dw != nullptr, a.piece, ldw);
  char* ws = static_cast<char*>(a.ws);
  Header* head = reinterpret_cast<Header*>(ws + l.head);
  int* row = reinterpret_cast<int*>(ws + l.row);
  int* target = reinterpret_cast<int*>(ws + l.target);
  int* place = reinterpret_cast<int*>(ws + l.place);
  uint16_t* hp = reinterpret_cast<uint16_t*>(ws + l.h);
  uint16_t* wp = reinterpret_cast<uint16_t*>(ws + l.w);
  CE_TRY(launch_kernel(ce_scan_kernel, dim3(1), dim3(1024), 0, s, 0, a.targets, T, a.V, a.ignore, head, row, target,
                       place, a.status));
  auto pack_grid = [&](int64_t rows) {
    return dim3(static_cast<unsigned>(std::min<int64_t>((rows * (l.Dp / 8) + 255) / 256, num_sms * 16)));
  };
  CE_TRY(launch_kernel(ce_pack_kernel<E, P>, pack_grid(l.padded), dim3(256), 0, s, 0, static_cast<const E*>(a.h), a.ldh,
                       row, &head->valid, a.T, l.padded, D, static_cast<int>(l.Dp), hp));
  const void* w = a.w;
  int64_t wld = a.ldw;
  if (l.pack_w) {
    CE_TRY(launch_kernel(ce_pack_kernel<E, P>, pack_grid(a.V), dim3(256), 0, s, 0, static_cast<const E*>(a.w), a.ldw,
                         static_cast<const int*>(nullptr), static_cast<const int*>(nullptr), a.V, a.V, D,
                         static_cast<int>(l.Dp), wp));
    w = wp;
    wld = l.Dp;
  }
  const int64_t hplane = l.padded * l.Dp, wplane = l.pack_w ? a.V * l.Dp : a.V * wld;
  CUtensorMap h_rows, w_rows;  // K = D contiguous
  CE_TRY(make_map(&h_rows, hp, D, l.padded, P, l.Dp, hplane, kM));
  CE_TRY(make_map(&w_rows, w, D, a.V, P, wld, wplane, kM));
  Gemm g = {};
  g.head = head;
  g.row = row;
  g.target = target;
  g.T = T;
  g.D = D;
  g.terms = bf16 ? 1 : 6;
  g.spin_limit = a.spin_limit;
  g.status = a.status;
  // K blocks of an accumulator: 16 steps for the logits that the loss shows in
  // fp32, 32 for fp32 gradients, any number where results are rounded to bf16
  const int any = 1 << 30, few = 4, some = 8;
  const int64_t mt = l.padded / kPair, dt = (a.D + kN - 1) / kN;
  const float* lse = a.lse_in;
  if (a.loss != nullptr) {
    g.width = static_cast<int>(a.V);
    g.part = reinterpret_cast<float2*>(ws + l.part);
    g.at_target = reinterpret_cast<float*>(ws + l.at_target);
    float* out = a.lse != nullptr ? a.lse : reinterpret_cast<float*>(ws + l.lse);
    g.chunk = few;
    CE_TRY(launch_gemm<kLoss>(h_rows, w_rows, g, mt * ((a.V + kN - 1) / kN), num_sms, s));
    CE_TRY(launch_kernel(ce_finish_kernel, dim3((T + 7) / 8), dim3(256), 0, s, 0, T, place, g.part, l.parts, g.at_target,
                         a.loss, out));
    lse = out;
  }
  if (a.dw == nullptr) return cudaSuccess;
  g.lse = lse;
  g.gloss = a.gloss;
  g.coef = reinterpret_cast<uint16_t*>(ws + l.coef);
  g.ldc = l.ldc;
  g.coef_plane = l.padded * l.ldc;
  g.sum = reinterpret_cast<float*>(ws + l.sum);
  g.lds = l.lds;
  g.sum_split = l.padded * l.lds;
  g.splits = splits_for(a.T, a.D, l.piece);
  g.dw = a.dw;
  g.lddw = a.lddw;
  g.dw_bf16 = bf16;
  g.dw_wide = (a.lddw * sizeof(E)) % 32 == 0 && reinterpret_cast<uintptr_t>(a.dw) % 32 == 0;
  CUtensorMap w_cols, h_cols;  // K = vocabulary, tokens: boxes of 64 columns x 64 k
  CE_TRY(make_map(&w_cols, w, D, a.V, P, wld, wplane, kK));
  CE_TRY(make_map(&h_cols, hp, D, l.padded, P, l.Dp, hplane, kK));
  for (int64_t v0 = 0; v0 < a.V; v0 += l.piece) {
    const int width = static_cast<int>(std::min(l.piece, a.V - v0));
    const int64_t vt = (width + kN - 1) / kN;
    g.v0 = v0;
    g.width = width;
    g.first = v0 == 0;
    CUtensorMap c_rows, c_cols;
    CE_TRY(make_map(&c_rows, g.coef, width, l.padded, P, l.ldc, g.coef_plane, kM));
    CE_TRY(make_map(&c_cols, g.coef, width, l.padded, P, l.ldc, g.coef_plane, kK));
    g.chunk = bf16 ? any : few;
    CE_TRY(launch_gemm<kCoef>(h_rows, w_rows, g, mt * vt, num_sms, s));
    g.chunk = bf16 ? any : some;
    CE_TRY(launch_gemm<kDh>(c_rows, w_cols, g, mt * dt * g.splits, num_sms, s));
    CE_TRY(launch_gemm<kDw>(c_cols, h_cols, g, (width + kPair - 1) / kPair * dt, num_sms, s));
  }
  return launch_kernel(ce_dh_out_kernel<E>, dim3(static_cast<unsigned>(std::min<int64_t>(a.T, 4096))), dim3(256), 0, s, 0,
                       T, a.D, place, g.sum, l.lds, g.splits, g.sum_split, static_cast<E*>(a.dh), a.lddh);
}

}  // namespace

size_t linear_ce_workspace_bytes(int64_t T, int64_t D, int64_t V, int bf16, int grad, int64_t piece, int64_t ldw) {
  return layout(T, D, V, bf16 != 0, grad != 0, piece, ldw).total;
}

cudaError_t launch_linear_ce(const LinearCeArgs& a, int num_sms, cudaStream_t s) {
  return a.bf16 ? run<__nv_bfloat16>(a, num_sms, s) : run<float>(a, num_sms, s);
}

}  // namespace mpc
