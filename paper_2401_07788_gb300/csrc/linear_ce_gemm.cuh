// linear_ce_gemm.cuh -- the matrix products of the linear cross entropy on the
// tensor cores, with the softmax in their epilogues.
#pragma once

#include <cuda_bf16.h>

#include "tcgen05.cuh"

namespace mpc {
namespace {

constexpr int kM = 128;        // rows of a CTA's output tile (lanes of tensor memory)
constexpr int kPair = 2 * kM;  // rows of a CTA pair's output tile
constexpr int kN = 256;        // columns of an output tile
constexpr int kK = 64;         // K elements of a stage: 128 bytes, one swizzle row
constexpr int kStages = 6;    // of one plane; fp32 has kStages / 3 of three
constexpr int kBytesA = kM * kK * 2;
constexpr int kBytesB = kN / 2 * kK * 2;
constexpr int kStageBytes = kBytesA + kBytesB;
constexpr int kEpiWarps = 8;
constexpr int kStoreBytes = 4096;  // of an epilogue warp's stores of c
constexpr int kGemmThreads = (2 + kEpiWarps) * 32;
constexpr int kHalf = kN / 2;  // columns an epilogue warp takes
constexpr int kRun = 16;       // sorted tokens whose target gradients one CTA sums
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Header {
  int valid;   // tokens that count
  float mean;  // 1 / valid (0 when none counts)
  int redo;    // some token's exponentials are formed again (see kExp)
};

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

// ---------------------------------------------------------------------------
// The matrix products: C[m][n] = sum_k A[m][k] B[n][k] in 256 x 256 tiles.
//
// A persistent pair of CTAs on two SMs per tile, 128 rows each: every CTA copies
// its rows of A and half the rows of B, so an SM reads 32 KB from L2 for 2^20
// products (48 KB with a tile of its own).  Warp 0 copies operand tiles through
// tensor maps (six stages of 32 KB a CTA; for fp32 two stages with the three planes
// of both operands, which serve six plane products), one thread of the first CTA's warp
// 1 issues the products of both, eight warps a CTA take the finished tile from
// tensor memory.  Two
// accumulators of 256 columns fill the tensor memory, so a tile's epilogue runs
// under the next tile's products.
//
// kLoss   A = h [valid][D],  B = w [V][D]: a tile's logits become, for each token
//         and half tile, their largest and the sum of exponentials over it, the
//         target's logit left out and kept by itself.
// kExp    the same for a training step that keeps the exponentials: with a reference
//         ref[t] near the logits, e = 2^(l log2e - ref) rounded to bf16 planes (its
//         relative error is that of a rounded probability) and their sums.  The
//         factor that makes them coefficients is applied where it is exact: to dh's
//         sums, and to h for dw.  e of the target is 0: its coefficient p - 1 goes its
//         own way in fp32.  ref is the target's logit, so a sum is out of range only
//         for a token with a loss over 27; such tokens set
//         a flag, take their largest logit as ref, and a second launch of the kernel
//         (which returns at once without a flag) forms their row tiles again.
// kCoef   the logits' products again, when lse is known: the coefficients c of a
//         piece of the vocabulary, rounded to bf16 planes.  In bf16 the target's c,
//         g (p - 1), is no entry to be rounded: it is a sum's largest term for most
//         tokens, and where p is small the c of all tokens lie side by side, off in
//         the same direction by up to 2^-8 (0.05 % of dh and dw at 600 x 64 x 300).
//         Up to 256 tokens it goes its own way in fp32 (`apart`); beyond, a token's
//         coefficients are taken over g (1 - p) (`over`): -1 for the target, and the
//         factor is applied in fp32 to dh's sums and, with one rounding an element,
//         to h for dw.
// kDh     A = c [valid][piece], B = w^T [D][piece]: dh, K split over several CTAs
//         where there are few tiles, each split's sum kept in fp32.
// kDw     A = c^T [piece][valid], B = h^T [D][valid]: dw of the piece, or as for dh
//         the fp32 sums of parts of K where the vocabulary has few tiles.
//
// An accumulator adds each product step of 16 with truncation towards zero, each of
// its terms to about 2^-25 of the largest.  Measured on logits: random signs lose
// 7e-10 of the terms' magnitudes a step, 48 steps of one size and sign 1.2e-8 of the
// sum a step; steps added to a value that is large beside them 4e-8 of it a step for
// one term, 1.7e-7 for 16, which is the bound that the chunks go by.  So an
// accumulator sums a chunk of K blocks only (see run; within a block of fp32 the
// smallest plane products first), and the epilogue adds the chunks in fp32 with
// rounding to nearest; two accumulators in turn keep the products running.
//
// Measured at 7373 tokens that count x 768 x 50257 in bf16 (0.57 TFLOP each): kExp
// 380 us (302 without its epilogue, 350 without its stores: eight warps' latency and
// the 0.7 GB of c), kDh 355, kDw 340 (1.6 to 1.7 PFLOP/s; cuBLAS does 1.7 for seconds,
// 1.9 in a burst; the tensor pipe is 74 % busy at 1.78 GHz).  2048 tokens in fp32
// (0.95 TFLOP of plane products each): 530, 467 and 500 us.
//
// Operands whose K is not the contiguous axis (w^T, c^T, h^T) are read as they
// are: rows of 64 M/N-elements, and the product's descriptors say so.
// ---------------------------------------------------------------------------
enum Mode { kLoss, kExp, kCoef, kDh, kDw };

struct Gemm {
  const Header* head;
  const int* row;       // token of a listed row
  const int* target;
  int T;                // tokens (upper bound of the list)
  int D;
  int width;            // vocabulary entries of the piece
  int64_t v0;           // its first one
  int tile_n;           // columns of a tile: 64 (dh, dw), 128 or 256
  int chunk;            // K blocks that one accumulator sums (see ce_gemm_kernel)
  int splits;           // kDh, kDw: parts of K
  int first;            // kDh: the piece that starts the sums
  float2* part;         // kLoss, kExp: [half tile][T] (largest logit, sum), base 2
  float* at_target;     // kLoss, kExp: [T]
  const float* ref;     // kExp: [T]
  const int* redo;      // kExp: nullptr, or the row tiles to form again
  const int* seg_first; // kDw: nullptr, or per entry 1 + the first sorted token with that target (0: none)
  const float* seg_sum; // kDw: [T][lds], the sum of its tokens' gradients at that position
  const float* lse;     // kCoef: [T] by token
  const float* gloss;   // kCoef: [T] by token, or nullptr for the mean
  const float* loss;    // kCoef: [T] by token where the forward pass gave it, or nullptr
  int apart;            // kCoef: the target's c goes its own way in fp32
  const float* over;    // kCoef: nullptr, or [T] 1 / (1 - p): c over g (1 - p)
  float* sum;           // kDh, kDw in parts (else nullptr): [split][rows][lds]
  int64_t lds, sum_split;
  void* dw;             // kDw
  int64_t lddw;
  int dw_bf16, dw_wide; // type; rows and base suit 32-byte stores
  uint32_t spin_limit;
  unsigned* status;
};

// Plane pair of a product, smallest products first.
template <int PLANES>
__device__ __forceinline__ void term_planes(int t, int* a, int* b) {
  if (PLANES == 1) {
    *a = *b = 0;
  } else {  // (2,0) (0,2) (1,1) (1,0) (0,1) (0,0), two bits each
    *a = (0x052 >> (2 * t)) & 3;
    *b = (0x118 >> (2 * t)) & 3;
  }
}

// What an epilogue needs of its row, loaded before the tile is waited for.
struct Row {
  int target;
  float ref;  // kExp
  int first;  // kDw: seg_first
};

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
  s.n_tiles = (n + g.tile_n - 1) / g.tile_n;
  s.blocks = (k + kK - 1) / kK;
  s.splits = MODE == kDh || MODE == kDw ? g.splits : 1;
  return s;
}

// Order of the tiles: those that run at the same time share operands in L2.  For
// the logits all tokens pass one stretch of the vocabulary; for dh and dw the
// columns of one row tile of c run together, so that c is read from HBM once.
template <int MODE>
__device__ __forceinline__ Tile tile_of(const Gemm& g, const Shape& s, int i) {
  Tile t;
  if (MODE == kLoss || MODE == kExp || MODE == kCoef) {
    t.m0 = i % s.m_tiles * kPair;
    t.n0 = i / s.m_tiles * g.tile_n;
    t.split = 0;
  } else {
    t.n0 = i % s.n_tiles * g.tile_n;
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

// A warp's 32 rows of a half tile as bf16 planes of the coefficients, by tensor-map
// stores of 64 columns from its 4 KB of shared memory: a row's 16-byte groups lie
// swizzled, so the lanes' writes meet in no bank, and HBM gets whole lines (one
// 32-byte store a lane reached 32 lines an instruction).  What lies outside the
// piece is not written.
template <int PLANES>
__device__ __forceinline__ void store_planes(const Gemm& g, const CUtensorMap* map, uint8_t* buf, int m, int n0,
                                             float (&x)[kHalf]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int h = 0; h < kHalf; h += 64) {
    if (n0 + h < g.width) {
#pragma unroll
      for (int p = 0; p < PLANES; ++p) {
        uint32_t u[32];
#pragma unroll
        for (int q = 0; q < 32; ++q) {
          float &lo = x[h + 2 * q], &hi = x[h + 2 * q + 1];
          u[q] = pack_bf16(lo, hi);
          if (p + 1 < PLANES) {
            lo = fsub(lo, __uint_as_float(u[q] << 16));
            hi = fsub(hi, __uint_as_float(u[q] & 0xffff0000u));
          }
        }
        if (lane == 0) bulk_wait_read();
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 8; ++c)
          *reinterpret_cast<uint4*>(buf + lane * 128 + ((c ^ (lane & 7)) * 16)) =
              make_uint4(u[4 * c], u[4 * c + 1], u[4 * c + 2], u[4 * c + 3]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tensor_s2g(map, n0 + h, m - lane, p, buf);
      }
    }
  }
}

// A warp's 32 rows of a half tile of dw whose rows start anywhere: 128 bytes of each
// row at a time in shared memory (rows 33 words apart).  Of a row, a lane of eight
// takes one 16-byte group of the destination, on its own alignment; the 16 bytes
// before the first and after the last whole group go element by element in a second
// pass.  (Element stores throughout, two rows an instruction: 68 us against 49 at 149
// x 788 x 31773 in bf16, where rows on 32 bytes take 33.)
template <int SIZE>
__device__ __forceinline__ void store_anywhere(const Gemm& g, int m, int n0, int cols, const float (&x)[kHalf],
                                               uint32_t* scratch) {
  constexpr int kSeg = 128 / SIZE, kEach = 16 / SIZE;
  const int lane = threadIdx.x & 31, m0 = m - lane, rows = min(g.width - m0, 32);
  const int64_t ld = g.lddw * SIZE;
  uint8_t* base = static_cast<uint8_t*>(g.dw) + (g.v0 + m0) * ld + static_cast<int64_t>(n0) * SIZE;
#pragma unroll
  for (int j = 0; j < kHalf; j += kSeg) {
    if (j < cols) {
      __syncwarp();
#pragma unroll
      for (int q = 0; q < 32; ++q)
        scratch[lane * 33 + q] = SIZE == 4 ? __float_as_uint(x[j + q % kSeg])
                                           : pack_bf16(x[j + 2 * q % kSeg], x[j + (2 * q + 1) % kSeg]);
      __syncwarp();
      uint8_t* seg = base + j * SIZE;
      if (cols - j >= kSeg) {
        int r = lane >> 3;
        uint8_t* to = seg + r * ld;
#pragma unroll 2
        for (; r < rows; r += 4, to += 4 * ld) {
          const int lead = (16 - static_cast<int>(reinterpret_cast<uintptr_t>(to))) & 15;  // bytes before a whole group
          const int off = lead + 16 * (lane & 7);
          if (off + 16 <= 128) {
            const uint32_t* w = scratch + r * 33 + off / 4;
            uint4 v;
            if (SIZE == 4 || (off & 2) == 0) {
              v = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
              const uint32_t w1 = w[1], w2 = w[2], w3 = w[3];
              v = make_uint4(__byte_perm(w[0], w1, 0x5432), __byte_perm(w1, w2, 0x5432), __byte_perm(w2, w3, 0x5432),
                             __byte_perm(w3, w[4], 0x5432));
            }
            *reinterpret_cast<uint4*>(to + off) = v;
          }
        }
#pragma unroll
        for (int i = lane; i < 32 * kEach; i += 32) {
          const int q = i / kEach;
          uint8_t* row = seg + q * ld;
          const int lead = (16 - static_cast<int>(reinterpret_cast<uintptr_t>(row))) & 15;
          int at = i % kEach * SIZE;
          if (at >= lead) at += 112;  // after the 7 whole groups
          if (lead != 0 && q < rows) {
            const uint32_t* from = scratch + q * 33;
            if (SIZE == 4) *reinterpret_cast<uint32_t*>(row + at) = from[at / 4];
            else *reinterpret_cast<uint16_t*>(row + at) = reinterpret_cast<const uint16_t*>(from)[at / 2];
          }
        }
      } else {  // the last columns: neighbouring lanes neighbouring elements
        const int left = cols - j;
        for (int r = 0; r < rows; ++r)
          for (int c = lane; c < left; c += 32) {
            const uint32_t* from = scratch + r * 33;
            if (SIZE == 4) *reinterpret_cast<uint32_t*>(seg + r * ld + c * 4) = from[c];
            else *reinterpret_cast<uint16_t*>(seg + r * ld + c * 2) = reinterpret_cast<const uint16_t*>(from)[c];
          }
      }
    }
  }
}

// One lane's row of a half tile: x[j] = C[m][n0 + j], j < 128.
template <int MODE, int PLANES>
__device__ __forceinline__ void epilogue(const Gemm& g, int valid, const Tile& t, int m, int n0, const Row& row, float (&x)[kHalf],
                                         uint32_t* scratch, const CUtensorMap* map_c, uint8_t* buf) {
  if (MODE == kLoss || MODE == kExp) {
    const int cols = min(g.width - n0, kHalf);
    if (MODE == kLoss && (cols <= 0 || m >= valid)) return;
    const bool live = m < valid;
    if (live && cols > 0) {
      const int y = row.target - n0;
      if (cols < kHalf) {
#pragma unroll
        for (int j = 0; j < kHalf; ++j)
          if (j >= cols) x[j] = -INFINITY;
      }
      if (y >= 0 && y < cols) {  // out of the sum: a small loss is the logarithm of 1 + the others
        float v = x[0];
#pragma unroll
        for (int j = 1; j < kHalf; ++j) v = j == y ? x[j] : v;
        g.at_target[m] = v;
#pragma unroll
        for (int j = 0; j < kHalf; ++j)
          if (j == y) x[j] = -INFINITY;
      }
      // base 2 throughout: exp(l - top) = 2^(l log2e - top log2e), one rounding in the exponent
      float tops[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
      for (int j = 4; j < kHalf; ++j) tops[j & 3] = fmaxf(tops[j & 3], x[j]);
      const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
      const float base = fmul(top, kLog2e);
      const float shift = MODE == kExp ? -row.ref : base == -INFINITY ? 0.0f : -base;
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < kHalf; ++j) {
        const float e = exp2_approx(__fmaf_rn(x[j], kLog2e, shift));
        sum[j & 3] = fadd(sum[j & 3], e);
        if (MODE == kExp) x[j] = e;
      }
      g.part[static_cast<int64_t>(n0 / kHalf) * g.T + m] =
          make_float2(base, fadd(fadd(sum[0], sum[1]), fadd(sum[2], sum[3])));
    }
    if (MODE == kExp) {
      if (!live) {
#pragma unroll
        for (int j = 0; j < kHalf; ++j) x[j] = 0.0f;
      }
      store_planes<PLANES>(g, map_c, buf, m, n0, x);
    }
  } else if (MODE == kCoef) {
    const bool live = m < valid;
    float shift = 0.0f, scale = 0.0f, at_y = 0.0f;
    int y = -1;
    if (live) {
      const int token = g.row[m];
      const float lse = g.lse[token];
      const float weight = g.over != nullptr ? g.over[m] : g.gloss != nullptr ? g.gloss[token] : g.head->mean;
      // what the rounding of lse log2e leaves out goes into the factor
      shift = fmul(lse, -kLog2e);
      scale = fmul(weight, exp2f(-__fmaf_rn(lse, kLog2e, shift)));
      y = static_cast<int>(g.target[m] - g.v0 - n0);
      if (y >= 0 && y < kHalf && !g.apart) {  // p - 1 from the loss, not as a difference
        float v = x[0];
#pragma unroll
        for (int j = 1; j < kHalf; ++j) v = j == y ? x[j] : v;
        at_y = g.over != nullptr ? -1.0f : fmul(weight, expm1f(g.loss != nullptr ? -g.loss[token] : fsub(v, lse)));
      }
    }
#pragma unroll
    for (int j = 0; j < kHalf; ++j)
      x[j] = live ? fmul(scale, exp2_approx(__fmaf_rn(x[j], kLog2e, shift))) : 0.0f;
    if (y >= 0 && y < kHalf) {
#pragma unroll
      for (int j = 0; j < kHalf; ++j)
        if (j == y) x[j] = at_y;
    }
    store_planes<PLANES>(g, map_c, buf, m, n0, x);
  } else if (MODE == kDh || g.sum != nullptr) {
    if (m >= (MODE == kDh ? valid : g.width)) return;
    float* out = g.sum + t.split * g.sum_split + m * g.lds + n0;
    const int cols = min(static_cast<int>(g.lds) - n0, g.tile_n);
#pragma unroll
    for (int j = 0; j < kHalf; j += 8) {
      if (j < cols) {
        uint32_t u[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if (MODE == kDh && !g.first) x[j + q] = fadd(x[j + q], out[j + q]);
          u[q] = __float_as_uint(x[j + q]);
        }
        st_v8(out + j, u);
      }
    }
  } else {
    if (row.first > 0) {  // the tokens whose target this entry is
      const float* add = g.seg_sum + (row.first - 1) * g.lds + n0;
#pragma unroll
      for (int j = 0; j < kHalf; j += 4) {
        if (n0 + j < g.D) {
          const float4 v = *reinterpret_cast<const float4*>(add + j);
          x[j] = fadd(x[j], v.x);
          x[j + 1] = fadd(x[j + 1], v.y);
          x[j + 2] = fadd(x[j + 2], v.z);
          x[j + 3] = fadd(x[j + 3], v.w);
        }
      }
    }
    const int cols = min(g.D - n0, g.tile_n);
    if (g.dw_wide) {
      if (m >= g.width) return;
      const int64_t at = (g.v0 + m) * g.lddw + n0;
      if (g.dw_bf16) {
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(g.dw) + at;
#pragma unroll
        for (int j = 0; j < kHalf; j += 16) {
          if (j + 16 <= cols) {
            uint32_t u[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) u[q] = pack_bf16(x[j + 2 * q], x[j + 2 * q + 1]);
            st_v8(out + j, u);
          } else {
#pragma unroll
            for (int q = 0; q < 16; ++q)
              if (j + q < cols) out[j + q] = __float2bfloat16_rn(x[j + q]);
          }
        }
      } else {
        float* out = static_cast<float*>(g.dw) + at;
#pragma unroll
        for (int j = 0; j < kHalf; j += 8) {
          if (j + 8 <= cols) {
            uint32_t u[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) u[q] = __float_as_uint(x[j + q]);
            st_v8(out + j, u);
          } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
              if (j + q < cols) out[j + q] = x[j + q];
          }
        }
      }
    } else {
      if (g.dw_bf16) store_anywhere<2>(g, m, n0, cols, x, scratch);
      else store_anywhere<4>(g, m, n0, cols, x, scratch);
    }
  }
}

template <int MODE>
__device__ __forceinline__ bool skipped(const Gemm& g, const Tile& t) {
  return MODE == kExp && g.redo != nullptr && g.redo[t.m0 / kPair] == 0;
}

// Columns of a tile that the product forms: a multiple of 16.  Each CTA of the
// pair holds half of them as rows of B.
__device__ __forceinline__ int tile_cols(const Gemm& g, int cols, int n0) {
  return min((cols - n0 + 15) / 16 * 16, g.tile_n);
}

template <int MODE, int PLANES>
__global__ void __launch_bounds__(kGemmThreads, 1)
    ce_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_c, const __grid_constant__ Gemm g) {
  constexpr bool A_MN = MODE == kDw, B_MN = MODE == kDh || MODE == kDw;
  extern __shared__ uint8_t raw[];
  // full and taken are used in the first CTA, for both; empty and done in each
  __shared__ uint64_t full[kStages], empty[kStages], done[2], taken[2], drain;
  __shared__ uint32_t tmem;
  __shared__ uint32_t scratch[MODE == kDw ? kEpiWarps * 32 * 33 : 1];
  uint8_t* stage0 = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_rank());
  if (MODE == kExp && g.redo != nullptr) {
    pdl_begin();
    if (g.head->redo == 0) return;
  }
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
  cluster_sync();  // both CTAs have started: the allocation is the pair's
  if (warp == 1) tmem_alloc(&tmem, 512);
  tc_fence_before();
  cluster_sync();
  tc_fence_after();
  const uint32_t acc = tmem;
  pdl_begin();
  const int valid = g.head->valid;
  const Shape s = shape_of<MODE>(g, valid);
  const int total = s.total();
  const int cols = MODE == kDh || MODE == kDw ? g.D : g.width;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  constexpr uint32_t stages = kStages / PLANES;

  if (warp == 0) {
    if (lane == 0) {
      fence_proxy_async_all();  // operands that earlier kernels wrote
      uint32_t it = 0;
      bool ok = true;
      // a CTA's rows of B in a stage: half the tile's, in blocks of 64 where they are columns
      const int b_blocks = (g.tile_n / 2 + 63) / 64;
      const uint32_t bytes = 2 * PLANES * (kBytesA + (B_MN ? b_blocks * kK * 128 : g.tile_n / 2 * kK * 2));
      for (int i = pair; i < total && ok; i += pairs) {
        const Tile t = tile_of<MODE>(g, s, i);
        if (skipped<MODE>(g, t)) continue;
        const int m0 = t.m0 + rank * kM, n0 = t.n0 + rank * (tile_cols(g, cols, t.n0) / 2);
        for (int kb = t.k0; kb < t.k1; ++kb, ++it) {
          const int st = it % stages;
          ok = mbar_wait_bounded(&empty[st], (it / stages & 1) ^ 1, g.spin_limit, g.status);
          if (!ok) break;
          const uint32_t bar = dsmem_addr(&full[st], 0);
          if (rank == 0) mbar_arrive_expect_tx(&full[st], bytes);
#pragma unroll
          for (int p = 0; p < PLANES; ++p) {
            uint8_t* a = stage0 + (st * PLANES + p) * kStageBytes;
            uint8_t* b = a + kBytesA;
            if (A_MN) {
#pragma unroll
              for (int q = 0; q < kM / 64; ++q) tensor_g2s(a + q * kK * 128, &map_a, m0 + q * 64, kb * kK, p, bar);
            } else {
              tensor_g2s(a, &map_a, kb * kK, m0, p, bar);
            }
            if (B_MN) {
              const int k_at = kb * kK + (MODE == kDh ? static_cast<int>(g.v0) : 0);
              for (int q = 0; q < b_blocks; ++q) tensor_g2s(b + q * kK * 128, &map_b, n0 + q * 64, k_at, p, bar);
            } else {
              tensor_g2s(b, &map_b, kb * kK, static_cast<int>(g.v0) + n0, p, bar);
            }
          }
        }
      }
      // Copies in flight must land before either CTA leaves (the cluster barrier
      // below).  The first CTA's barriers count both CTAs' copies.  The second CTA knows
      // its own by the products that read them, which have not been formed where the
      // first one gave up: then it gives them a millisecond.
      if (rank == 0) {
        for (uint32_t i = it > stages ? it - stages : 0; i < it; ++i)
          mbar_wait_bounded(&full[i % stages], i / stages & 1, kDrainPolls, g.status);
      } else {
        for (uint32_t i = it > stages ? it - stages : 0; i < it && ok; ++i)
          ok = mbar_wait_bounded(&empty[i % stages], i / stages & 1, g.spin_limit, g.status);
        if (!ok) {
          const uint64_t until = global_ns() + 1000000;
          while (global_ns() < until) __nanosleep(1000);
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, n = 0;
      bool ok = true;
      for (int i = pair; i < total && ok; i += pairs) {
        const Tile t = tile_of<MODE>(g, s, i);
        if (skipped<MODE>(g, t)) continue;
        const uint32_t idesc = mma_desc(kPair, tile_cols(g, cols, t.n0), A_MN, B_MN);
        for (int c = t.k0; c < t.k1 && ok; c += g.chunk, ++n) {
          ok = mbar_wait_bounded(&taken[n & 1], (n / 2 & 1) ^ 1, g.spin_limit, g.status);
          tc_fence_after();
          const uint32_t d = acc + (n & 1) * kN;
          bool fresh = true;
          const int steps = min(g.chunk, t.k1 - c);
          for (int k = 0; k < steps; ++k, ++it) {
            const int st = it % stages;
            ok = mbar_wait_bounded(&full[st], it / stages & 1, g.spin_limit, g.status);
            if (!ok) break;
            tc_fence_after();
            const uint32_t base = smem_addr(stage0 + st * PLANES * kStageBytes);
#pragma unroll
            for (int term = 0; term < (PLANES == 1 ? 1 : 6); ++term) {
              int pa, pb;
              term_planes<PLANES>(term, &pa, &pb);
              const uint32_t a = base + pa * kStageBytes, b = base + pb * kStageBytes + kBytesA;
#pragma unroll
              for (int q = 0; q < kK / 16; ++q) {
                // 16 K-elements on: 32 bytes along a row, or 16 rows of 128 bytes
                const uint64_t da = A_MN ? smem_desc(a + q * 2048, kK * 128, 1024) : smem_desc(a + q * 32, 16, 1024);
                const uint64_t db = B_MN ? smem_desc(b + q * 2048, kK * 128, 1024) : smem_desc(b + q * 32, 16, 1024);
                mma_bf16(d, da, db, idesc, fresh);
                fresh = false;
              }
            }
            mma_commit_pair(&empty[st]);
          }
          if (ok) mma_commit_pair(&done[n & 1]);
        }
      }
      // products in flight must end before the tensor memory and the stages are given
      // back, also where an epilogue that gave up no longer waits for them
      mma_commit(&drain);
      mbar_wait_bounded(&drain, 0, kDrainPolls, g.status);
    }
  } else {
    const int quad = warp & 3, half = (warp - 2) >> 2;
    uint32_t n = 0;
    bool ok = true;
    for (int i = pair; i < total; i += pairs) {
      const Tile t = tile_of<MODE>(g, s, i);
      if (skipped<MODE>(g, t)) continue;
      const int m = t.m0 + rank * kM + quad * 32 + lane;
      Row row = {-1, 0.0f, 0};
      if (MODE == kDw && g.seg_first != nullptr && m < g.width) row.first = g.seg_first[g.v0 + m];
      if ((MODE == kLoss || MODE == kExp) && m < valid) {
        row.target = g.target[m];
        if (MODE == kExp) row.ref = g.ref[m];
      }
      float x[kHalf];
      if (t.k0 == t.k1) {
#pragma unroll
        for (int q = 0; q < kHalf; ++q) x[q] = 0.0f;
      }
      for (int c = t.k0; c < t.k1; c += g.chunk, ++n) {
        ok = mbar_wait_bounded(&done[n & 1], n / 2 & 1, g.spin_limit, g.status);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tc_fence_after();
        if (half * kHalf >= g.tile_n) {  // a narrow tile: the first four warps take it
          if (lane == 0) mbar_arrive_cluster(dsmem_addr(&taken[n & 1], 0));
          continue;
        }
        const uint32_t at = acc + (n & 1) * kN + half * kHalf + (static_cast<uint32_t>(quad * 32) << 16);
        if (c == t.k0) {
#pragma unroll
          for (int q = 0; q < kHalf; q += 32) tmem_ld32(at + q, x + q);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < kHalf; ++j) asm volatile("" : "+f"(x[j]));  // nothing uses x before the wait
        } else {
#pragma unroll
          for (int q = 0; q < kHalf; q += 64) {
            float y[64];
            tmem_ld32(at + q, y);
            tmem_ld32(at + q + 32, y + 32);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 64; ++j) {
              asm volatile("" : "+f"(y[j]));
              x[q + j] = fadd(x[q + j], y[j]);
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(dsmem_addr(&taken[n & 1], 0));
      }
      if (!ok) break;
      if (half * kHalf >= g.tile_n) continue;
      epilogue<MODE, PLANES>(g, valid, t, m, t.n0 + half * kHalf, row, x, scratch + (MODE == kDw ? (warp - 2) * 32 * 33 : 0),
                             &map_c, stage0 + kStages * kStageBytes + (warp - 2) * kStoreBytes);
    }
  }
  if ((MODE == kExp || MODE == kCoef) && lane == 0) bulk_wait();
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // nothing signals or reads the other CTA's shared memory any more
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(acc, 512);
  }
}

}  // namespace
}  // namespace mpc
