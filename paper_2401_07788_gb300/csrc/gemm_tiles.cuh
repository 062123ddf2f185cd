// gemm_tiles.cuh -- what the matrix products on the tensor cores share: tile sizes,
// operands in bf16 planes, tensor maps, and the choice of tiles.
#pragma once

#include <algorithm>
#include <cuda_bf16.h>

#include "tcgen05.cuh"

namespace mpc {
namespace {

constexpr int kM = 128;        // rows of a CTA's output tile (lanes of tensor memory)
constexpr int kPair = 2 * kM;  // rows of a CTA pair's output tile
constexpr int kN = 256;        // columns of an output tile
constexpr int kK = 64;         // K elements of a stage: 128 bytes, one swizzle row
constexpr int kBytesA = kM * kK * 2;
constexpr int kBytesB = kN / 2 * kK * 2;
constexpr int kStageBytes = kBytesA + kBytesB;
constexpr int kEpiWarps = 8;
constexpr int kGemmThreads = (2 + kEpiWarps) * 32;
constexpr int kHalf = kN / 2;  // columns an epilogue warp takes

// ---------------------------------------------------------------------------
// Operands in bf16 planes.  A bf16 tensor is one plane.  An fp32 x is the sum of
// three, x0 = bf16(x), x1 = bf16(x - x0), x2 = bf16(x - x0 - x1) (24 bits, down
// to bf16's smallest number 2^-133, which entries below 2^-110 reach), and a
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

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  uint32_t u;
  memcpy(&u, &p, 4);
  return u;
}

// Columns of a tile that the product forms: a multiple of 16.  Each CTA of the
// pair holds half of them as rows of B.
__device__ __forceinline__ int tile_cols(int cols, int n0, int tile_n) { return min((cols - n0 + 15) / 16 * 16, tile_n); }

template <typename E>
__device__ __forceinline__ void planes_of(E x, uint16_t (&p)[3]);
template <>
__device__ __forceinline__ void planes_of<float>(float x, uint16_t (&p)[3]) { split(x, p); }
template <>
__device__ __forceinline__ void planes_of<__nv_bfloat16>(__nv_bfloat16 x, uint16_t (&p)[3]) {
  p[0] = __bfloat16_as_ushort(x);
}

// Eight elements from p on; those from `left` on are zero.
template <typename E>
__device__ __forceinline__ void load8(const E* p, int left, bool wide, E (&x)[8]) {
  if (wide && left >= 8) {
    uint4 u[sizeof(E) / 2];
#pragma unroll
    for (int k = 0; k < static_cast<int>(sizeof(E)) / 2; ++k) u[k] = reinterpret_cast<const uint4*>(p)[k];
    memcpy(x, u, sizeof(x));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? p[j] : E(0.0f);
  }
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

template <int P>
__device__ __forceinline__ void store_planes8(uint16_t* out, int64_t plane, const uint16_t (&p)[8][3]) {
#pragma unroll
  for (int k = 0; k < P; ++k) {
    uint4 u;
    u.x = p[0][k] | static_cast<uint32_t>(p[1][k]) << 16;
    u.y = p[2][k] | static_cast<uint32_t>(p[3][k]) << 16;
    u.z = p[4][k] | static_cast<uint32_t>(p[5][k]) << 16;
    u.w = p[6][k] | static_cast<uint32_t>(p[7][k]) << 16;
    *reinterpret_cast<uint4*>(out + k * plane) = u;
  }
}
// ---------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------
size_t up(size_t x) { return (x + 255) / 256 * 256; }
int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// Widths of tiles, and parts of K, by an estimate of the products' time in
// cycles: waves of tiles over the SM pairs, a K block of a tile bound by its copies
// from L2 (about 60 bytes a cycle an SM: in bf16 546 cycles for 256 columns, 410
// for 128, 341 for 64) or its products (512, 256, 128; in fp32 six times as many on
// three times the bytes), an epilogue a tile, and for each part its sums written
// and read once more.
constexpr int kPairs = 76;  // of the 152 SMs

struct Plan {
  int tile_n, splits;
};

Plan plan_tiles(int64_t m, int64_t n, int64_t blocks, int planes, int narrowest, int most_splits) {
  Plan best = {kN, 1};
  double least = 1e300;
  const int64_t mt = (m + kPair - 1) / kPair;
  for (int tn = kN; tn >= narrowest; tn /= 2) {
    const int64_t nt = (n + tn - 1) / tn;
    const double copies = planes * (kBytesA + tn / 2 * kK * 2) / 60.0, products = (planes == 1 ? 2.0 : 12.0) * tn;
    const double step = std::max(copies, products), end = 1000.0 + 3000.0 * tn / kN;
    for (int s = 1; s <= most_splits && s <= std::max<int64_t>(blocks, 1); ++s) {
      const int64_t waves = (mt * nt * s + kPairs - 1) / kPairs;
      const double sums = s > 1 ? static_cast<double>(s) * m * n * 8.0 / 3500.0 : 0.0;
      const double cost = waves * (((blocks + s - 1) / s) * step + end) + sums;
      if (cost < 0.98 * least) {
        least = cost;
        best = Plan{tn, s};
      }
    }
  }
  return best;
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

// A map over [planes][rows][cols] bf16 with rows ld elements apart, in boxes
// of 64 columns x box_rows rows; what lies outside reads as zero and is not written.
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

}  // namespace
}  // namespace mpc
