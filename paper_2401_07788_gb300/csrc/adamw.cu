// adamw.cu -- the optimiser step of a pipeline stage: AdamW over many tensors
// in one launch, its states in fp32 or in 8-bit codes, and the global norm of
// the gradients that the step clips by.
//
// Mathematics (decoupled weight decay; every operation one fp32 round-to-nearest
// operation in this order, no contraction):
//   g <- g * min(1, max_norm / (norm + 1e-6))            (when a norm is given)
//   m <- b1 m + (1-b1) g;   v <- b2 v + ((1-b2) g) g
//   p <- p (1 - lr wd) - (lr / (1-b1^t)) * (m / (sqrt(v) / sqrt(1-b2^t) + eps))
// 8-bit states: blocks of 256 consecutive entries of a tensor share one fp32
// scale s, the block's largest |m| (or v).  A code c stands for
//   m: sign(c) (c/127)^2 s, c in -127..127;      v: (c/255)^4 s, c in 0..255.
// The squares spend the codes on small values: the least non-zero |m| is s/16129,
// the least non-zero sqrt(v) is sqrt(s)/65025.  The code is the nearest one, for
// m in m/s and for v in sqrt(v/s) (what the step divides by); a v > 0 never gets
// code 0, so that a small v cannot turn into a division by eps alone.  The step
// itself uses the m and v of before the coding.  No code stands for NaN: a block
// that has one gets the scale NaN, and all of it stands for NaN from then on.
//
// What bounds it: memory.  fp32 states move 28 bytes an entry (p, m, v read and
// written, g read).  The work is laid out over chunks of 2048 entries that never
// straddle two tensors: a CTA of 256 threads takes a contiguous range of chunks
// of the whole list, a warp 256 entries, a lane 8 consecutive ones (32-byte
// accesses in fp32; a warp's entries are one 8-bit block, so a block's largest is one warp
// reduction).  The list travels as a kernel argument: no copy to the device
// precedes the launch, and a captured graph holds it by value.  Measured on 153M
// entries: fp32 states 650 us (6.6 TB/s), 8-bit states with bf16 gradients and a
// bf16 copy 405 us (16 bytes an entry, 6.1 TB/s), their decoding 257 us (6.0 TB/s),
// the norm 108 us (5.7 TB/s).
#include <algorithm>
#include <cmath>
#include <cuda_bf16.h>

#include "common.cuh"
#include "kernels.h"
#include "launch_util.h"

namespace mpc {
namespace {

constexpr int kThreads = 256;
constexpr int kLane = 8;                   // entries a lane holds
constexpr int kChunk = kThreads * kLane;   // entries a CTA takes at a time

struct Entry {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* sm;
  float* sv;
  void* copy;
  int64_t n;
  float keep;  // 1 - lr wd
  float step;  // lr / (1 - b1^t)
  int first;   // the tensor's first chunk in the launch
  int wide;    // every pointer is on 32 bytes
};

template <int N>
struct Table {
  Entry e[N];
  int count;
  int chunks;
};

// Table sizes: the small one keeps the kernel arguments under 4 KB (a launch
// then costs what any other does), the large one fills the 32 KB limit.
constexpr int kSmallTable = 48;
constexpr int kLargeTable = 400;
static_assert(sizeof(Table<kSmallTable>) + 64 <= 4096, "");
static_assert(sizeof(Table<kLargeTable>) + 64 <= 32764, "");

struct Scalars {
  float b1, c1, b2, c2, rs, eps, max_norm;
  const float* norm;
};

// The contiguous range of chunks of this CTA, and the tensor of its first one.
template <int N>
__device__ __forceinline__ void my_range(const Table<N>& t, int* c0, int* c1, int* at) {
  const int64_t total = t.chunks;
  *c0 = static_cast<int>(total * blockIdx.x / gridDim.x);
  *c1 = static_cast<int>(total * (blockIdx.x + 1) / gridDim.x);
  int lo = 0, hi = t.count - 1;  // the last tensor whose first chunk is <= c0
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].first <= *c0) lo = mid;
    else hi = mid - 1;
  }
  *at = lo;
}

// Calls f(entry, k0, k1) for each tensor's chunks k0..k1-1 in this CTA's range.
template <int N, class F>
__device__ __forceinline__ void for_range(const Table<N>& t, F f) {
  int c, c1, at;
  my_range(t, &c, &c1, &at);
  while (c < c1) {
    const Entry& e = t.e[at];
    const int end = at + 1 < t.count ? min(c1, t.e[at + 1].first) : c1;
    f(e, c - e.first, end - e.first);
    c = end;
    ++at;
  }
}

__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

__device__ __forceinline__ float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {
  __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
  uint32_t u;
  memcpy(&u, &p, 4);
  return u;
}

// Eight entries from i on as floats (left = how many of them exist).  fp32 goes by
// 32-byte accesses: a lane's whole sector at once.
__device__ __forceinline__ void load8(const float* p, int64_t i, int left, bool wide, float (&x)[8]) {
  if (wide && left >= 8) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                 : "l"(p + i));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? p[i + j] : 0.0f;
  }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int64_t i, int left, bool wide, float (&x)[8]) {
  if (wide && left >= 8) {
    const uint4 a = *reinterpret_cast<const uint4*>(p + i);
    x[0] = bf_lo(a.x); x[1] = bf_hi(a.x); x[2] = bf_lo(a.y); x[3] = bf_hi(a.y);
    x[4] = bf_lo(a.z); x[5] = bf_hi(a.z); x[6] = bf_lo(a.w); x[7] = bf_hi(a.w);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = j < left ? __bfloat162float(p[i + j]) : 0.0f;
  }
}
__device__ __forceinline__ void store8(float* p, int64_t i, int left, bool wide, const float (&x)[8]) {
  if (wide && left >= 8) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + i), "f"(x[0]), "f"(x[1]),
                 "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
                 : "memory");
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[i + j] = x[j];
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, int64_t i, int left, bool wide, const float (&x)[8]) {
  if (wide && left >= 8) {
    *reinterpret_cast<uint4*>(p + i) = make_uint4(bf_pack(x[0], x[1]), bf_pack(x[2], x[3]),
                                                  bf_pack(x[4], x[5]), bf_pack(x[6], x[7]));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[i + j] = __float2bfloat16_rn(x[j]);
  }
}

// Eight codes (one byte each, low byte first) as two words.
__device__ __forceinline__ uint2 load_codes(const void* p, int64_t i, int left, bool wide) {
  const uint8_t* b = static_cast<const uint8_t*>(p) + i;
  if (wide && left >= 8) return *reinterpret_cast<const uint2*>(b);
  uint2 u = make_uint2(0, 0);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < left) (j < 4 ? u.x : u.y) |= static_cast<uint32_t>(b[j]) << (8 * (j & 3));
  return u;
}
__device__ __forceinline__ void store_codes(void* p, int64_t i, int left, bool wide, uint2 u) {
  uint8_t* b = static_cast<uint8_t*>(p) + i;
  if (wide && left >= 8) {
    *reinterpret_cast<uint2*>(b) = u;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) b[j] = static_cast<uint8_t>((j < 4 ? u.x : u.y) >> (8 * (j & 3)));
  }
}

// Byte j of a word as a float: the bits of 2^23 + byte, less 2^23 (exact, and two
// full-rate instructions where an integer conversion runs at a quarter rate).
__device__ __forceinline__ float byte_float(uint32_t u, int j, float less) {
  return fsub(__uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540 | j)), less);
}
constexpr float kTwo23 = 8388608.0f;

// The squares of a code are exact in fp32, so a value carries three (m) or four
// (v) roundings.  Signed codes are read with their sign bit flipped (c + 128).
__device__ __forceinline__ float decode_m(uint32_t flipped, int j, float s) {
  const float c = byte_float(flipped, j, kTwo23 + 128.0f);
  return fmul(fmul(fmul(c, fabsf(c)), static_cast<float>(1.0 / (127.0 * 127.0))), s);
}
__device__ __forceinline__ float decode_v(uint32_t u, int j, float s) {
  const float c = byte_float(u, j, kTwo23);
  const float c2 = fmul(c, c);
  return fmul(fmul(fmul(c2, c2), static_cast<float>(1.0 / (255.0 * 255.0 * 255.0 * 255.0))), s);
}
constexpr uint32_t kFlip = 0x80808080u;

// 1/top, or 0 for a block without a value in the normal range (its codes are 0).
__device__ __forceinline__ float inverse(float top) {
  return top < 1.17549435e-38f ? 0.0f : fdiv(1.0f, top);
}

__device__ __forceinline__ float root_approx(float x) {  // subnormal x counts as 0
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float inverse_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// The code of y in [0, 1], as 2^23 + code: how many midpoints lie at or below y.
// The midpoint under code c of LEVELS is K (2c(c-1) + 1), K = 1/(2 LEVELS^2),
// halfway between the neighbouring squares, and its square for FOURTH (v).  There
// the root of LEVELS^2 y - 1/4 is c - 1/2, so the floor of an approximate root
// (off by less than 2e-4) is the code or the one before it, and the exact midpoint
// over it decides: the result does not depend on the approximation.  (2c(c+1) + 1
// is exact in fp32.  Below a quarter the root of the negative value's magnitude,
// at most 1/2, gives 0 as well.)
template <int LEVELS, bool FOURTH>
__device__ __forceinline__ float encode(float y) {
  constexpr float K = static_cast<float>(1.0 / (2.0 * LEVELS * LEVELS));
  const float s = FOURTH ? root_approx(y) : y;
  const float z = __fmaf_rn(s, static_cast<float>(LEVELS * LEVELS), -0.25f);
  const float t = __fadd_rd(root_approx(fabsf(z)), kTwo23);
  const float c = fsub(t, kTwo23);
  float mid = fmul(__fmaf_rn(c, __fmaf_rn(c, 2.0f, 2.0f), 1.0f), K);
  if (FOURTH) mid = fmul(mid, mid);
  return y >= mid ? fadd(t, 1.0f) : t;
}

// The low bytes of four floats in [2^23, 2^23 + 256) as one word.
__device__ __forceinline__ uint32_t low_bytes(float a, float b, float c, float d) {
  const uint32_t lo = __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040);
  const uint32_t hi = __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040);
  return __byte_perm(lo, hi, 0x5410);
}

// The larger one, NaN where either is (as its bits 0x7fffffff, which warp_max takes
// for the largest).
__device__ __forceinline__ float max_nan(float x, float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}
__device__ __forceinline__ float warp_max(float x) {  // x >= 0 or NaN
  return __uint_as_float(__reduce_max_sync(kFull, __float_as_uint(x)));
}

template <typename P, typename G, int BITS, int N>
__global__ void __launch_bounds__(kThreads)
    adamw_kernel(const __grid_constant__ Table<N> t, const Scalars k) {
  pdl_begin();
  float clip = 1.0f;
  if (k.norm != nullptr) {
    const float norm = *k.norm;
    if (!(norm <= 3.402823466e38f)) return;  // not finite: the step is skipped
    if (k.max_norm > 0.0f) clip = fminf(fdiv(k.max_norm, fadd(norm, 1e-6f)), 1.0f);
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for_range(t, [&](const Entry& e, int k0, int k1) {
    const bool wide = e.wide;
    const float keep = e.keep, rate = e.step;
    for (int chunk = k0; chunk < k1; ++chunk) {
      const int64_t base = static_cast<int64_t>(chunk) * kChunk + warp * (32 * kLane);
      if (base >= e.n) break;  // the tensor's last chunk
      const int64_t i = base + lane * kLane;
      const int left = static_cast<int>(min64(max64(e.n - i, 0), kLane));
      if (BITS == 8 && i + kChunk < e.n) {
        // this warp's next entries, from HBM while these are worked on: 459 -> 401 us
        // for 153M entries (fp32 states, which have more bytes in flight, lose 6 %)
        const int64_t next = i + kChunk;
        prefetch_l2(static_cast<const P*>(e.param) + next);
        prefetch_l2(static_cast<const G*>(e.grad) + next);
        prefetch_l2(static_cast<const uint8_t*>(e.m) + next);
        prefetch_l2(static_cast<const uint8_t*>(e.v) + next);
      }
      float p[8], g[8], m[8], v[8];
      load8(static_cast<const G*>(e.grad), i, left, wide, g);
      load8(static_cast<const P*>(e.param), i, left, wide, p);
      const int64_t block = base >> 8;
      if (BITS == 32) {
        load8(static_cast<const float*>(e.m), i, left, wide, m);
        load8(static_cast<const float*>(e.v), i, left, wide, v);
      } else {
        const uint2 um = load_codes(e.m, i, left, wide), uv = load_codes(e.v, i, left, wide);
        const float sm = e.sm[block], sv = e.sv[block];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          m[j] = decode_m((j < 4 ? um.x : um.y) ^ kFlip, j & 3, sm);
          v[j] = decode_v(j < 4 ? uv.x : uv.y, j & 3, sv);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float gj = fmul(g[j], clip);
        m[j] = fadd(fmul(m[j], k.b1), fmul(gj, k.c1));
        v[j] = fadd(fmul(v[j], k.b2), fmul(fmul(gj, k.c2), gj));
        // 8-bit states are bound by instructions: the root and the quotient, which
        // reach param alone, are the 1 and 2 ulp ones there
        const float root = BITS == 32 ? __fsqrt_rn(v[j]) : root_approx(v[j]);
        const float under = fadd(fmul(root, k.rs), k.eps);
        const float quotient = BITS == 32 ? fdiv(m[j], under) : fmul(m[j], inverse_approx(under));
        p[j] = fsub(fmul(p[j], keep), fmul(quotient, rate));
      }
      store8(static_cast<P*>(e.param), i, left, wide, p);
      if (e.copy != nullptr) store8(static_cast<__nv_bfloat16*>(e.copy), i, left, wide, p);
      if (BITS == 32) {
        store8(static_cast<float*>(e.m), i, left, wide, m);
        store8(static_cast<float*>(e.v), i, left, wide, v);
      } else {
        if (left < 8) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j >= left) m[j] = v[j] = 0.0f;
        }
        float tm = 0.0f, tv = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          tm = max_nan(tm, fabsf(m[j]));
          tv = max_nan(tv, v[j]);
        }
        tm = warp_max(tm);
        tv = warp_max(tv);
        const float im = inverse(tm), iv = inverse(tv);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // 2^23 + 128 + c for m >= 0; (2^24 + 128) - (2^23 + c) below
          const float cm = encode<127, false>(fmul(fabsf(m[j]), im));
          m[j] = m[j] < 0.0f ? fsub(2.0f * kTwo23 + 128.0f, cm) : fadd(cm, 128.0f);
          const float y = fmul(v[j], iv);
          v[j] = encode<255, true>(y);
          if (y > 0.0f) v[j] = fmaxf(v[j], kTwo23 + 1.0f);
        }
        store_codes(e.m, i, left, wide,
                    make_uint2(low_bytes(m[0], m[1], m[2], m[3]) ^ kFlip, low_bytes(m[4], m[5], m[6], m[7]) ^ kFlip));
        store_codes(e.v, i, left, wide,
                    make_uint2(low_bytes(v[0], v[1], v[2], v[3]), low_bytes(v[4], v[5], v[6], v[7])));
        if (lane == 0) {
          e.sm[block] = tm;
          e.sv[block] = tv;
        }
      }
    }
  });
}

// The values that 8-bit states stand for: param and copy of an entry are the
// fp32 outputs of m and v here.
template <int N>
__global__ void __launch_bounds__(kThreads) adamw_decode_kernel(const __grid_constant__ Table<N> t) {
  pdl_begin();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto decode = [&](const Entry& e, int chunk, bool whole) {
    const int64_t base = static_cast<int64_t>(chunk) * kChunk + warp * (32 * kLane);
    if (!whole && base >= e.n) return;
    const int64_t i = base + lane * kLane;
    const int left = whole ? kLane : static_cast<int>(min64(max64(e.n - i, 0), kLane));
    const bool wide = whole || e.wide;
    const uint2 um = load_codes(e.m, i, left, wide), uv = load_codes(e.v, i, left, wide);
    const float sm = e.sm[base >> 8], sv = e.sv[base >> 8];
    float m[8], v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      m[j] = decode_m((j < 4 ? um.x : um.y) ^ kFlip, j & 3, sm);
      v[j] = decode_v(j < 4 ? uv.x : uv.y, j & 3, sv);
    }
    store8(static_cast<float*>(e.param), i, left, wide, m);
    store8(static_cast<float*>(e.copy), i, left, wide, v);
  };
  for_range(t, [&](const Entry& e, int k0, int k1) {
    const int whole = e.wide ? static_cast<int>(min64(k1, e.n / kChunk)) : k0;
    int chunk = k0;
#pragma unroll 2
    for (; chunk < whole; ++chunk) decode(e, chunk, true);  // no condition between the loads
    for (; chunk < k1; ++chunk) decode(e, chunk, false);
  });
}

// Sum of squares of this CTA's chunks: fp32 over the entries of a thread, then
// fp64 over the CTA.  No atomics: the sum depends on the grid alone.
template <typename G, int N>
__global__ void __launch_bounds__(kThreads)
    grad_square_kernel(const __grid_constant__ Table<N> t, double* part) {
  pdl_begin();
  float sum = 0.0f;
  auto add = [&](const Entry& e, int chunk, bool whole) {
    const int64_t i = static_cast<int64_t>(chunk) * kChunk + threadIdx.x * kLane;
    float g[8];
    load8(static_cast<const G*>(e.grad), i, whole ? kLane : static_cast<int>(min64(max64(e.n - i, 0), kLane)),
          whole || e.wide, g);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fadd(s, fmul(g[j], g[j]));
    sum = fadd(sum, s);
  };
  for_range(t, [&](const Entry& e, int k0, int k1) {
    const int whole = e.wide ? static_cast<int>(min64(k1, e.n / kChunk)) : k0;
    int chunk = k0;
#pragma unroll 4
    for (; chunk < whole; ++chunk) add(e, chunk, true);  // no condition between the loads
    for (; chunk < k1; ++chunk) add(e, chunk, false);
  });
  __shared__ double warp_sum[kThreads / 32];
  double d = sum;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(kFull, d, o);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = d;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 32; ++w) d += warp_sum[w];
    part[blockIdx.x] = d;
  }
}

__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double* part, int n, float* norm) {
  pdl_begin();
  double d = 0.0;
  for (int i = threadIdx.x; i < n; i += kThreads) d += part[i];
  __shared__ double warp_sum[kThreads / 32];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(kFull, d, o);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = d;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 32; ++w) d += warp_sum[w];
    *norm = static_cast<float>(sqrt(d));
  }
}

// Both steps in one CTA for a short list (kOneCta chunks): groups of 256 threads
// take chunks in turn.
constexpr int kOneCta = 32;
template <typename G, int N>
__global__ void __launch_bounds__(4 * kThreads)
    grad_norm_one_kernel(const __grid_constant__ Table<N> t, float* norm) {
  pdl_begin();
  const int group = threadIdx.x / kThreads, lane = threadIdx.x % kThreads;
  float sum = 0.0f;
  int at = 0;
  for (int c = group; c < t.chunks; c += 4) {
    while (at + 1 < t.count && t.e[at + 1].first <= c) ++at;
    const Entry& e = t.e[at];
    const int64_t i = static_cast<int64_t>(c - e.first) * kChunk + lane * kLane;
    float g[8];
    load8(static_cast<const G*>(e.grad), i, static_cast<int>(min64(max64(e.n - i, 0), kLane)), e.wide, g);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fadd(s, fmul(g[j], g[j]));
    sum = fadd(sum, s);
  }
  __shared__ double warp_sum[4 * kThreads / 32];
  double d = sum;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(kFull, d, o);
  if ((threadIdx.x & 31) == 0) warp_sum[threadIdx.x >> 5] = d;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 4 * kThreads / 32; ++w) d += warp_sum[w];
    *norm = static_cast<float>(sqrt(d));
  }
}

bool on32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; }

// CTAs of a launch over `chunks` chunks: as many as are resident, so that every
// CTA takes one contiguous range.
template <typename K>
int grid_of(K kernel, int chunks, int num_sms) {
  const int64_t full = static_cast<int64_t>(num_sms) * resident_blocks(kernel, kThreads, 0);
  return static_cast<int>(std::min<int64_t>(chunks, full));
}

// Calls fn(table) for the list in as few tables as it takes.
template <typename Fn>
cudaError_t for_tables(const Entry* list, int64_t count, Fn fn) {
  int64_t i = 0;
  while (i < count) {
    Table<kLargeTable> big;
    big.count = 0;
    int64_t chunks = 0;
    for (; i < count && big.count < kLargeTable; ++i) {
      if (list[i].n == 0) continue;
      const int64_t c = (list[i].n + kChunk - 1) / kChunk;
      if (chunks + c > 0x7fffffff) {
        if (big.count > 0) break;
        return cudaErrorInvalidValue;  // a tensor of 2^42 entries
      }
      big.e[big.count] = list[i];
      big.e[big.count++].first = static_cast<int>(chunks);
      chunks += c;
    }
    if (big.count == 0) break;
    big.chunks = static_cast<int>(chunks);
    cudaError_t e;
    if (big.count <= kSmallTable) {
      Table<kSmallTable> small;
      std::copy(big.e, big.e + big.count, small.e);
      small.count = big.count;
      small.chunks = big.chunks;
      e = fn(small);
    } else {
      e = fn(big);
    }
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

template <typename P, typename G, int BITS>
cudaError_t step_tables(const Entry* list, int64_t count, const Scalars& k, int num_sms, cudaStream_t s) {
  return for_tables(list, count, [&](const auto& t) {
    constexpr int N = sizeof(t.e) / sizeof(Entry);
    auto kernel = adamw_kernel<P, G, BITS, N>;
    return launch_kernel(kernel, dim3(grid_of(kernel, t.chunks, num_sms)), dim3(kThreads), 0, s, 0, t, k);
  });
}

}  // namespace

cudaError_t launch_adamw(const AdamwArgs& a, int num_sms, cudaStream_t s) {
  Scalars k;
  k.b1 = static_cast<float>(a.beta1);
  k.c1 = static_cast<float>(1.0 - a.beta1);
  k.b2 = static_cast<float>(a.beta2);
  k.c2 = static_cast<float>(1.0 - a.beta2);
  k.rs = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(a.beta2, static_cast<double>(a.step))));
  k.eps = static_cast<float>(a.eps);
  k.norm = a.grad_norm;
  k.max_norm = static_cast<float>(a.max_norm);
  const double rate = a.lr / (1.0 - std::pow(a.beta1, static_cast<double>(a.step)));
  constexpr int kBatch = 4 * kLargeTable;
  Entry list[kBatch];
  for (int64_t i0 = 0; i0 < a.count; i0 += kBatch) {
    const int64_t n = std::min<int64_t>(kBatch, a.count - i0);
    for (int64_t i = 0; i < n; ++i) {
      const mpc_adamw_tensor& t = a.tensors[i0 + i];
      list[i] = Entry{t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.scale_m, t.scale_v, t.copy, t.n,
                      static_cast<float>(1.0 - a.lr * t.lr_scale * t.weight_decay),
                      static_cast<float>(rate * t.lr_scale), 0,
                      on32(t.param) && on32(t.grad) && on32(t.exp_avg) && on32(t.exp_avg_sq) && on32(t.copy)};
    }
    cudaError_t e;
    using b16 = __nv_bfloat16;
    if (a.state_bits == 32) {
      if (a.param_bf16) e = a.grad_bf16 ? step_tables<b16, b16, 32>(list, n, k, num_sms, s) : step_tables<b16, float, 32>(list, n, k, num_sms, s);
      else e = a.grad_bf16 ? step_tables<float, b16, 32>(list, n, k, num_sms, s) : step_tables<float, float, 32>(list, n, k, num_sms, s);
    } else {
      if (a.param_bf16) e = a.grad_bf16 ? step_tables<b16, b16, 8>(list, n, k, num_sms, s) : step_tables<b16, float, 8>(list, n, k, num_sms, s);
      else e = a.grad_bf16 ? step_tables<float, b16, 8>(list, n, k, num_sms, s) : step_tables<float, float, 8>(list, n, k, num_sms, s);
    }
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_adamw_decode(const mpc_adamw_tensor* tensors, int64_t count, float* const* m_out,
                                float* const* v_out, int num_sms, cudaStream_t s) {
  constexpr int kBatch = 4 * kLargeTable;
  Entry list[kBatch];
  for (int64_t i0 = 0; i0 < count; i0 += kBatch) {
    const int64_t n = std::min<int64_t>(kBatch, count - i0);
    for (int64_t i = 0; i < n; ++i) {
      const mpc_adamw_tensor& t = tensors[i0 + i];
      float* mo = m_out[i0 + i];
      float* vo = v_out[i0 + i];
      list[i] = Entry{mo, nullptr, t.exp_avg, t.exp_avg_sq, t.scale_m, t.scale_v, vo, t.n, 0.0f, 0.0f, 0,
                      on32(mo) && on32(vo) && on32(t.exp_avg) && on32(t.exp_avg_sq)};
    }
    const cudaError_t e = for_tables(list, n, [&](const auto& t) {
      constexpr int N = sizeof(t.e) / sizeof(Entry);
      auto kernel = adamw_decode_kernel<N>;
      return launch_kernel(kernel, dim3(grid_of(kernel, t.chunks, num_sms)), dim3(kThreads), 0, s, 0, t);
    });
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

// The partial sums take one fp64 value a CTA; every table of a long list (see
// for_tables) has its own kNormGrid of them.
constexpr int kNormGrid = 2048;

size_t grad_norm_workspace_bytes(int64_t count) {
  const int64_t tables = std::max<int64_t>(1, 2 * (count / kLargeTable + 1));
  return static_cast<size_t>(tables) * kNormGrid * sizeof(double);
}

cudaError_t launch_grad_norm(const mpc_adamw_tensor* tensors, int64_t count, int grad_bf16, float* norm,
                             double* part, int num_sms, cudaStream_t s) {
  constexpr int kBatch = 4 * kLargeTable;
  Entry list[kBatch];
  int used = 0;
  for (int64_t i0 = 0; i0 < count; i0 += kBatch) {
    const int64_t n = std::min<int64_t>(kBatch, count - i0);
    for (int64_t i = 0; i < n; ++i) {
      const mpc_adamw_tensor& t = tensors[i0 + i];
      list[i] = Entry{};
      list[i].grad = t.grad;
      list[i].n = t.n;
      list[i].wide = on32(t.grad);
    }
    bool whole = false;
    auto launch = [&](auto type) {
      using G = decltype(type);
      return for_tables(list, n, [&](const auto& t) {
        constexpr int N = sizeof(t.e) / sizeof(Entry);
        if constexpr (N == kSmallTable) {
          if (count <= kSmallTable && t.chunks <= kOneCta) {  // the whole list
            whole = true;
            return launch_kernel(grad_norm_one_kernel<G, N>, dim3(1), dim3(4 * kThreads), 0, s, 0, t, norm);
          }
        }
        auto kernel = grad_square_kernel<G, N>;
        const int grid = std::min(kNormGrid, grid_of(kernel, t.chunks, num_sms));
        const cudaError_t e = launch_kernel(kernel, dim3(grid), dim3(kThreads), 0, s, 0, t, part + used);
        used += grid;
        return e;
      });
    };
    const cudaError_t e = grad_bf16 ? launch(__nv_bfloat16{}) : launch(float{});
    if (e != cudaSuccess || whole) return e;
  }
  return launch_kernel(grad_norm_kernel, dim3(1), dim3(kThreads), 0, s, 0, part, used, norm);
}

}  // namespace mpc
