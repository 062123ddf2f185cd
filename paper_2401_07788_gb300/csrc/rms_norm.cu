// rms_norm.cu -- root-mean-square norm of every row with the residual's addition,
// its output in the input's type or as an 8-bit quantisation payload, and its gradient.
//
//   h = x + r;   rstd = 1 / sqrt(mean h^2 + eps);   y = h rstd w
//   dx = dh + rstd (w dy - n mean(w dy n)),  n = h rstd;   dw = sum_rows dy n
//
// A row is held in the registers of a group of threads, 16 entries each, and read once.
// Longer rows (over 16384 entries) are read twice, the second time mostly from L2.
//
// 8 bits: the codes of y would be those of u = h w, as y is u times a number of the
// row; so codes come from u's extremes, in the same reduction as the sum of squares,
// and rstd goes to scale and minimum.  Codes then depend on no rounding of rstd.
//
// Rounded to fewer bits in bf16: h, which the gradient reads as the forward pass left it (the residual
// stream, kept anyway).  This loses precision against a gradient from the fp32 sum x + r: dw of
// 16384 x 4096 is 2.0e-3 to 2.9e-3 off 64 bits (41 sets of inputs), from the fp32 sum 1.4e-3 to 2.1e-3, and
// 1.4 times as far (up to 1.6) on the same inputs.  An h in fp32
// would be written and read at twice the bytes; the sum made again would read x and r for h.
//
// What bounds it: HBM where rows are wide and aligned.  16384 x 4096 in bf16 with residual: forward
// 80 us (6.7 TB/s), gradient 96 us (5.6 TB/s) and 5 us for dw's parts; in fp32 153 us (7.0 TB/s) and 163
// with dw's parts (6.6 TB/s); 8192 x 768 in fp32 to 8 bits 14 us (6.1 TB/s).  Rows beyond 16384 entries are
// read entry by entry also where they are aligned: 600 x 20000 in bf16 18 us (2.7 TB/s), gradient 50 us (1.4
// TB/s).  Rows on odd addresses are read entry by entry and wait for latency:
// 3001 x 2051 in bf16 to 8 bits 21 us, 0.9 TB/s.
#include <algorithm>

#include "launch_util.h"
#include "layers.cuh"

namespace mpc {
namespace {

constexpr int kEach = 16;           // entries of a row a thread holds
constexpr int kLongest = kEach * 1024;  // of a row in registers
constexpr int kBlock = 128;         // threads of a CTA of short rows
constexpr int kLongBlock = 1024;

// The columns that thread t of a row's NT threads holds: 16-byte groups (wide), or
// single entries.
template <typename T, int NT, bool WIDE>
__device__ __forceinline__ int column(int t, int j) {
  constexpr int V = kVec<T>;
  return WIDE ? ((j / V) * NT + t) * V + j % V : j * NT + t;
}

template <typename T, int NT, bool WIDE>
__device__ __forceinline__ void load_row(const T* p, int t, int D, float (&v)[kEach]) {
  constexpr int V = kVec<T>;
  if (WIDE) {
    uint4 u[kEach / V];
#pragma unroll
    for (int c = 0; c < kEach / V; ++c) {
      const int col = (c * NT + t) * V;
      u[c] = col < D ? *reinterpret_cast<const uint4*>(p + col) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int c = 0; c < kEach / V; ++c) {
      float f[V];
      unpack16(u[c], f);
#pragma unroll
      for (int i = 0; i < V; ++i) v[c * V + i] = f[i];
    }
  } else {
    T e[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) e[j] = j * NT + t < D ? p[j * NT + t] : T(0.0f);
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] = as_float(e[j]);
  }
}

template <typename T, int NT, bool WIDE>
__device__ __forceinline__ void store_row(T* p, int t, int D, const float (&v)[kEach]) {
  constexpr int V = kVec<T>;
  if (WIDE) {
#pragma unroll
    for (int c = 0; c < kEach / V; ++c) {
      const int col = (c * NT + t) * V;
      float f[V];
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = v[c * V + i];
      if (col < D) *reinterpret_cast<uint4*>(p + col) = pack16(f);
    }
  } else {
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (j * NT + t < D) put(p + j * NT + t, v[j]);
  }
}

// Extremes that a NaN takes over: a row with a NaN in u then has the scale and minimum NaN, as the
// quantiser's, whose keys order NaN beyond infinity (fminf and fmaxf would drop it, and the receiver read
// a finite value).
__device__ __forceinline__ float least(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float most(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

struct Stats {
  float sum, lo, hi;
};
__device__ __forceinline__ Stats merge(const Stats& a, const Stats& b, bool extremes) {
  Stats r = {fadd(a.sum, b.sum), a.lo, a.hi};
  if (extremes) {
    r.lo = least(a.lo, b.lo);
    r.hi = most(a.hi, b.hi);
  }
  return r;
}
__device__ __forceinline__ Stats shuffled(const Stats& s, int o, bool extremes) {
  Stats r = {__shfl_xor_sync(kFull, s.sum, o), 0.0f, 0.0f};
  if (extremes) {
    r.lo = __shfl_xor_sync(kFull, s.lo, o);
    r.hi = __shfl_xor_sync(kFull, s.hi, o);
  }
  return r;
}

// Over a row's NT threads, the result in all of them; every thread of the CTA calls it.
// `shared` holds a Stats a warp and is free again at the next barrier.
template <int NT>
__device__ __forceinline__ Stats reduce_row(Stats s, bool extremes, Stats* shared) {
#pragma unroll
  for (int o = (NT < 32 ? NT : 32) / 2; o > 0; o >>= 1) s = merge(s, shuffled(s, o, extremes), extremes);
  if (NT > 32) {
    constexpr int W = NT < 32 ? 1 : NT / 32;
    const int warp = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) shared[warp] = s;
    __syncthreads();
    const Stats* mine = shared + warp / W * W;
    s = mine[0];
#pragma unroll
    for (int i = 1; i < W; ++i) s = merge(s, mine[i], extremes);
  }
  return s;
}

// scale and code step of a row of u, as the quantiser's (quant.cu): a range that is 0 or
// infinite, or whose inverse is, sends codes 0 and scale 0; one that is NaN the scale NaN.
struct Code {
  float lo, inv, scale;
};
__device__ __forceinline__ Code code_of(float lo, float hi) {
  const float range = fsub(hi, lo);
  const float levels = 255.0f;
  Code c = {lo, fdiv(levels, range), 0.0f};
  if (range == 0.0f || isinf(range) || isinf(c.inv)) c.inv = 0.0f;
  else c.scale = fdiv(range, levels);
  return c;
}
// (u - lo) inv rounded half to even, in the low byte: 0 <= (u - lo) inv < 255.001
__device__ __forceinline__ uint32_t code8(float u, const Code& c) {
  return c.inv == 0.0f ? 0u : __float_as_uint(fadd(fmul(fsub(u, c.lo), c.inv), 8388608.0f)) & 255u;
}

__device__ __forceinline__ float rstd_of(float sum, int D, float eps) {
  return fdiv(1.0f, __fsqrt_rn(fadd(fdiv(sum, static_cast<float>(D)), eps)));
}

// Rows of up to 16 NT entries; CTAs of `block` threads take block / NT rows each.
template <typename T, int NT, bool WIDE, bool CODES>
__global__ void __launch_bounds__(NT < kBlock ? kBlock : NT) rms_row_kernel(const RmsNormArgs a) {
  constexpr int kRows = (NT < kBlock ? kBlock : NT) / NT;
  __shared__ Stats shared[NT < kBlock ? kBlock / 32 : NT / 32];
  pdl_begin();
  pdl_end();
  const int t = threadIdx.x % NT, D = static_cast<int>(a.D);
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / NT;
  const bool live = row < a.rows;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  float h[kEach], w[kEach];
  load_row<T, NT, WIDE>(x, t, live ? D : 0, h);
  if (a.residual != nullptr) {
    float r[kEach];
    load_row<T, NT, WIDE>(static_cast<const T*>(a.residual) + row * a.ldr, t, live ? D : 0, r);
#pragma unroll
    for (int j = 0; j < kEach; ++j) h[j] = fadd(h[j], r[j]);
  }
  load_row<T, NT, WIDE>(static_cast<const T*>(a.weight), t, D, w);
  float sums[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  Stats s = {0.0f, INFINITY, -INFINITY};
#pragma unroll
  for (int j = 0; j < kEach; ++j) sums[j & 3] = __fmaf_rn(h[j], h[j], sums[j & 3]);
  s.sum = fadd(fadd(sums[0], sums[1]), fadd(sums[2], sums[3]));
  if (CODES) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const float u = fmul(h[j], w[j]);
      if (column<T, NT, WIDE>(t, j) < D) {
        s.lo = least(s.lo, u);
        s.hi = most(s.hi, u);
      }
    }
  }
  s = reduce_row<NT>(s, CODES, shared);
  if (!live) return;
  const float rstd = rstd_of(s.sum, D, a.eps);
  if (t == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
  if (a.h != nullptr) store_row<T, NT, WIDE>(static_cast<T*>(a.h) + row * a.ldh, t, D, h);
  if (!CODES) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) h[j] = fmul(fmul(h[j], rstd), w[j]);
    store_row<T, NT, WIDE>(static_cast<T*>(a.y) + row * a.ldy, t, D, h);
  } else {
    const Code c = code_of(s.lo, s.hi);
    if (t == 0) {
      a.scale[row] = fmul(c.scale, rstd);
      a.minv[row] = fmul(s.lo, rstd);
    }
    uint8_t* out = reinterpret_cast<uint8_t*>(a.codes + row * a.W);
    if (WIDE) {
#pragma unroll
      for (int g = 0; g < kEach / 4; ++g) {
        const int col = column<T, NT, WIDE>(t, g * 4);
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) word |= code8(fmul(h[g * 4 + i], w[g * 4 + i]), c) << (8 * i);
        if (col < D) *reinterpret_cast<uint32_t*>(out + col) = word;
      }
    } else {
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        if (j * NT + t < D) out[j * NT + t] = static_cast<uint8_t>(code8(fmul(h[j], w[j]), c));
    }
    for (int i = D + t; i < a.W * 4; i += NT) out[i] = 0;  // up to 15 bytes of the row's padding
  }
}

// Longer rows: a CTA a row, one entry a thread at a time, the row read twice.
template <typename T, bool CODES>
__global__ void __launch_bounds__(kLongBlock) rms_long_kernel(const RmsNormArgs a) {
  __shared__ Stats shared[kLongBlock / 32];
  pdl_begin();
  pdl_end();
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const T* r = a.residual == nullptr ? nullptr : static_cast<const T*>(a.residual) + row * a.ldr;
  const T* w = static_cast<const T*>(a.weight);
  const int D = static_cast<int>(a.D);
  auto at = [&](int i) { return r == nullptr ? as_float(x[i]) : fadd(as_float(x[i]), as_float(r[i])); };
  Stats s = {0.0f, INFINITY, -INFINITY};
#pragma unroll 4
  for (int i = threadIdx.x; i < D; i += kLongBlock) {
    const float h = at(i);
    s.sum = __fmaf_rn(h, h, s.sum);
    if (CODES) {
      const float u = fmul(h, as_float(w[i]));
      s.lo = least(s.lo, u);
      s.hi = most(s.hi, u);
    }
  }
  s = reduce_row<kLongBlock>(s, CODES, shared);
  const float rstd = rstd_of(s.sum, D, a.eps);
  const Code c = code_of(s.lo, s.hi);
  if (threadIdx.x == 0) {
    if (a.rstd != nullptr) a.rstd[row] = rstd;
    if (CODES) {
      a.scale[row] = fmul(c.scale, rstd);
      a.minv[row] = fmul(s.lo, rstd);
    }
  }
  T* y = static_cast<T*>(a.y) + row * a.ldy;
  T* ho = a.h == nullptr ? nullptr : static_cast<T*>(a.h) + row * a.ldh;
  uint8_t* out = reinterpret_cast<uint8_t*>(a.codes + row * a.W);
#pragma unroll 4
  for (int i = threadIdx.x; i < D; i += kLongBlock) {
    const float h = at(i), wi = as_float(w[i]);
    if (ho != nullptr) put(ho + i, h);
    if (CODES) out[i] = static_cast<uint8_t>(code8(fmul(h, wi), c));
    else put(y + i, fmul(fmul(h, rstd), wi));
  }
  if (CODES)
    for (int i = D + threadIdx.x; i < a.W * 4; i += kLongBlock) out[i] = 0;
}

// ---------------------------------------------------------------------------
// Gradient.  A CTA an SM takes every gridDim.x-th set of rows and keeps its sums of dw in
// registers, which leave as one row of `part`.  A thread holds 32 bytes of each tensor's row and
// asks for those of the next set before it works on this one: what bounds the pass is the bytes
// in flight (16384 x 4096 in bf16, four tensors: 124 us without that).
// ---------------------------------------------------------------------------
constexpr int kBackBlock = 512;
constexpr int kParts = 304;  // most rows of `part`
template <typename T>
constexpr int kBackEach = 32 / static_cast<int>(sizeof(T));
template <typename T>
constexpr int64_t kBackLongest = kBackEach<T> * 1024;

template <typename T, int NT, bool WIDE>
struct Raw {
  static constexpr int E = kBackEach<T>, V = kVec<T>;
  uint4 u[2];
  __device__ __forceinline__ void load(const T* p, int t, int D) {
    if (WIDE) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int col = (c * NT + t) * V;
        u[c] = col < D ? *reinterpret_cast<const uint4*>(p + col) : make_uint4(0, 0, 0, 0);
      }
    } else {
      T e[E];
#pragma unroll
      for (int j = 0; j < E; ++j) e[j] = j * NT + t < D ? p[j * NT + t] : T(0.0f);
      memcpy(u, e, 32);
    }
  }
  __device__ __forceinline__ void floats(float (&v)[E]) const {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float f[V];
      unpack16(u[c], f);
#pragma unroll
      for (int i = 0; i < V; ++i) v[c * V + i] = f[i];
    }
  }
  __device__ __forceinline__ void store(T* p, int t, int D, const float (&v)[E]) const {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float f[V];
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = v[c * V + i];
      if (WIDE) {
        const int col = (c * NT + t) * V;
        if (col < D) *reinterpret_cast<uint4*>(p + col) = pack16(f);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if ((c * V + i) * NT + t < D) put(p + (c * V + i) * NT + t, f[i]);
      }
    }
  }
};

template <typename T, int NT, bool WIDE>
__global__ void __launch_bounds__(NT < kBackBlock ? kBackBlock : NT, 1) rms_backward_kernel(const RmsNormArgs a, float* part) {
  constexpr int kThreads = NT < kBackBlock ? kBackBlock : NT;
  constexpr int kRows = kThreads / NT, E = kBackEach<T>;
  using R = Raw<T, NT, WIDE>;
  __shared__ Stats shared[2][kThreads / 32];
  extern __shared__ float sums[];  // [kRows][D] when kRows > 1
  pdl_begin();
  pdl_end();
  const int t = threadIdx.x % NT, D = static_cast<int>(a.D);
  R wr, h, dy, dh;
  float dw[E];
  wr.load(static_cast<const T*>(a.weight), t, D);
#pragma unroll
  for (int j = 0; j < E; ++j) dw[j] = 0.0f;
  const int64_t apart = static_cast<int64_t>(gridDim.x) * kRows;
  int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / NT;
  float rstd = 0.0f;
  auto ask = [&](int64_t r) {  // a row that does not exist is one of zeros
    const bool live = r < a.rows;
    const int width = live ? D : 0;
    h.load(static_cast<const T*>(a.x) + r * a.ldx, t, width);
    dy.load(static_cast<const T*>(a.dy) + r * a.lddy, t, width);
    if (a.dh != nullptr) dh.load(static_cast<const T*>(a.dh) + r * a.lddh, t, width);
    rstd = live ? a.rstd_in[r] : 0.0f;
  };
  ask(row);
  int turn = 0;
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * kRows; first < a.rows; first += apart, row += apart, turn ^= 1) {
    const bool live = row < a.rows;
    float n[E], g[E], w[E];
    const float mine = rstd;
    const R dh_now = dh;
    h.floats(n);
    dy.floats(g);
    wr.floats(w);
    ask(row + apart);
    float dot[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < E; ++j) {
      n[j] = fmul(n[j], mine);
      dw[j] = __fmaf_rn(g[j], n[j], dw[j]);
      g[j] = fmul(g[j], w[j]);
      dot[j & 3] = __fmaf_rn(g[j], n[j], dot[j & 3]);
    }
    Stats s = {fadd(fadd(dot[0], dot[1]), fadd(dot[2], dot[3])), 0.0f, 0.0f};
    s = reduce_row<NT>(s, false, shared[turn]);
    const float c = fdiv(s.sum, static_cast<float>(D));
    if (live) {
      float add[E];
      if (a.dh != nullptr) dh_now.floats(add);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        g[j] = fmul(mine, __fmaf_rn(-c, n[j], g[j]));
        if (a.dh != nullptr) g[j] = fadd(g[j], add[j]);
      }
      h.store(static_cast<T*>(a.dx) + row * a.lddx, t, D, g);
    }
  }
  if (part == nullptr) return;
  float* out = part + static_cast<int64_t>(blockIdx.x) * D;
  float* mine = kRows == 1 ? out : sums + threadIdx.x / NT * D;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    const int col = column<T, NT, WIDE>(t, j);
    if (col < D) mine[col] = dw[j];
  }
  if (kRows > 1) {
    __syncthreads();
    for (int i = threadIdx.x; i < D; i += kThreads) {
      float v = sums[i];
      for (int r = 1; r < kRows; ++r) v = fadd(v, sums[r * D + i]);
      out[i] = v;
    }
  }
}

// Longer rows: first mean(w dy n) of every row, then the columns.
template <typename T>
__global__ void __launch_bounds__(kLongBlock) rms_long_dot_kernel(const RmsNormArgs a, float* dot) {
  __shared__ Stats shared[kLongBlock / 32];
  pdl_begin();
  pdl_end();
  const int64_t row = blockIdx.x;
  const T* h = static_cast<const T*>(a.x) + row * a.ldx;
  const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
  const T* w = static_cast<const T*>(a.weight);
  const int D = static_cast<int>(a.D);
  const float rstd = a.rstd_in[row];
  Stats s = {0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int i = threadIdx.x; i < D; i += kLongBlock)
    s.sum = __fmaf_rn(fmul(as_float(dy[i]), as_float(w[i])), fmul(as_float(h[i]), rstd), s.sum);
  s = reduce_row<kLongBlock>(s, false, shared);
  if (threadIdx.x == 0) dot[row] = fdiv(s.sum, static_cast<float>(D));
}
template <typename T>
__global__ void __launch_bounds__(256) rms_long_backward_kernel(const RmsNormArgs a, const float* dot, float* part) {
  pdl_begin();
  pdl_end();
  const int i = blockIdx.x * 256 + threadIdx.x, D = static_cast<int>(a.D);
  if (i >= D) return;
  const float w = as_float(static_cast<const T*>(a.weight)[i]);
  float dw = 0.0f;
#pragma unroll 2
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float rstd = a.rstd_in[row];
    const float n = fmul(as_float(static_cast<const T*>(a.x)[row * a.ldx + i]), rstd);
    const float dy = as_float(static_cast<const T*>(a.dy)[row * a.lddy + i]);
    dw = __fmaf_rn(dy, n, dw);
    float g = fmul(rstd, __fmaf_rn(-dot[row], n, fmul(dy, w)));
    if (a.dh != nullptr) g = fadd(g, as_float(static_cast<const T*>(a.dh)[row * a.lddh + i]));
    put(static_cast<T*>(a.dx) + row * a.lddx + i, g);
  }
  if (part != nullptr) part[static_cast<int64_t>(blockIdx.y) * D + i] = dw;
}

// dw = sum of `parts` rows of part: 32 columns a CTA, 16 rows of threads.
template <typename T>
__global__ void __launch_bounds__(512) rms_dweight_kernel(const float* part, int parts, int D, T* dw) {
  __shared__ float sums[16][33];
  pdl_begin();
  pdl_end();
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), r = threadIdx.x >> 5;
  float v = 0.0f;
  if (col < D) {
#pragma unroll 4
    for (int p = r; p < parts; p += 16) v = fadd(v, part[static_cast<int64_t>(p) * D + col]);
  }
  sums[r][threadIdx.x & 31] = v;
  __syncthreads();
  if (r == 0 && col < D) {
#pragma unroll
    for (int p = 1; p < 16; ++p) v = fadd(v, sums[p][threadIdx.x]);
    put(dw + col, v);
  }
}

bool rows_wide(const void* p, int64_t ld, int V) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % V == 0);
}

template <typename T, int NT, bool WIDE>
cudaError_t launch_rows(const RmsNormArgs& a, cudaStream_t s) {
  constexpr int kThreads = NT < kBlock ? kBlock : NT, kRows = kThreads / NT;
  const unsigned grid = static_cast<unsigned>((a.rows + kRows - 1) / kRows);
  return launch_kernel(a.codes != nullptr ? rms_row_kernel<T, NT, WIDE, true> : rms_row_kernel<T, NT, WIDE, false>,
                       dim3(grid), dim3(kThreads), 0, s, 0u, a);
}

template <typename T, int NT, bool WIDE>
cudaError_t launch_rows_backward(const RmsNormArgs& a, float* part, int* parts, int num_sms, cudaStream_t s) {
  constexpr int kThreads = NT < kBackBlock ? kBackBlock : NT, kRows = kThreads / NT;
  const int64_t sets = (a.rows + kRows - 1) / kRows;
  *parts = static_cast<int>(std::min<int64_t>(sets, std::min(kParts, num_sms)));
  return launch_kernel(rms_backward_kernel<T, NT, WIDE>, dim3(*parts), dim3(kThreads),
                       kRows > 1 ? kRows * a.D * sizeof(float) : 0, s, 0u, a, part);
}

// Threads of a row: as few as hold it.
template <int EACH, typename F>
cudaError_t with_threads(int64_t D, F f) {
  if (D <= 8 * EACH) return f(std::integral_constant<int, 8>());
  if (D <= 32 * EACH) return f(std::integral_constant<int, 32>());
  if (D <= 64 * EACH) return f(std::integral_constant<int, 64>());
  if (D <= 128 * EACH) return f(std::integral_constant<int, 128>());
  if (D <= 256 * EACH) return f(std::integral_constant<int, 256>());
  if (D <= 512 * EACH) return f(std::integral_constant<int, 512>());
  return f(std::integral_constant<int, 1024>());
}

template <typename T>
cudaError_t run_forward(const RmsNormArgs& a, cudaStream_t s) {
  if (a.D > kLongest)
    return launch_kernel(a.codes != nullptr ? rms_long_kernel<T, true> : rms_long_kernel<T, false>,
                         dim3(static_cast<unsigned>(a.rows)), dim3(kLongBlock), 0, s, 0u, a);
  constexpr int V = kVec<T>;
  const bool wide = a.D % V == 0 && rows_wide(a.x, a.ldx, V) && rows_wide(a.residual, a.ldr, V) &&
                    rows_wide(a.weight, 0, V) && rows_wide(a.y, a.ldy, V) && rows_wide(a.h, a.ldh, V);
  if (wide)
    return with_threads<kEach>(a.D, [&](auto nt) { return launch_rows<T, decltype(nt)::value, true>(a, s); });
  return with_threads<kEach>(a.D, [&](auto nt) { return launch_rows<T, decltype(nt)::value, false>(a, s); });
}

template <typename T>
cudaError_t run_backward(const RmsNormArgs& a, int num_sms, cudaStream_t s) {
  constexpr int V = kVec<T>;
  float* part = a.dweight == nullptr ? nullptr : static_cast<float*>(a.ws);
  int parts = 0;
  cudaError_t e;
  if (a.D > kBackLongest<T>) {
    parts = static_cast<int>(std::min<int64_t>(a.rows, kParts));
    float* dot = static_cast<float*>(a.ws) + parts * a.D;
    e = launch_kernel(rms_long_dot_kernel<T>, dim3(static_cast<unsigned>(a.rows)), dim3(kLongBlock), 0, s, 0u, a, dot);
    if (e != cudaSuccess) return e;
    e = launch_kernel(rms_long_backward_kernel<T>, dim3(static_cast<unsigned>((a.D + 255) / 256), parts), dim3(256), 0, s, 0u, a,
                      static_cast<const float*>(dot), part);
  } else {
    const bool wide = a.D % V == 0 && rows_wide(a.x, a.ldx, V) && rows_wide(a.dy, a.lddy, V) &&
                      rows_wide(a.dh, a.lddh, V) && rows_wide(a.weight, 0, V) && rows_wide(a.dx, a.lddx, V);
    if (wide)
      e = with_threads<kBackEach<T>>(a.D, [&](auto nt) { return launch_rows_backward<T, decltype(nt)::value, true>(a, part, &parts, num_sms, s); });
    else
      e = with_threads<kBackEach<T>>(a.D, [&](auto nt) { return launch_rows_backward<T, decltype(nt)::value, false>(a, part, &parts, num_sms, s); });
  }
  if (e != cudaSuccess || part == nullptr) return e;
  return launch_kernel(rms_dweight_kernel<T>, dim3(static_cast<unsigned>((a.D + 31) / 32)), dim3(512), 0, s, 0u,
                       static_cast<const float*>(part), parts, static_cast<int>(a.D), static_cast<T*>(a.dweight));
}

}  // namespace

size_t rms_norm_workspace_bytes(int64_t rows, int64_t D) {
  const int64_t parts = std::min<int64_t>(rows, kParts);
  return static_cast<size_t>(parts * D + (D > kBackLongest<float> ? rows : 0)) * 4;  // either type's
}

cudaError_t launch_rms_norm(const RmsNormArgs& a, int, cudaStream_t s) {
  return a.bf16 ? run_forward<__nv_bfloat16>(a, s) : run_forward<float>(a, s);
}
cudaError_t launch_rms_norm_backward(const RmsNormArgs& a, int num_sms, cudaStream_t s) {
  return a.bf16 ? run_backward<__nv_bfloat16>(a, num_sms, s) : run_backward<float>(a, num_sms, s);
}

}  // namespace mpc
