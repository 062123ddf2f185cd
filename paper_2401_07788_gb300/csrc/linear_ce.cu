// linear_ce.cu -- softmax cross entropy of a linear head over a large
// vocabulary, with its gradient.  The loss keeps no logits; a gradient keeps bf16
// planes of the coefficients, of a piece of the vocabulary or of all of it (one plane
// in bf16, three in fp32).
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
//
// Forward: one pass of products (kLoss).  Backward from lse: per piece of the
// vocabulary the products again (kCoef), then dh and dw: 8 T D V operations with
// the forward's.  Training in one call, where g is known beforehand: the
// exponentials of the one pass are kept in bf16 planes (kExp) and made coefficients
// without forming the logits again, 6 T D V operations:
//   e[t][v] = 2^(l log2e - ref[t]) (0 at the target),  s[t] = sum of all of them
//   dh[t] = g/s sum_v e w + g (p - 1) w[target],   p = softmax at the target
//   dw[v] = sum_t e (g/s h[t]) + sum over tokens with target v of g (p - 1) h[t]
// The last sum needs the tokens grouped by target; a stable order is found by
// counting, for each token, those before it (rank_tokens).
//
// A few tokens go another way (linear_ce_few.cu).  The small kernels here let
// their successor be scheduled as they start.
//
// NaN: a logit that is NaN makes its token's loss, lse and gradients NaN.  An fp32
// infinity in h or w becomes NaN in its planes.
//
// What bounds it: the matrix units (linear_ce_gemm.cuh).  Measured over several boxes:
// 8192 tokens (a tenth ignored) x 768 x 50257 in bf16 1.20 to 1.26 ms, of which the
// three products 1.08 ms (the gradient from lse where all count 1.14, the loss 0.38);
// 8192 x 4096 x 131072 16.2 to 17.9 ms, 1.47 to 1.63 PFLOP/s of the 6 T D V operations;
// 2048 x 768 x 50257 in fp32 1.69 to 1.74 ms; 129 x 203 x 5003 in fp32 66 to 69 us,
// where eleven launches wait on one another.
#include <algorithm>

#include "kernels.h"
#include "launch_util.h"
#include "linear_ce_gemm.cuh"

namespace mpc {
namespace {

__device__ __forceinline__ void from_float(float x, float* p) { *p = x; }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16* p) { *p = __float2bfloat16_rn(x); }

// ---------------------------------------------------------------------------
// The list of tokens that count: row[i] = token, target[i], and place[t] = i
// (-1 for the others), in token order.  A CTA takes 1024 tokens and counts those
// before them itself, 8 bytes each from L2; beyond kScanAlone tokens a launch counts
// each CTA's first and the CTA adds up 4 bytes for 1024 of them (forward of 2^21 x 64 x
// 500 in bf16 3.66 -> 2.89 ms, 2^17 174 -> 168 us, 2^16 + 1 alike).  A target outside
// [0, V) that is not ignore_index is reported and left out too.
// ---------------------------------------------------------------------------
constexpr int kScan = 1024;
constexpr int64_t kScanAlone = int64_t{1} << 16;

__device__ __forceinline__ bool target_counts(int64_t v, int64_t V, int64_t ignore) { return v != ignore && v >= 0 && v < V; }

__global__ void __launch_bounds__(kScan)
    ce_count_kernel(const int64_t* __restrict__ targets, int T, int64_t V, int64_t ignore, int* counts) {
  pdl_begin();
  pdl_end();
  const int t = blockIdx.x * kScan + threadIdx.x;
  const int n = __syncthreads_count(t < T && target_counts(targets[t], V, ignore));
  if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

__global__ void __launch_bounds__(kScan)
    ce_scan_kernel(const int64_t* __restrict__ targets, int T, int64_t V, int64_t ignore, const int* __restrict__ counts,
                   Header* head, int* row, int* target, int* place, int* pos, int* flags, unsigned* status) {
  pdl_begin();
  pdl_end();
  __shared__ int before_of[32], count_of[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t0 = blockIdx.x * kScan, t = t0 + threadIdx.x;
  int64_t y = ignore;
  if (t < T) y = targets[t];
  int before = 0;
  if (counts != nullptr) {
    for (int i = threadIdx.x; i < static_cast<int>(blockIdx.x); i += kScan) before += counts[i];
  } else {
#pragma unroll 8
    for (int i = threadIdx.x; i < t0; i += kScan) before += target_counts(targets[i], V, ignore);
  }
  const bool keep = t < T && target_counts(y, V, ignore);
  if (y != ignore && !keep) set_status(status, STATUS_BAD_INDEX);
  before = __reduce_add_sync(kFull, before);
  const unsigned kept = __ballot_sync(kFull, keep);
  if (lane == 0) {
    before_of[warp] = before;
    count_of[warp] = __popc(kept);
  }
  __syncthreads();
  const int mine = count_of[lane];
  const int through = static_cast<int>(warp_inclusive_scan(static_cast<unsigned>(mine), lane));
  const int base = __reduce_add_sync(kFull, before_of[lane]);
  const int i = base + __shfl_sync(kFull, through - mine, warp) + __popc(kept & lanemask_lt());
  if (t < T) place[t] = keep ? i : -1;
  if (keep) {
    row[i] = t;
    target[i] = static_cast<int>(y);
  }
  if (t < T && pos != nullptr) pos[t] = 0;
  if (flags != nullptr && threadIdx.x < kScan / kPair) flags[blockIdx.x * (kScan / kPair) + threadIdx.x] = 0;
  const int total = base + __shfl_sync(kFull, through, 31);
  if (t0 + kScan >= T && threadIdx.x == 0) {
    head->valid = total;
    head->mean = total > 0 ? fdiv(1.0f, static_cast<float>(total)) : 0.0f;
    head->redo = 0;
  }
}

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
// Eight values of packed planes.
template <int P>
__device__ __forceinline__ void load_planes8(const uint16_t* in, int64_t plane, float (&x)[8]) {
#pragma unroll
  for (int k = P - 1; k >= 0; --k) {
    const uint4 u = *reinterpret_cast<const uint4*>(in + k * plane);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float v = __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
      x[j] = k == P - 1 ? v : fadd(v, x[j]);
    }
  }
}

// Rows that a product of row pairs may touch: zero from the last one that counts on.
__device__ __forceinline__ int64_t rows_touched(int64_t n) { return (n + kPair - 1) / kPair * kPair; }

// The listed rows of h in planes, out[plane][i][0..Dp), one warp a row; with `ref`
// also the logit of each row's target in base 2.
template <typename E, int P>
__device__ __forceinline__ void pack_h(unsigned block, const E* __restrict__ h, int64_t ldh, int n,
                                       const int* __restrict__ row, int64_t padded, int D, int Dp, int wide_h,
                                       uint16_t* __restrict__ out, const E* __restrict__ w, int64_t ldw,
                                       const int* __restrict__ target, int wide_w, float* ref) {
  const int lane = threadIdx.x & 31;
  const int64_t m = block * int64_t{8} + (threadIdx.x >> 5);
  if (m >= rows_touched(n)) return;
  const bool live = m < n;
  const E* src = live ? h + row[m] * ldh : nullptr;
  const E* at = live && ref != nullptr ? w + target[m] * ldw : nullptr;
  float dot = 0.0f;
  for (int d = lane * 8; d < Dp; d += 256) {
    uint16_t p[8][3] = {};
    if (live) {
      E x[8];
      load8(src + d, D - d, wide_h, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) planes_of<E>(x[j], p[j]);
      if (ref != nullptr) {
        E y[8];
        load8(at + d, D - d, wide_w, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) dot = __fmaf_rn(to_float(x[j]), to_float(y[j]), dot);
      }
    }
    store_planes8<P>(out + m * Dp + d, padded * Dp, p);
  }
  if (live && ref != nullptr) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot = fadd(dot, __shfl_xor_sync(kFull, dot, o));
    if (lane == 0) ref[m] = fmul(dot, kLog2e);
  }
}

// w in planes, for an fp32 w or rows that a tensor map cannot read: memory bound, 10
// bytes an entry in fp32 (50257 x 768: 55 us, 7.0 TB/s).
template <typename E, int P>
__device__ __forceinline__ void pack_w(unsigned block, unsigned blocks, const E* __restrict__ w, int64_t ldw, int64_t V,
                                       int D, int Dp, int wide, uint16_t* __restrict__ out) {
  const int groups = Dp / 8;
  for (int64_t q = block * int64_t{256} + threadIdx.x; q < V * groups; q += blocks * int64_t{256}) {
    const int64_t r = q / groups;
    const int d = static_cast<int>(q - r * groups) * 8;
    E x[8];
    uint16_t p[8][3];
    load8(w + r * ldw + d, D - d, wide, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) planes_of<E>(x[j], p[j]);
    store_planes8<P>(out + r * Dp + d, V * Dp, p);
  }
}

// pos[i] = tokens of the list that come before token i in the order by target,
// then by place.  Block (x, y) counts for 256 tokens over every ny-th block of 256
// others: two instructions a pair.  Integer sums: the
// order of the atomics does not show.
__device__ __forceinline__ void rank_tokens(int bx, int by, int ny, int n, const int* __restrict__ target, int* pos) {
  __shared__ int4 others[64];
  const int i = bx * 256 + threadIdx.x;
  if (bx * 256 >= n) return;
  const int y = i < n ? target[i] : 0;
  int count = 0;
  for (int b = by; b * 256 < n; b += ny) {
    const int j = b * 256 + threadIdx.x;
    __syncthreads();
    reinterpret_cast<int*>(others)[threadIdx.x] = j < n ? target[j] : 0x7fffffff;
    __syncthreads();
    if (b == bx) {
      for (int q = 0; q < 256; ++q) {
        const int o = reinterpret_cast<const int*>(others)[q];
        count += o < y || (o == y && q < static_cast<int>(threadIdx.x));
      }
    } else {
      const int below = b < bx ? y + 1 : y;  // earlier tokens with the same target come before
#pragma unroll 8
      for (int q = 0; q < 64; ++q) {
        const int4 o = others[q];
        count += (o.x < below) + (o.y < below) + (o.z < below) + (o.w < below);
      }
    }
  }
  if (i < n) atomicAdd(&pos[i], count);
}

// One launch for what the first products need: h packed, w packed where it has to
// be, and the tokens ranked where a gradient wants them by target.
template <typename E>
struct Prepare {
  const Header* head;
  const E* h;
  const E* w;
  int64_t ldh, ldw, V, padded;
  int D, Dp, wide_h, wide_w;
  const int* row;
  const int* target;
  uint16_t* hp;
  uint16_t* wp;
  float* ref;
  int* pos;
  unsigned h_blocks, w_blocks, rank_x, rank_y;
};

template <typename E, int P>
__global__ void __launch_bounds__(256) ce_prepare_kernel(const Prepare<E> f) {
  pdl_begin();
  pdl_end();
  const int n = f.head->valid;
  unsigned block = blockIdx.x;
  if (block < f.h_blocks) {
    pack_h<E, P>(block, f.h, f.ldh, n, f.row, f.padded, f.D, f.Dp, f.wide_h, f.hp, f.w, f.ldw, f.target, f.wide_w, f.ref);
    return;
  }
  block -= f.h_blocks;
  if (block < f.w_blocks) {
    pack_w<E, P>(block, f.w_blocks, f.w, f.ldw, f.V, f.D, f.Dp, f.wide_w, f.wp);
    return;
  }
  block -= f.w_blocks;
  rank_tokens(static_cast<int>(block % f.rank_x), static_cast<int>(block / f.rank_x), static_cast<int>(f.rank_y), n,
              f.target, f.pos);
}

// Largest value and sum of a row's half tiles over a CTA of 32 rows (lanes) x 32
// warps, in a fixed order; the result is valid in warp 0.  RELATIVE: the sums are
// over exp2 from each part's own largest value, else from one reference.  A part
// whose largest is -inf sums to 0, or to NaN: a largest value does not show NaN
// logits (fmaxf takes the other operand), so every sum is added.
template <bool RELATIVE>
__device__ __forceinline__ float2 sum_parts(const float2* part, int parts, int T, int m, int n) {
  __shared__ float top_of[32][33], sum_of[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float top = -INFINITY, sum = 0.0f;
  if (m < n) {
    if (RELATIVE) {
      for (int i = warp; i < parts; i += 32) top = fmaxf(top, part[static_cast<int64_t>(i) * T + m].x);
    }
    for (int i = warp; i < parts; i += 32) {
      const float2 p = part[static_cast<int64_t>(i) * T + m];
      if (RELATIVE) {
        sum = fadd(sum, p.x == -INFINITY ? p.y : fmul(p.y, exp2f(fsub(p.x, top))));
      } else {
        top = fmaxf(top, p.x);
        sum = fadd(sum, p.y);
      }
    }
  }
  top_of[warp][lane] = top;
  sum_of[warp][lane] = sum;
  __syncthreads();
  float2 r = make_float2(-INFINITY, 0.0f);
  if (warp == 0) {
    for (int w = 0; w < 32; ++w) r.x = fmaxf(r.x, top_of[w][lane]);
    for (int w = 0; w < 32; ++w) {
      const float t = top_of[w][lane];
      const float s = sum_of[w][lane];
      r.y = fadd(r.y, !RELATIVE || t == -INFINITY ? s : fmul(s, exp2f(fsub(t, r.x))));
    }
  }
  return r;
}

// log(1 + s 2^-d): the loss of a token from the sum s of the others' exponentials
// over a base (in base 2) that lies d under the target's logit l.  Where l is +inf it is
// inf - inf (an infinite d alone would make it 0).
__device__ __forceinline__ float loss_of(float s, float d, float l) {
  const float ratio = fmul(s, exp2f(-d));
  const float loss = ratio < 1e6f ? log1pf(ratio) : fmul(fsub(log2f(s), d), kLn2);
  return l == INFINITY ? __int_as_float(0x7fffffff) : loss;
}

// Forward: lse and loss of the tokens that count.
__global__ void __launch_bounds__(1024)
    ce_finish_kernel(int T, const Header* head, const int* row, const int* place, const float2* part, int parts,
                     const float* at_target, float* loss, float* lse) {
  pdl_begin();
  pdl_end();
  const int t = blockIdx.x * 32 + (threadIdx.x & 31), n = head->valid;
  if (threadIdx.x < 32 && t < T && place[t] < 0) loss[t] = lse[t] = 0.0f;
  if (blockIdx.x * 32 >= n) return;
  const int m = t;  // as a place in the list from here on
  const float2 r = sum_parts<true>(part, parts, T, m, n);
  if (threadIdx.x < 32 && m < n) {
    const float l = at_target[m], v = loss_of(r.y, __fmaf_rn(l, kLog2e, -r.x), l);
    loss[row[m]] = v;
    // of l + loss a target at -inf leaves nothing: that of the others; one at +inf is all of it
    lse[row[m]] = l == -INFINITY ? fmul(fadd(log2f(r.y), r.x), kLn2) : l == INFINITY ? fadd(l, r.y) : fadd(l, v);
  }
}

// Training: the sum of each row's exponentials without the target's.  A sum out
// of range (a loss over 27) takes the row's largest logit as reference and marks
// its row tile.
__global__ void __launch_bounds__(1024)
    ce_sum_kernel(int T, Header* head, const float2* part, int parts, float* sum, float* ref, int* flags) {
  pdl_begin();
  pdl_end();
  const int m = blockIdx.x * 32 + (threadIdx.x & 31), n = head->valid;
  if (blockIdx.x * 32 >= n) return;
  const float2 r = sum_parts<false>(part, parts, T, m, n);
  if (threadIdx.x < 32 && m < n) {
    sum[m] = r.y;
    if (!(r.y < 0x1p40f) && fabsf(r.x) < INFINITY) {
      ref[m] = r.x;
      flags[m / kPair] = 1;
      head->redo = 1;
    }
  }
}

struct Finish {
  int T, D, Dp, parts;
  int64_t V, padded;
  const Header* head;
  const int* row;
  const int* target;
  const int* place;
  const int* pos;
  const int* flags;
  const float2* part;
  const float* at_target;
  const float* ref;
  const float* sum;
  const float* gloss;
  const uint16_t* hp;
  const float* lse;    // given lse and no sums (logits formed twice): [T] by token
  const float* loss_in;
  uint16_t* hs;        // h times g/s in planes, or nullptr
  float* scale;        // g/s
  float* coef;         // g (p - 1)
  int* order;          // token at each position by target
  int* sorted;         // its target
  int* seg_first;
  float* loss;
};

// A row of hidden states times `scale`, in planes (zero for one that is not listed).
template <int P>
__device__ __forceinline__ void scale_row(const Finish& f, int64_t m, int n, float scale) {
  const int64_t plane = f.padded * f.Dp;
  for (int d = static_cast<int>(threadIdx.x & 31) * 8; d < f.Dp; d += 256) {
    uint16_t p[8][3] = {};
    if (m < n) {
      float x[8];
      load_planes8<P>(f.hp + m * f.Dp + d, plane, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) split(fmul(x[j], scale), p[j]);
    }
    store_planes8<P>(f.hs + m * f.Dp + d, plane, p);
  }
}

// Training: the target's coefficients and the order by target, and where the
// exponentials are kept the loss, the factors and the scaled hidden states; one
// warp a row.
template <int P>
__global__ void __launch_bounds__(256) ce_scale_kernel(const Finish f) {
  pdl_begin();
  pdl_end();
  const int n = f.head->valid, lane = threadIdx.x & 31;
  const int64_t m = blockIdx.x * int64_t{8} + (threadIdx.x >> 5);
  for (int64_t v = blockIdx.x * int64_t{256} + threadIdx.x; v < f.V; v += gridDim.x * int64_t{256}) f.seg_first[v] = 0;
  if (f.hs != nullptr && lane == 0 && m < f.T && f.place[m] < 0) f.loss[m] = 0.0f;  // m as a token here
  if (m >= rows_touched(n)) return;
  float scale = 0.0f;
  if (m < n) {
    const int t = f.row[m];
    const float g = f.gloss != nullptr ? f.gloss[t] : f.head->mean;
    float loss;
    if (f.hs != nullptr) {
      float s = f.sum[m];
      if (f.flags[m / kPair] != 0) {
        s = 0.0f;
        for (int i = lane; i < f.parts; i += 32) s = fadd(s, f.part[static_cast<int64_t>(i) * f.T + m].y);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s = fadd(s, __shfl_xor_sync(kFull, s, o));
      }
      const float d = __fmaf_rn(f.at_target[m], kLog2e, -f.ref[m]);
      loss = loss_of(s, d, f.at_target[m]);
      scale = fdiv(g, fadd(s, exp2f(d)));
      if (lane == 0) {
        f.loss[t] = loss;
        f.scale[m] = scale;
      }
    } else {
      loss = f.loss_in != nullptr ? f.loss_in[t] : __fmaf_rn(f.ref[m], -kLn2, f.lse[t]);
    }
    if (lane == 0) {
      f.coef[m] = fmul(g, expm1f(-loss));
      f.order[f.pos[m]] = static_cast<int>(m);
      f.sorted[f.pos[m]] = f.target[m];
    }
  }
  if (f.hs != nullptr) scale_row<P>(f, m, n, scale);
}

// A gradient from lse whose coefficients are taken over g (1 - p): 1 / (1 - p), the
// factor, and the scaled hidden states; one warp a row.  1 - p comes from the loss (of
// the forward pass, or lse less the target's logit).  Where p is 1 to the last digit
// any small 1 - p serves: the factor takes it back from the other coefficients.
template <int P>
__global__ void __launch_bounds__(256) ce_over_kernel(const Finish f) {
  pdl_begin();
  pdl_end();
  const int n = f.head->valid, lane = threadIdx.x & 31;
  const int64_t m = blockIdx.x * int64_t{8} + (threadIdx.x >> 5);
  if (m >= rows_touched(n)) return;
  float scale = 0.0f;
  if (m < n) {
    const int t = f.row[m];
    const float loss = f.loss_in != nullptr ? f.loss_in[t] : __fmaf_rn(f.ref[m], -kLn2, f.lse[t]);
    float q = -expm1f(-loss);
    if (q < 0x1p-60f) q = 0x1p-60f;
    scale = fmul(f.gloss != nullptr ? f.gloss[t] : f.head->mean, q);
    if (lane == 0) {
      f.scale[m] = scale;
      f.coef[m] = fdiv(1.0f, q);
    }
  }
  scale_row<P>(f, m, n, scale);
}

// Target gradients: a CTA takes kRun tokens in the order by target and sums
// coef h over each run with one target, in token order, into seg_sum at the run's
// first position.
template <int P>
__global__ void __launch_bounds__(256)
    ce_target_kernel(const Header* head, const int* __restrict__ order, const int* __restrict__ sorted,
                     const float* __restrict__ coef, const uint16_t* __restrict__ hp, int64_t plane, int Dp,
                     int* seg_first, int* seg_end, float* seg_sum, int64_t lds) {
  pdl_begin();
  pdl_end();
  __shared__ int at[kRun], y[kRun + 1];
  __shared__ float c[kRun];
  const int n = head->valid;
  const int p0 = blockIdx.x * kRun;
  if (p0 >= n) return;
  const int count = min(kRun, n - p0);
  if (threadIdx.x < count) {
    const int m = order[p0 + threadIdx.x];
    at[threadIdx.x] = m;
    c[threadIdx.x] = coef[m];
    const int mine = sorted[p0 + threadIdx.x];
    y[threadIdx.x] = mine;
    if (p0 + threadIdx.x == 0 || sorted[p0 + threadIdx.x - 1] != mine) seg_first[mine] = p0 + threadIdx.x + 1;
    if (p0 + threadIdx.x + 1 == n || sorted[p0 + threadIdx.x + 1] != mine) seg_end[mine] = p0 + threadIdx.x + 1;
  }
  __syncthreads();
  for (int d = threadIdx.x * 8; d < Dp; d += 256 * 8) {
    float s[8] = {};
    int first = 0;
#pragma unroll 8
    for (int q = 0; q < count; ++q) {
      float x[8];
      load_planes8<P>(hp + static_cast<int64_t>(at[q]) * Dp + d, plane, x);
      const float f = c[q];
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] = __fmaf_rn(f, x[j], s[j]);
      if (q + 1 == count || y[q + 1] != y[q]) {
        float4* out = reinterpret_cast<float4*>(seg_sum + (p0 + first) * lds + d);
        out[0] = make_float4(s[0], s[1], s[2], s[3]);
        out[1] = make_float4(s[4], s[5], s[6], s[7]);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = 0.0f;
        first = q + 1;
      }
    }
  }
}

// A target whose tokens go past the end of a block of kRun: the CTA of the block in
// which it starts adds up its blocks' sums, at the first one's place.  (Left to
// the rows of dw, a frequent target's blocks made one thread's tail: 40 us of 390
// at 8192 x 768 x 50257.)
__global__ void __launch_bounds__(256)
    ce_join_kernel(const Header* head, const int* __restrict__ sorted, const int* __restrict__ seg_first,
                   const int* __restrict__ seg_end, float* seg_sum, int64_t lds) {
  pdl_begin();
  pdl_end();
  const int n = head->valid;
  const int next = (blockIdx.x + 1) * kRun;
  if (next >= n) return;
  const int y = sorted[next];
  if (sorted[next - 1] != y) return;
  const int first = seg_first[y] - 1;
  if (first < next - kRun) return;  // starts in an earlier block
  const int end = seg_end[y];
  for (int64_t d = threadIdx.x; d < lds; d += 256) {
    float s = seg_sum[first * lds + d];
#pragma unroll 8
    for (int p = next; p < end; p += kRun) s = fadd(s, seg_sum[p * lds + d]);
    seg_sum[first * lds + d] = s;
  }
}

// dh in the caller's type and order from the splits' sums; zero for tokens that
// do not count.  Times `scale` and plus `coef` times the target's row of w where given.
template <typename E>
__global__ void __launch_bounds__(256)
    ce_dh_out_kernel(int T, int D, int groups, const int* place, const float* sum, int64_t lds, int splits,
                     int64_t sum_split, const float* scale, const float* coef, const E* __restrict__ w, int64_t ldw,
                     const int* target, int wide_w, E* dh, int64_t lddh, int wide) {
  pdl_begin();
  pdl_end();
  for (int64_t q = blockIdx.x * int64_t{256} + threadIdx.x; q < static_cast<int64_t>(T) * groups;
       q += gridDim.x * int64_t{256}) {
    const int t = static_cast<int>(q / groups);
    const int d = static_cast<int>(q - static_cast<int64_t>(t) * groups) * 8;
    const int m = place[t];
    float x[8] = {};
    if (m >= 0) {
#pragma unroll 8
      for (int i = 0; i < splits; ++i) {
        const float4* in = reinterpret_cast<const float4*>(sum + i * sum_split + m * lds + d);
        const float4 a = in[0], b = in[1];
        const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fadd(x[j], v[j]);
      }
      if (scale != nullptr) {
        const float s = scale[m];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fmul(x[j], s);
      }
      if (coef != nullptr) {
        const float c = coef[m];
        E y[8];
        load8(w + target[m] * ldw + d, D - d, wide_w, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __fmaf_rn(c, to_float(y[j]), x[j]);
      }
    }
    E out[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) from_float(x[j], &out[j]);
    E* to = dh + t * lddh + d;
    if (wide && d + 8 <= D) {
      uint4 u[sizeof(E) / 2];
      memcpy(u, out, sizeof(out));
#pragma unroll
      for (int k = 0; k < static_cast<int>(sizeof(E)) / 2; ++k) reinterpret_cast<uint4*>(to)[k] = u[k];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (d + j < D) to[j] = out[j];
    }
  }
}

// dw of a piece from the sums of parts of the tokens.
template <typename E>
__global__ void __launch_bounds__(256)
    ce_dw_out_kernel(int width, int D, int groups, const float* __restrict__ sum, int64_t lds, int splits,
                     int64_t sum_split, const int* __restrict__ seg_first, const float* __restrict__ seg_sum, E* dw,
                     int64_t lddw, int wide) {
  pdl_begin();
  pdl_end();
  for (int64_t q = blockIdx.x * int64_t{256} + threadIdx.x; q < static_cast<int64_t>(width) * groups;
       q += gridDim.x * int64_t{256}) {
    const int64_t v = q / groups;
    const int d = static_cast<int>(q - v * groups) * 8;
    float x[8] = {};
    auto add = [&](const float* from) {
      const float4 a = reinterpret_cast<const float4*>(from)[0], b = reinterpret_cast<const float4*>(from)[1];
      const float y[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = fadd(x[j], y[j]);
    };
#pragma unroll 4
    for (int i = 0; i < splits; ++i) add(sum + i * sum_split + v * lds + d);
    const int first = seg_first != nullptr ? seg_first[v] : 0;
    if (first > 0) add(seg_sum + (first - 1) * lds + d);
    E out[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) from_float(x[j], &out[j]);
    E* to = dw + v * lddw + d;
    if (wide && d + 8 <= D) {
      uint4 u[sizeof(E) / 2];
      memcpy(u, out, sizeof(out));
#pragma unroll
      for (int k = 0; k < static_cast<int>(sizeof(E)) / 2; ++k) reinterpret_cast<uint4*>(to)[k] = u[k];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (d + j < D) to[j] = out[j];
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
// A training step keeps the exponentials where they take 4 GiB at most and the
// tokens are few enough to be ordered by counting pairs (16384: 2^28 pairs, 20 us);
// beyond either it forms the logits twice, a third more operations.  So it does
// for the bf16 tokens of one row tile: there the products wait for w, and an entry
// of dw, a sum of few terms then, is spared one of its roundings (of g/s h); the
// targets' c, which dominate such sums, are added to dh and dw in fp32.
constexpr int64_t kKeptBytes = int64_t{4} << 30;
constexpr int64_t kKeptTokens = 16384;

enum Pass { kForward = 0, kBackward = 1, kTrain = 2 };

struct Layout {
  size_t head, counts, row, target, place, at_target, part, lse, h, w, coef, sum, dw_sum, total;
  size_t flags, pos, order, sorted, ref, sums, scale, factor, hs, seg_first, seg_end, seg_sum;  // kept
  int parts, planes, tiles;
  bool pack_w, kept, apart, over;
  int64_t piece, padded, Dp, ldc;
};

// Widths of tiles, and parts of K for dh, by an estimate of the products' time in
// cycles: waves of tiles over the SM pairs, a K block of a tile bound by its copies
// from L2 (about 60 bytes a cycle an SM: in bf16 546 cycles for 256 columns, 410
// for 128, 341 for 64) or its products (512, 256, 128; in fp32 six times as many on
// three times the bytes), an epilogue a tile, and for each part its sums written
// and read once more.
constexpr int kPairs = 76;  // of the 152 SMs
constexpr int kMaxSplits = 32;

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

// dw in parts needs its sums and one more pass, for a vocabulary of few tiles.
constexpr int kMostDwSplits = 16;
Plan plan_dw(int64_t T, int64_t D, int64_t piece, int planes) {
  return plan_tiles(piece, D, (T + kK - 1) / kK, planes, 64, kMostDwSplits);
}

Plan plan_dh(int64_t T, int64_t D, int64_t piece, int planes) {
  return plan_tiles(T, D, (piece + kK - 1) / kK, planes, 64, kMaxSplits);
}

Layout layout(int64_t T, int64_t D, int64_t V, bool bf16, int pass, int64_t piece, int64_t ldw) {
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
  l.tiles = static_cast<int>(l.padded / kPair);
  l.Dp = round_up(D, 8);
  l.parts = static_cast<int>((V + kHalf - 1) / kHalf);
  l.head = take(sizeof(Header));
  l.counts = take(T > kScanAlone ? (T + kScan - 1) / kScan * 4 : 0);
  l.row = take(T * 4);
  l.target = take(T * 4);
  l.place = take(T * 4);
  l.at_target = take(T * 4);
  l.lse = take(T * 4);
  l.part = take(static_cast<size_t>(l.parts) * T * 8);
  l.h = take(static_cast<size_t>(l.planes) * l.padded * l.Dp * 2);
  l.w = take(l.pack_w ? static_cast<size_t>(l.planes) * V * l.Dp * 2 : 0);
  if (pass == kForward) {
    l.total = at;
    return l;
  }
  l.kept = pass == kTrain && (!bf16 || T > kPair) && T <= kKeptTokens && (piece == 0 || piece >= V) &&
           l.padded * round_up(V, kN) * 2 * l.planes <= kKeptBytes;
  const int64_t most = std::max<int64_t>(kN, kPieceBytes / (l.padded * 2 * l.planes) / kN * kN);
  l.piece = l.kept ? V : std::min(V, piece > 0 ? piece : most);
  l.ldc = round_up(l.piece, kN);
  l.coef = take(static_cast<size_t>(l.planes) * l.padded * l.ldc * 2);
  const Plan dw = plan_dw(T, D, l.piece, l.planes);
  l.dw_sum = take(dw.splits > 1 ? static_cast<size_t>(dw.splits) * l.piece * l.Dp * 4 : 0);
  l.sum = take(static_cast<size_t>(plan_dh(T, D, l.piece, l.planes).splits) * l.padded * l.Dp * 4);
  l.apart = !l.kept && bf16 && T <= kPair;
  l.over = !l.kept && bf16 && T > kPair;
  if (l.kept || l.over) l.hs = take(static_cast<size_t>(l.planes) * l.padded * l.Dp * 2);
  if (l.over)
    for (size_t* p : {&l.ref, &l.scale, &l.factor}) *p = take(T * 4);
  if (l.kept || l.apart) {
    l.flags = take(round_up(l.tiles, kScan / kPair) * 4);
    for (size_t* p : {&l.pos, &l.order, &l.sorted, &l.ref, &l.sums, &l.scale, &l.factor}) *p = take(T * 4);
    l.seg_first = take(V * 4);
    l.seg_end = take(V * 4);
    l.seg_sum = take(static_cast<size_t>(T) * l.Dp * 4);
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

template <int MODE, int PLANES>
cudaError_t launch_gemm(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& c, const Gemm& g, int64_t m, int64_t n, int num_sms,
                        cudaStream_t s) {
  const int64_t tiles = (m + kPair - 1) / kPair * ((n + g.tile_n - 1) / g.tile_n) *
                        (MODE == kDh || MODE == kDw ? g.splits : 1);
  if (tiles > 0x7fffffff - num_sms) return cudaErrorInvalidValue;
  constexpr bool stores = MODE == kExp || MODE == kCoef;
  constexpr int smem = kStages * kStageBytes + 1024 + (stores ? kEpiWarps * kStoreBytes : 0);
  const cudaError_t e = ensure_dynamic_smem(ce_gemm_kernel<MODE, PLANES>, smem);
  if (e != cudaSuccess) return e;
  const unsigned grid = static_cast<unsigned>(2 * std::min<int64_t>(tiles, num_sms / 2));
  return launch_kernel(ce_gemm_kernel<MODE, PLANES>, dim3(grid), dim3(kGemmThreads), smem, s, 2, a, b, c, g);
}

#define CE_TRY(...)                       \
  do {                                    \
    const cudaError_t e_ = (__VA_ARGS__); \
    if (e_ != cudaSuccess) return e_;     \
  } while (0)

template <typename E>
cudaError_t run(const LinearCeArgs& a, int num_sms, cudaStream_t s) {
  constexpr bool bf16 = sizeof(E) == 2;
  constexpr int P = bf16 ? 1 : 3;
  const int T = static_cast<int>(a.T), D = static_cast<int>(a.D);
  auto on16 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
  const int pass = a.dw == nullptr ? kForward : a.loss == nullptr ? kBackward : kTrain;
  const Layout l = layout(a.T, a.D, a.V, bf16, pass, a.piece, on16(a.w) ? a.ldw : 0);
  char* ws = static_cast<char*>(a.ws);
  auto ints = [&](size_t at) { return reinterpret_cast<int*>(ws + at); };
  auto floats = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
  Header* head = reinterpret_cast<Header*>(ws + l.head);
  int *row = ints(l.row), *target = ints(l.target), *place = ints(l.place);
  uint16_t* hp = reinterpret_cast<uint16_t*>(ws + l.h);
  uint16_t* wp = reinterpret_cast<uint16_t*>(ws + l.w);
  const E* h = static_cast<const E*>(a.h);
  const E* w = static_cast<const E*>(a.w);
  const int wide_h = on16(h) && a.ldh * sizeof(E) % 16 == 0, wide_w = on16(w) && a.ldw * sizeof(E) % 16 == 0;
  const int wide_dh = on16(a.dh) && a.lddh * sizeof(E) % 16 == 0;
  const int Dp = static_cast<int>(l.Dp);
  const unsigned rows8 = static_cast<unsigned>(l.padded / 8), rows32 = static_cast<unsigned>((a.T + 31) / 32);
  const bool by_target = l.kept || l.apart;
  const dim3 scans(static_cast<unsigned>((a.T + kScan - 1) / kScan));
  int* counts = a.T > kScanAlone ? ints(l.counts) : nullptr;
  if (counts != nullptr)
    CE_TRY(launch_kernel(ce_count_kernel, scans, dim3(kScan), 0, s, 0, a.targets, T, a.V, a.ignore, counts));
  CE_TRY(launch_kernel(ce_scan_kernel, scans, dim3(kScan), 0, s, 0, a.targets, T, a.V, a.ignore, counts, head,
                       row, target, place, by_target ? ints(l.pos) : nullptr,
                       l.kept ? ints(l.flags) : nullptr, a.status));
  Prepare<E> pre = {head, h, w, a.ldh, a.ldw, a.V, l.padded, D, Dp, wide_h, wide_w, row, target, hp, wp,
                    by_target || (l.over && a.loss == nullptr) ? floats(l.ref) : nullptr, by_target ? ints(l.pos) : nullptr, rows8, 0, 0, 0};
  if (l.pack_w)
    pre.w_blocks = static_cast<unsigned>(std::min<int64_t>((a.V * (Dp / 8) + 255) / 256, int64_t{num_sms} * 16));
  if (by_target) {
    pre.rank_x = static_cast<unsigned>((a.T + 255) / 256);
    pre.rank_y = std::min(pre.rank_x, 32u);
  }
  CE_TRY(launch_kernel(ce_prepare_kernel<E, P>, dim3(pre.h_blocks + pre.w_blocks + pre.rank_x * pre.rank_y), dim3(256), 0,
                       s, 0, pre));
  const void* wt = l.pack_w ? static_cast<const void*>(wp) : w;
  const int64_t wld = l.pack_w ? l.Dp : a.ldw;
  const int64_t hplane = l.padded * l.Dp, wplane = a.V * wld;
  CUtensorMap h_rows, w_rows;  // K = D contiguous
  CE_TRY(make_map(&h_rows, hp, D, l.padded, P, l.Dp, hplane, kM));
  const int64_t d_blocks = (a.D + kK - 1) / kK;
  const int logits_n = plan_tiles(a.T, a.V, d_blocks, P, 128, 1).tile_n;
  CE_TRY(make_map(&w_rows, wt, D, a.V, P, wld, wplane, logits_n / 2));
  Gemm g = {};
  g.head = head;
  g.row = row;
  g.target = target;
  g.T = T;
  g.D = D;
  g.spin_limit = a.spin_limit;
  g.status = a.status;
  g.part = reinterpret_cast<float2*>(ws + l.part);
  g.at_target = floats(l.at_target);
  uint16_t* coef = reinterpret_cast<uint16_t*>(ws + l.coef);
  const int64_t coef_plane = l.padded * l.ldc;
  g.sum = floats(l.sum);
  g.lds = l.Dp;
  g.sum_split = l.padded * l.Dp;
  g.dw = a.dw;
  g.lddw = a.lddw;
  g.dw_bf16 = bf16;
  g.dw_wide = (a.lddw * sizeof(E)) % 32 == 0 && reinterpret_cast<uintptr_t>(a.dw) % 32 == 0;
  // K blocks of an accumulator (4 truncating steps each in bf16, 24 in fp32; see
  // linear_ce_gemm.cuh).  fp32: two, 48 steps (four measured 3 to 8 % faster and
  // 1.3e-6 off, more than an fp32 sum).  bf16 logits, whose loss is fp32: equal chunks
  // of up to 12, and 2 for few tokens, where the products wait for memory anyway.
  // bf16 gradients: 128, which costs nothing that shows.  (Without a limit dh over 262144
  // entries whose first were the largest was 3.3e-4 too small, over 131072 1.2e-4.)
  const int many = 128, exact = 2;
  const int64_t parts = (d_blocks + 11) / 12;
  const int logits = !bf16 || a.T <= kPair ? exact : static_cast<int>((d_blocks + parts - 1) / parts);
  const int gradients = bf16 ? many : exact;
  const Plan dh_plan = pass == kForward ? Plan{kN, 1} : plan_dh(a.T, a.D, l.piece, P);
  const Plan dw_plan = pass == kForward ? Plan{kN, 1} : plan_dw(a.T, a.D, l.piece, P);
  const int wide_dw = on16(a.dw) && a.lddw * sizeof(E) % 16 == 0;
  const unsigned out_blocks =
      static_cast<unsigned>(std::min<int64_t>((a.T * (Dp / 8) + 255) / 256, int64_t{num_sms} * 16));
  auto dh_out = [&](const float* scale, const float* coef) {
    return launch_kernel(ce_dh_out_kernel<E>, dim3(out_blocks), dim3(256), 0, s, 0, T, D, Dp / 8, place, g.sum, g.lds,
                         g.splits, g.sum_split, scale, coef, w, a.ldw, target, wide_w, static_cast<E*>(a.dh), a.lddh,
                         wide_dh);
  };
  // dw of the piece in g, from the maps of c^T and of h^T
  auto dw_of_piece = [&](const CUtensorMap& c, const CUtensorMap& hm) {
    Gemm d = g;
    d.tile_n = dw_plan.tile_n;
    d.splits = dw_plan.splits;
    d.sum = dw_plan.splits > 1 ? floats(l.dw_sum) : nullptr;
    d.sum_split = l.piece * l.Dp;
    CE_TRY(launch_gemm<kDw, P>(c, hm, hm, d, d.width, a.D, num_sms, s));
    if (d.sum == nullptr) return cudaSuccess;
    const int64_t blocks = std::min<int64_t>((static_cast<int64_t>(d.width) * (Dp / 8) + 255) / 256, int64_t{num_sms} * 16);
    return launch_kernel(ce_dw_out_kernel<E>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, s, 0, d.width, D, Dp / 8,
                         d.sum, d.lds, d.splits, d.sum_split, d.seg_first == nullptr ? nullptr : d.seg_first + d.v0,
                         d.seg_sum, static_cast<E*>(a.dw) + d.v0 * a.lddw, a.lddw, wide_dw);
  };
  CUtensorMap w_cols, h_cols, c_rows, c_cols;  // K = vocabulary, tokens: boxes of 64 columns x 64 k
  CUtensorMap c_out;                           // boxes of 64 columns x 32 rows
  if (pass != kForward) CE_TRY(make_map(&w_cols, wt, D, a.V, P, wld, wplane, kK));

  int* pos = ints(l.pos);
  float *ref = floats(l.ref), *scale = floats(l.scale), *factor = floats(l.factor);
  Finish f = {T, D, Dp, l.parts, a.V, l.padded, head, row, target, place, pos, ints(l.flags), g.part, g.at_target, ref,
              floats(l.sums), a.gloss, hp, a.lse_in, nullptr, nullptr, scale, factor, ints(l.order), ints(l.sorted),
              ints(l.seg_first), a.loss};
  auto by_targets = [&] {  // the factors, then the targets' part of dw
    CE_TRY(launch_kernel(ce_scale_kernel<P>, dim3(rows8), dim3(256), 0, s, 0, f));
    g.seg_first = f.seg_first;
    g.seg_sum = floats(l.seg_sum);
    const unsigned runs = static_cast<unsigned>((a.T + kRun - 1) / kRun);
    CE_TRY(launch_kernel(ce_target_kernel<P>, dim3(runs), dim3(256), 0, s, 0, head, f.order, f.sorted, factor, hp, hplane,
                         Dp, f.seg_first, ints(l.seg_end), floats(l.seg_sum), l.Dp));
    return launch_kernel(ce_join_kernel, dim3(runs), dim3(256), 0, s, 0, head, f.sorted, f.seg_first, ints(l.seg_end),
                         floats(l.seg_sum), l.Dp);
  };

  if (l.kept) {
    uint16_t* hs = reinterpret_cast<uint16_t*>(ws + l.hs);
    f.hs = hs;
    CE_TRY(make_map(&c_out, coef, a.V, l.padded, P, l.ldc, coef_plane, 32));
    g.width = static_cast<int>(a.V);
    g.ref = ref;
    g.chunk = logits;
    g.tile_n = logits_n;
    CE_TRY(launch_gemm<kExp, P>(h_rows, w_rows, c_out, g, a.T, a.V, num_sms, s));
    CE_TRY(launch_kernel(ce_sum_kernel, dim3(rows32), dim3(1024), 0, s, 0, T, head, g.part, l.parts, floats(l.sums), ref,
                         ints(l.flags)));
    g.redo = ints(l.flags);
    CE_TRY(launch_gemm<kExp, P>(h_rows, w_rows, c_out, g, a.T, a.V, num_sms, s));
    CE_TRY(by_targets());
    CE_TRY(make_map(&h_cols, hs, D, l.padded, P, l.Dp, hplane, kK));
    CE_TRY(make_map(&c_rows, coef, a.V, l.padded, P, l.ldc, coef_plane, kM));
    CE_TRY(make_map(&c_cols, coef, a.V, l.padded, P, l.ldc, coef_plane, kK));
    g.first = 1;
    g.splits = dh_plan.splits;
    g.tile_n = dh_plan.tile_n;
    g.chunk = gradients;
    CE_TRY(launch_gemm<kDh, P>(c_rows, w_cols, w_cols, g, a.T, a.D, num_sms, s));
    CE_TRY(dh_out(scale, factor));
    return dw_of_piece(c_cols, h_cols);
  }

  const float* lse = a.lse_in;
  if (a.loss != nullptr) {
    float* out = a.lse != nullptr ? a.lse : floats(l.lse);
    g.width = static_cast<int>(a.V);
    g.chunk = logits;
    g.tile_n = logits_n;
    CE_TRY(launch_gemm<kLoss, P>(h_rows, w_rows, w_rows, g, a.T, a.V, num_sms, s));
    CE_TRY(launch_kernel(ce_finish_kernel, dim3(rows32), dim3(1024), 0, s, 0, T, head, row, place, g.part, l.parts,
                         g.at_target, a.loss, out));
    lse = out;
  }
  if (pass == kForward) return cudaSuccess;
  g.lse = lse;
  g.gloss = a.gloss;
  g.loss = a.loss;
  if (l.apart) {
    g.apart = 1;
    f.lse = lse;
    f.loss_in = a.loss;
    CE_TRY(by_targets());
  }
  const uint16_t* h_dw = hp;
  if (l.over) {
    uint16_t* hs = reinterpret_cast<uint16_t*>(ws + l.hs);
    f.hs = hs;
    f.lse = lse;
    f.loss_in = a.loss;
    CE_TRY(launch_kernel(ce_over_kernel<P>, dim3(rows8), dim3(256), 0, s, 0, f));
    g.over = factor;
    h_dw = hs;
  }
  g.splits = dh_plan.splits;
  CE_TRY(make_map(&h_cols, h_dw, D, l.padded, P, l.Dp, hplane, kK));
  for (int64_t v0 = 0; v0 < a.V; v0 += l.piece) {
    const int width = static_cast<int>(std::min(l.piece, a.V - v0));
    g.v0 = v0;
    g.width = width;
    g.first = v0 == 0;
    CE_TRY(make_map(&c_rows, coef, width, l.padded, P, l.ldc, coef_plane, kM));
    CE_TRY(make_map(&c_cols, coef, width, l.padded, P, l.ldc, coef_plane, kK));
    CE_TRY(make_map(&c_out, coef, width, l.padded, P, l.ldc, coef_plane, 32));
    g.chunk = bf16 ? many : logits;
    g.tile_n = logits_n;
    CE_TRY(launch_gemm<kCoef, P>(h_rows, w_rows, c_out, g, a.T, width, num_sms, s));
    g.chunk = gradients;
    g.tile_n = dh_plan.tile_n;
    CE_TRY(launch_gemm<kDh, P>(c_rows, w_cols, w_cols, g, a.T, a.D, num_sms, s));
    CE_TRY(dw_of_piece(c_cols, h_cols));
  }
  return dh_out(l.over ? scale : nullptr, l.apart ? factor : nullptr);
}

}  // namespace

size_t linear_ce_workspace_bytes(int64_t T, int64_t D, int64_t V, int bf16, int pass, int64_t piece, int64_t ldw) {
  if (linear_ce_few_fits(T, D, V, ldw, bf16 != 0, pass != kForward))
    return linear_ce_few_workspace_bytes(T, D, V, pass != kForward);
  return layout(T, D, V, bf16 != 0, pass, piece, ldw).total;
}

cudaError_t launch_linear_ce(const LinearCeArgs& a, int num_sms, cudaStream_t s) {
  const int64_t ldw = reinterpret_cast<uintptr_t>(a.w) % 16 == 0 ? a.ldw : 0;
  if (linear_ce_few_fits(a.T, a.D, a.V, ldw, a.bf16 != 0, a.dw != nullptr))
    return launch_linear_ce_few(a, num_sms, s);
  return a.bf16 ? run<__nv_bfloat16>(a, num_sms, s) : run<float>(a, num_sms, s);
}

}  // namespace mpc
