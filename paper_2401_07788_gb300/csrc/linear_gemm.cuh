// linear_gemm.cuh -- the matrix products of the linear layer on the tensor cores, with
// the layer's bias, activation, dropout and residual in their epilogue.
#pragma once

#include "gemm_tiles.cuh"
#include "layers.cuh"

namespace mpc {
namespace {

// ---------------------------------------------------------------------------
// C[m][n] = sum_k A[m][k] B[n][k] in 256 x 256 tiles of a CTA pair, 128 rows each.
//
// kForward  A = x [rows][in],   B = w [out][in]     (K contiguous in both)
// kDx       A = dz [rows][out], B = w^T [in][out]   (B read as it is: rows of 64 entries of `in`)
// kDw       A = dz^T [out][rows], B = x^T [in][rows]  (both read as they are)
//
// Warp 0 copies operand tiles through tensor maps, six stages of 32 KB a CTA, each of one
// plane (fp32's three planes of a K block serve six plane products and are given back
// one by one: 4096^3 took 566 us with two stages of three planes, 454 so).  One lane of the first
// CTA's warp 1 issues the products of both CTAs.  What these two warps do for a K block has to take less
// than the products' 512 cycles, and they wait for every instruction: so all lanes run their loops,
// which keeps the operands of copies and products in uniform registers, and one of them issues
// (8192^3 in bf16 593 us with one lane in the loops, 558 so).  Sixteen warps a CTA take the finished tile from
// tensor memory, 32 rows by twice 32 columns each.  Tensor memory holds two accumulators: a
// tile's epilogue runs under the next one's products, and should take no longer than those
// (512 cycles a K block; 560 to 590 are reached).
//
// What an epilogue takes is latency.  The matrix units and the copies leave little of shared
// memory's bandwidth, so results go from registers to global memory, 64 bytes a lane, and four
// warps a scheduler hide the exponentials of one another; its arrival for the accumulator is a
// relaxed one (a release waits for the stores: 2000 cycles a tile).  8192 x 64 x 8192 in bf16, 14 waves of
// tiles with one K block: 42 us for z alone, 63 with gelu_tanh, 74 with dropout, 100 with both: 5800, 8800, 10300
// and 13900 cycles a tile; no pipe is busy half of the time (with gelu_tanh the one of the special functions 19 %, with
// dropout that of integers 48 %).  Measured in bf16 (one GB300 each, they differ
// by 3 %): 8192 x 1024 x 4096 44 us, with gelu_tanh and bias 58 to 65 (cuBLAS without any of it 37);
// 8192^3 558 us (546); 2000 x 4096 x 8192 81 to 87 (72), whose 256 tiles are 3.4 waves of the 76
// pairs.  Eight stages of 24 KB for tiles of 128 columns were 2 to 3 % slower: their addresses
// are no constants of the loops.
//
// An accumulator truncates as it adds (1.7e-7 of a large value a step of 16 at most), so it
// sums `chunk` K blocks, and the epilogue adds the chunks in fp32 rounded to nearest: 2
// for fp32, whose results keep fp32's digits, 128 for bf16.
// ---------------------------------------------------------------------------
enum LinearMode { kForward, kDx, kDw };

// Quotient and remainder by a divisor that the host knows (a division takes 40 instructions, three of
// them a tile and warp).
struct Divisor {
  uint32_t d, inverse;  // floor(2^32 / d): its quotient is at most one too small
  __device__ __forceinline__ uint32_t of(uint32_t i, uint32_t* rest) const {
    uint32_t q = __umulhi(i, inverse), r = i - q * d;
    if (r >= d) {
      ++q;
      r -= d;
    }
    *rest = r;
    return q;
  }
};
inline Divisor divisor(uint32_t d) {
  return Divisor{d, d == 1 ? 0xffffffffu : static_cast<uint32_t>((uint64_t{1} << 32) / d)};
}

struct LinearGemm {
  int m, n;            // of C
  int blocks;          // K blocks of 64
  int m_tiles, n_tiles;
  int whole;           // tiles formed in one piece; the others, the last ones, in `splits` parts of K
  int splits;
  int group;           // row tiles that run together over all columns
  Divisor band, rows, last_rows;  // by the tiles of a group, its row tiles, those of the last group
  int tile_n, chunk;
  float* sum;          // [split][tiles in parts][256][tile_n]
  int wide;            // y, z and residual have rows on 16 bytes (1), on 32 (2)
  const void* bias;
  int bias_wide;
  const void* residual;
  int64_t ldr;
  void* y;
  int64_t ldy;
  void* z;
  int64_t ldz;
  int act;
  Drop drop;           // its factor scales C of the gradients
  uint32_t spin_limit;
  unsigned* status;
};

constexpr int kLinearEpi = 16;                      // epilogue warps
constexpr int kLinearThreads = (2 + kLinearEpi) * 32;
constexpr int kLinearBox = 2048;                    // 32 rows of 64 bytes, where rows lie on no 16 bytes

template <int PLANES>
struct LinearTiles {
  static constexpr int kStages = 6;  // of one plane of both operands
  static constexpr int kSmem = kStages * kStageBytes + kLinearEpi * kLinearBox + 1024;
};

struct LinearTile {
  int m0, n0, k0, k1;  // K blocks [k0, k1)
  int slot;            // of the sums, -1: a whole tile
};
// The tiles that run at the same time, one a pair, are `group` row tiles by as many column
// tiles: of 76 pairs, 8 x 9.5 read 18 strips of operands where one row tile after the
// other over all of a large x would read it from HBM once a wave.
__device__ __forceinline__ void place_tile(const LinearGemm& g, int i, int* m0, int* n0) {
  uint32_t in, row;
  const uint32_t first = g.band.of(i, &in) * g.group;
  const uint32_t col = (first + g.group <= static_cast<uint32_t>(g.m_tiles) ? g.rows : g.last_rows).of(in, &row);
  *m0 = static_cast<int>(first + row) * kPair;
  *n0 = static_cast<int>(col) * g.tile_n;
}
__device__ __forceinline__ int linear_units(const LinearGemm& g) {
  return g.whole + (g.m_tiles * g.n_tiles - g.whole) * g.splits;
}
__device__ __forceinline__ LinearTile linear_tile(const LinearGemm& g, int i) {
  LinearTile t;
  if (i < g.whole) {
    t.slot = -1;
    t.k0 = 0;
    t.k1 = g.blocks;
  } else {
    const int rest = g.m_tiles * g.n_tiles - g.whole;
    t.slot = i - g.whole;
    const int split = t.slot / rest;
    i = g.whole + t.slot - split * rest;
    t.k0 = static_cast<int>(static_cast<int64_t>(g.blocks) * split / g.splits);
    t.k1 = static_cast<int>(static_cast<int64_t>(g.blocks) * (split + 1) / g.splits);
  }
  place_tile(g, i, &t.m0, &t.n0);
  return t;
}

// 32 columns of a lane's row, from `p` on, of which `left` exist; rows on 16 (or 32) bytes.
template <typename T>
__device__ __forceinline__ void store_wide(T* p, int left, bool wider, const float (&v)[32]) {
  constexpr int V = kVec<T>;
#pragma unroll
  for (int c = 0; c < 32 / V; c += 2) {
    float f[2][V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) f[i / V][i % V] = v[c * V + i];
    const uint4 a = pack16(f[0]), b = pack16(f[1]);
    if (wider && left >= (c + 2) * V) {
      const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      st_v8(p + c * V, u);
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (left >= (c + e + 1) * V) {
          *reinterpret_cast<uint4*>(p + (c + e) * V) = e == 0 ? a : b;
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i)
            if ((c + e) * V + i < left) put(p + (c + e) * V + i, f[e][i]);
        }
      }
    }
  }
}
// The residual's bytes, asked for before they are wanted.
template <typename T>
struct Ahead {
  uint4 u[32 / kVec<T>];
};
template <typename T>
__device__ __forceinline__ void load_wide(const T* p, int left, Ahead<T>& a) {
  constexpr int V = kVec<T>;
#pragma unroll
  for (int c = 0; c < 32 / V; ++c) {
    if (left >= (c + 1) * V) {
      a.u[c] = *reinterpret_cast<const uint4*>(p + c * V);
    } else {
      float f[V];
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] = c * V + i < left ? as_float(p[c * V + i]) : 0.0f;
      a.u[c] = pack16(f);
    }
  }
}
template <typename T>
__device__ __forceinline__ void add_ahead(const Ahead<T>& a, float (&v)[32]) {
  constexpr int V = kVec<T>;
#pragma unroll
  for (int c = 0; c < 32 / V; ++c) {
    float f[V];
    unpack16(a.u[c], f);
#pragma unroll
    for (int i = 0; i < V; ++i) v[c * V + i] = fadd(f[i], v[c * V + i]);
  }
}

template <typename T>
__device__ __forceinline__ void add_wide(const T* p, int left, float (&v)[32]) {
  constexpr int V = kVec<T>;
#pragma unroll
  for (int c = 0; c < 32 / V; ++c) {
    if (left >= (c + 1) * V) {
      float f[V];
      unpack16(*reinterpret_cast<const uint4*>(p + c * V), f);
#pragma unroll
      for (int i = 0; i < V; ++i) v[c * V + i] = fadd(f[i], v[c * V + i]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c * V + i < left) v[c * V + i] = fadd(as_float(p[c * V + i]), v[c * V + i]);
    }
  }
}

// The same where rows lie on no 16 bytes, by way of a warp's 2 KB of shared memory, so that
// neighbouring lanes take neighbouring entries: 64 bytes of 32 rows at a time, a row's
// words swizzled by its number.
template <typename T>
__device__ __forceinline__ uint32_t* box_word(uint8_t* box, int row, int word) {
  return reinterpret_cast<uint32_t*>(box) + row * 16 + (word ^ (row & 15));
}
template <typename T, bool LOAD>
__device__ __forceinline__ void box_rows(uint8_t* box, T* p, int64_t ld, int rows, int left) {
  const int lane = threadIdx.x & 31;
  __syncwarp();
  if (sizeof(T) == 2) {
#pragma unroll 8
    for (int r = 0; r < 32; ++r) {
      uint16_t* at = reinterpret_cast<uint16_t*>(box_word<T>(box, r, lane / 2)) + (lane & 1);
      uint16_t* out = reinterpret_cast<uint16_t*>(p) + r * ld + lane;
      if (r < rows && lane < left) {
        if (LOAD) *at = *out;
        else *out = *at;
      }
    }
  } else {
#pragma unroll 8
    for (int i = 0; i < 16; ++i) {
      const int r = 2 * i + (lane >> 4), c = lane & 15;
      uint32_t* at = box_word<T>(box, r, c);
      uint32_t* out = reinterpret_cast<uint32_t*>(p) + r * ld + c;
      if (r < rows && c < left) {
        if (LOAD) *at = *out;
        else *out = *at;
      }
    }
  }
  __syncwarp();
}
template <typename T>
__device__ __forceinline__ void store_any(uint8_t* box, T* p, int64_t ld, int rows, int left, const float (&v)[32]) {
  constexpr int E = 64 / sizeof(T);  // entries of 64 bytes
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int h = 0; h < 32; h += E) {
    if (h < left) {
#pragma unroll
      for (int w = 0; w < 16; ++w)
        *box_word<T>(box, lane, w) = sizeof(T) == 2 ? pack2(v[(2 * w) % 32], v[(2 * w + 1) % 32]) : __float_as_uint(v[(h + w) % 32]);
      box_rows<T, false>(box, p + h, ld, rows, left - h);
    }
  }
}
template <typename T>
__device__ __forceinline__ void add_any(uint8_t* box, const T* p, int64_t ld, int rows, int left, float (&v)[32]) {
  constexpr int E = 64 / sizeof(T);
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int h = 0; h < 32; h += E) {
    if (h < left) {
      box_rows<T, true>(box, const_cast<T*>(p) + h, ld, rows, left - h);
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        const uint32_t u = *box_word<T>(box, lane, w);
        if (sizeof(T) == 2) {
          v[(2 * w) % 32] = fadd(__uint_as_float(u << 16), v[(2 * w) % 32]);
          v[(2 * w + 1) % 32] = fadd(__uint_as_float(u & 0xffff0000u), v[(2 * w + 1) % 32]);
        } else {
          v[(h + w) % 32] = fadd(__uint_as_float(u), v[(h + w) % 32]);
        }
      }
      __syncwarp();
    }
  }
}

template <int W, bool FAST>
__device__ __forceinline__ void apply_act(int act, float* v) {
#define MPC_EACH(A) \
  case A:           \
    _Pragma("unroll") for (int j = 0; j < W; ++j) v[j] = act_value<FAST>(A, v[j]); \
    break
  switch (act) {
    MPC_EACH(MPC_ACT_RELU);
    MPC_EACH(MPC_ACT_GELU);
    MPC_EACH(MPC_ACT_GELU_TANH);
    MPC_EACH(MPC_ACT_SILU);
    default: break;
  }
#undef MPC_EACH
}

// Entries first .. first + W - 1: a draw serves four that start at a multiple of four; off
// such a multiple the parts of two draws are shifted together.
template <int W>
__device__ __forceinline__ void apply_drop(const Drop& d, uint64_t seed, uint64_t first, float* v) {
  const int off = static_cast<int>(first & 3) * 16;
  Draws draws(seed, first >> 2);
  uint64_t z = draws.next();
#pragma unroll
  for (int q = 0; q < W / 4; ++q) {
    uint64_t use = z;
    if (off != 0 || q + 1 < W / 4) z = draws.next();
    if (off != 0) use = (use >> off) | (z << (64 - off));
#pragma unroll
    for (int k = 0; k < 4; ++k) v[4 * q + k] = kept(use, k, d.level) ? fmul(v[4 * q + k], d.scale) : 0.0f;
  }
}

// bias[n .. n + W) to v; entries from `left` on do not exist.
template <typename T, int W>
__device__ __forceinline__ void add_bias(const T* bias, bool wide, int left, float* v) {
  if (wide && left >= W) {
#pragma unroll
    for (int c = 0; c < W / kVec<T>; ++c) {
      float f[kVec<T>];
      unpack16(reinterpret_cast<const uint4*>(bias)[c], f);
#pragma unroll
      for (int i = 0; i < kVec<T>; ++i) v[c * kVec<T> + i] = fadd(v[c * kVec<T> + i], f[i]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < left) v[j] = fadd(v[j], as_float(bias[j]));
  }
}

// What is done to 32 columns of an epilogue warp's 32 rows, from row m0 and column n on, a row a
// lane: v[j] = C[m0 + lane][n + j].
template <int MODE, int PLANES>
__device__ __forceinline__ void linear_piece(const LinearGemm& g, int m0, int n, uint64_t seed, float (&v)[32],
                                             const Ahead<typename std::conditional<PLANES == 1, __nv_bfloat16, float>::type>& ahead,
                                             uint8_t* box) {
  using T = typename std::conditional<PLANES == 1, __nv_bfloat16, float>::type;
  const int lane = threadIdx.x & 31, m = m0 + lane, rows = min(g.m - m0, 32), left = g.n - n;
  auto store = [&](void* base, int64_t ld) {
    T* p = static_cast<T*>(base) + n;
    if (g.wide == 0) store_any<T>(box, p + m0 * ld, ld, rows, left, v);
    else if (lane < rows) store_wide<T>(p + m * ld, left, g.wide == 2, v);
  };
  if (MODE == kForward) {
    const T* r = static_cast<const T*>(g.residual) + n;
    if (g.bias != nullptr) add_bias<T, 32>(static_cast<const T*>(g.bias) + n, g.bias_wide, left, v);
    if (g.z != nullptr) store(g.z, g.ldz);
    apply_act<32, PLANES == 1>(g.act, v);
    if (g.drop.level > 0) apply_drop<32>(g.drop, seed, static_cast<uint64_t>(m) * g.n + n, v);
    if (g.residual != nullptr) {
      if (PLANES == 1 && g.wide != 0) add_ahead<T>(ahead, v);
      else if (g.wide != 0) add_wide<T>(r + min(m, g.m - 1) * g.ldr, left, v);
      else add_any<T>(box, r + m0 * g.ldr, g.ldr, rows, left, v);
    }
  } else if (g.drop.level > 0) {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = fmul(v[j], g.drop.scale);
  }
  store(g.y, g.ldy);
}

// The same 32 columns of a tile in parts: into its slot of the sums.
__device__ __forceinline__ void sum_piece(const LinearGemm& g, int slot, int row, int col, const float (&v)[32]) {
  float* out = g.sum + (static_cast<int64_t>(slot) * kPair + row) * g.tile_n + col;
#pragma unroll
  for (int j = 0; j < 32; j += 8) {
    uint32_t u[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) u[q] = __float_as_uint(v[j + q]);
    st_v8(out + j, u);
  }
}

__device__ __forceinline__ void landed(float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; ++j) asm volatile("" : "+f"(v[j]));  // nothing uses v before the wait
}

// ONE: a tile has one chunk, and the epilogue takes 32 columns at a time from tensor memory; else it
// keeps its 64 in registers and adds the chunks.
template <int MODE, int PLANES, bool ONE>
__global__ void __launch_bounds__(kLinearThreads, 1)
    linear_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                       const __grid_constant__ LinearGemm g) {
  constexpr bool A_MN = MODE == kDw, B_MN = MODE != kForward;
  constexpr int stages = LinearTiles<PLANES>::kStages;
  extern __shared__ uint8_t raw[];
  // full and taken are used in the first CTA, for both; empty and done in each
  __shared__ uint64_t full[stages], empty[stages], done[2], taken[2], drain;
  __shared__ uint32_t tmem;
  uint8_t* stage0 = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
  const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int rank = blockIdx.x & 1;
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&done[i], 1);
      mbar_init(&taken[i], 2 * kLinearEpi);
    }
    mbar_init(&drain, 1);
    fence_mbar_init();
    prefetch_map(&map_a);
    prefetch_map(&map_b);
  }
  cluster_sync();  // both CTAs have started: the allocation is the pair's
  if (warp == 1) tmem_alloc(&tmem, 512);
  tc_fence_before();
  cluster_sync();  // both have their tensor memory
  tc_fence_after();
  pdl_begin();
  pdl_end();
  const int total = linear_units(g);
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (warp == 0) {
    const bool leader = elect_one();
    fence_proxy_async_all();  // operands that earlier kernels wrote
    uint32_t it = 0;
    bool ok = true;
    // a CTA's rows of B in a stage: half the tile's, in blocks of 64 where they are columns
    const int b_blocks = (g.tile_n / 2 + 63) / 64;
    const uint32_t bytes = 2 * (kBytesA + (B_MN ? b_blocks * kK * 128 : g.tile_n / 2 * kK * 2));
    const uint32_t full0 = dsmem_addr(full, 0);
    uint32_t st = 0, parity = 1;  // of the stage's `empty` to wait for
    for (int i = pair; i < total && ok; i += pairs) {
      const LinearTile t = linear_tile(g, i);
      const int m0 = t.m0 + rank * kM, n0 = t.n0 + rank * (tile_cols(g.n, t.n0, g.tile_n) / 2);
      int kb = t.k0, p = PLANES - 1;  // planes in the order in which they are given back
      for (int left = (t.k1 - t.k0) * PLANES; left > 0; --left, ++it) {
        ok = __all_sync(kFull, mbar_wait_bounded(&empty[st], parity, g.spin_limit, g.status));
        if (!ok) break;
        const uint32_t bar = full0 + st * 8;
        uint8_t* a = stage0 + st * kStageBytes;
        uint8_t* b = a + kBytesA;
        if (leader) {
          if (rank == 0) mbar_arrive_expect_tx(&full[st], bytes);
          if (A_MN) {
#pragma unroll
            for (int q = 0; q < kM / 64; ++q) tensor_g2s(a + q * kK * 128, &map_a, m0 + q * 64, kb * kK, p, bar);
          } else {
            tensor_g2s(a, &map_a, kb * kK, m0, p, bar);
          }
          if (B_MN) {
            for (int q = 0; q < b_blocks; ++q) tensor_g2s(b + q * kK * 128, &map_b, n0 + q * 64, kb * kK, p, bar);
          } else {
            tensor_g2s(b, &map_b, kb * kK, n0, p, bar);
          }
        }
        __syncwarp();
        if (++st == stages) {
          st = 0;
          parity ^= 1;
        }
        if (PLANES == 1 || --p < 0) {
          p = PLANES - 1;
          ++kb;
        }
      }
    }
    // Copies in flight must land before either CTA leaves (the cluster barrier
    // below).  The first CTA's barriers count both CTAs' copies.  The second CTA knows
    // its own by the products that read them, which have not been formed where the
    // first one gave up: then it gives them a millisecond.
    if (lane == 0) {
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
    if (rank == 0) {
      const bool leader = elect_one();
      const uint32_t base = smem_addr(stage0), acc = __shfl_sync(kFull, tmem, 0);
      const uint64_t a0 = A_MN ? smem_desc(base, kK * 128, 1024) : smem_desc(base, 16, 1024);
      const uint64_t b0 = B_MN ? smem_desc(base + kBytesA, kK * 128, 1024) : smem_desc(base + kBytesA, 16, 1024);
      // 16 K-elements on: 32 bytes along a row, or 16 rows of 128 bytes
      constexpr uint64_t kStepA = (A_MN ? 2048 : 32) >> 4, kStepB = (B_MN ? 2048 : 32) >> 4;
      uint32_t st = 0, parity = 0, n = 0;
      bool ok = true;
      LinearTile next = linear_tile(g, pair);
      for (int i = pair; i < total && ok; i += pairs) {
        const LinearTile t = next;
        const uint32_t idesc = mma_desc(kPair, tile_cols(g.n, t.n0, g.tile_n), A_MN, B_MN);
        for (int c = t.k0; c < t.k1 && ok; c += g.chunk, ++n) {
          ok = __all_sync(kFull, mbar_wait_bounded(&taken[n & 1], (n / 2 & 1) ^ 1, g.spin_limit, g.status));
          tc_fence_after();
          const uint32_t d = acc + (n & 1) * kN;
          const int steps = min(g.chunk, t.k1 - c);
          for (int k = 0; k < steps; ++k) {
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
              ok = ok && __all_sync(kFull, mbar_wait_bounded(&full[st + p], parity, g.spin_limit, g.status));
            if (!ok) break;
            tc_fence_after();
            const uint64_t as = a0 + st * (kStageBytes >> 4), bs = b0 + st * (kStageBytes >> 4);
            if (leader) {
#pragma unroll
              for (int term = 0; term < (PLANES == 1 ? 1 : 6); ++term) {
                int pa, pb;
                term_planes<PLANES>(term, &pa, &pb);
#pragma unroll
                for (int q = 0; q < kK / 16; ++q)
                  mma_bf16(d, as + (PLANES - 1 - pa) * (kStageBytes >> 4) + q * kStepA,
                           bs + (PLANES - 1 - pb) * (kStageBytes >> 4) + q * kStepB, idesc, term == 0 && q == 0 && k == 0);
                // a plane is given back after its last product
                if (PLANES == 1 || term == 5) mma_commit_pair(&empty[st + PLANES - 1]);
                else if (term == 1) mma_commit_pair(&empty[st]);
                else if (term == 4) mma_commit_pair(&empty[st + 1]);
              }
              if (k + 1 == steps) mma_commit_pair(&done[n & 1]);
            }
            __syncwarp();
            st += PLANES;
            if (st == stages) {
              st = 0;
              parity ^= 1;
            }
            if (c + k == t.k0) next = linear_tile(g, min(i + pairs, total - 1));  // while these products run
          }
        }
      }
      // products in flight must end before the tensor memory and the stages are given
      // back, also where an epilogue that gave up no longer waits for them
      if (leader) {
        mma_commit(&drain);
        mbar_wait_bounded(&drain, 0, kDrainPolls, g.status);
      }
      __syncwarp();
    }
  } else {
    // its lanes of tensor memory, and the first of its pieces of 32 columns: 64 columns of a
    // wide tile (a lane writes whole lines), one piece of a narrow one
    const int quad = warp & 3, first = ((warp - 2) >> 2) * (g.tile_n > 128 ? 64 : 32);
    const uint32_t acc = tmem;
    const uint64_t seed = MODE == kForward && g.drop.level > 0 ? drop_seed(g.drop) : 0;
    uint8_t* box = stage0 + stages * kStageBytes + (warp - 2) * kLinearBox;
    constexpr int kPieces = 2;
    uint32_t n = 0;
    for (int i = pair; i < total; i += pairs) {
      const LinearTile t = linear_tile(g, i);
      const int m0 = t.m0 + rank * kM + quad * 32, n0 = t.n0 + first;
      const int width = min(g.n - n0, g.tile_n - first);
      const int pieces = m0 < g.m && width > 0 ? min((width + 31) / 32, g.tile_n > 128 ? 2 : 1) : 0;
      const uint32_t columns = first + (static_cast<uint32_t>(quad * 32) << 16);
      const int row = rank * kM + quad * 32 + lane;
      // the residual's bytes come while the products run (fp32: no registers are left for them)
      using T = typename std::conditional<PLANES == 1, __nv_bfloat16, float>::type;
      Ahead<T> ahead[kPieces];
      if (MODE == kForward && PLANES == 1 && g.residual != nullptr && g.wide != 0 && t.slot < 0) {
#pragma unroll
        for (int q = 0; q < kPieces; ++q)
          if (q < pieces)
            load_wide<T>(static_cast<const T*>(g.residual) + min(m0 + lane, g.m - 1) * g.ldr + n0 + 32 * q, g.n - n0 - 32 * q, ahead[q]);
      }
      auto out = [&](int q, float (&v)[32]) {
        if (t.slot >= 0) sum_piece(g, t.slot, row, first + 32 * q, v);
        else linear_piece<MODE, PLANES>(g, m0, n0 + 32 * q, seed, v, ahead[q], box);
      };
      bool ok = true;
      if (ONE) {
        ok = mbar_wait_bounded(&done[n & 1], n / 2 & 1, g.spin_limit, g.status);
        ok = __all_sync(kFull, ok);
        if (!ok) break;
        tc_fence_after();
        const uint32_t at = acc + (n & 1) * kN + columns;
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
          float v[32];
          if (q < pieces) {
            tmem_ld32(at + 32 * q, v);
            tmem_wait_ld();
            landed(v);
          }
          if (q + 1 == max(pieces, 1)) {  // its columns are in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_relaxed(dsmem_addr(&taken[n & 1], 0));
          }
          if (q < pieces) out(q, v);
        }
        ++n;
      } else {
        float x[kPieces][32];
        for (int c = t.k0; c < t.k1; c += g.chunk, ++n) {
          ok = mbar_wait_bounded(&done[n & 1], n / 2 & 1, g.spin_limit, g.status);
          ok = __all_sync(kFull, ok);
          if (!ok) break;
          tc_fence_after();
          const uint32_t at = acc + (n & 1) * kN + columns;
          if (pieces > 0) {
            if (c == t.k0) {
#pragma unroll
              for (int q = 0; q < kPieces; ++q) tmem_ld32(at + 32 * q, x[q]);
              tmem_wait_ld();
#pragma unroll
              for (int q = 0; q < kPieces; ++q) landed(x[q]);
            } else {
#pragma unroll
              for (int q = 0; q < 2 * kPieces; ++q) {
                float y[16];
                tmem_ld16(at + 16 * q, y);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                  asm volatile("" : "+f"(y[j]));
                  x[q / 2][q % 2 * 16 + j] = fadd(x[q / 2][q % 2 * 16 + j], y[j]);
                }
              }
            }
            tc_fence_before();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive_relaxed(dsmem_addr(&taken[n & 1], 0));
        }
        if (!ok) break;
#pragma unroll
        for (int q = 0; q < kPieces; ++q)
          if (q < pieces) out(q, x[q]);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // nothing signals or reads the other CTA's shared memory any more
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace
}  // namespace mpc
