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
// Warp 0 copies operand tiles through tensor maps, one thread of the first CTA's warp 1
// issues the products of both CTAs, eight warps a CTA take the finished tile from tensor
// memory, which holds two accumulators: a tile's epilogue runs under the next one's
// products.  bf16: five stages of 32 KB a CTA and two 4 KB boxes an epilogue warp for what
// it loads and stores (32 rows of 128 bytes, by tensor maps); fp32: two stages of three
// planes, which serve six plane products, and one box.
//
// An accumulator truncates as it adds (1.7e-7 of a large value a step of 16 at most), so it
// sums `chunk` K blocks, and the epilogue adds the chunks in fp32 rounded to nearest: 2
// for fp32, whose results keep fp32's digits, 128 for bf16.
// ---------------------------------------------------------------------------
enum LinearMode { kForward, kDx, kDw };

struct LinearGemm {
  int m, n;            // of C
  int blocks;          // K blocks of 64
  int m_tiles, n_tiles, splits;
  int group;           // row tiles that run together over all columns
  int tile_n, chunk;
  float* sum;          // parts of K (else nullptr): [split][m][lds]
  int64_t lds, sum_split;
  int mapped;          // y, z and residual go through tensor maps
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

template <int PLANES>
struct LinearTiles {
  static constexpr int kStages = PLANES == 1 ? 5 : 2;
  static constexpr int kBoxes = PLANES == 1 ? 2 : 1;  // of an epilogue warp
  static constexpr int kBoxBytes = 4096;
  static constexpr int kSmem = kStages * PLANES * kStageBytes + kEpiWarps * kBoxes * kBoxBytes + 1024;
};

struct LinearTile {
  int m0, n0, split, k0, k1;  // K blocks [k0, k1)
};
// The tiles that run at the same time, one a pair, are `group` row tiles by as many column
// tiles: of 76 pairs, 8 x 9.5 read 18 strips of operands where one row tile after the
// other over all of a large x would read it from HBM once a wave.
__device__ __forceinline__ LinearTile linear_tile(const LinearGemm& g, int i) {
  LinearTile t;
  const int per_split = g.m_tiles * g.n_tiles;
  t.split = i / per_split;
  i -= t.split * per_split;
  const int band = g.group * g.n_tiles, b = i / band, first = b * g.group;
  const int rows = min(g.group, g.m_tiles - first);
  i -= b * band;
  t.m0 = (first + i % rows) * kPair;
  t.n0 = i / rows * g.tile_n;
  t.k0 = static_cast<int>(static_cast<int64_t>(g.blocks) * t.split / g.splits);
  t.k1 = static_cast<int>(static_cast<int64_t>(g.blocks) * (t.split + 1) / g.splits);
  return t;
}

// A lane's 128 bytes of a box of 32 rows, 16-byte groups swizzled as the tensor maps do.
template <typename T>
__device__ __forceinline__ void box_put(uint8_t* box, const float* v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    float f[kVec<T>];
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) f[i] = v[c * kVec<T> + i];
    *reinterpret_cast<uint4*>(box + lane * 128 + ((c ^ (lane & 7)) * 16)) = pack16(f);
  }
}
template <typename T>
__device__ __forceinline__ void box_add(const uint8_t* box, float* v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    float f[kVec<T>];
    unpack16(*reinterpret_cast<const uint4*>(box + lane * 128 + ((c ^ (lane & 7)) * 16)), f);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) v[c * kVec<T> + i] = fadd(f[i], v[c * kVec<T> + i]);
  }
}
template <typename T>
__device__ __forceinline__ T* box_at(uint8_t* box, int row, int col) {
  const int at = col * static_cast<int>(sizeof(T));
  return reinterpret_cast<T*>(box + row * 128 + (((at >> 4) ^ (row & 7)) << 4) + (at & 15));
}
// A box to or from rows that tensor maps do not reach: neighbouring lanes neighbouring entries.
template <typename T, bool LOAD>
__device__ __forceinline__ void box_rows(uint8_t* box, T* p, int64_t ld, int rows, int cols) {
  constexpr int W = 128 / sizeof(T);
  const int lane = threadIdx.x & 31;
  __syncwarp();
#pragma unroll 8
  for (int r = 0; r < 32; ++r) {
#pragma unroll
    for (int c = lane; c < W; c += 32) {
      if (r < rows && c < cols) {
        if (LOAD) *box_at<T>(box, r, c) = p[r * ld + c];
        else p[r * ld + c] = *box_at<T>(box, r, c);
      }
    }
  }
  __syncwarp();
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
  uint64_t z = splitmix64_at(seed, first >> 2);
#pragma unroll
  for (int q = 0; q < W / 4; ++q) {
    uint64_t use = z;
    if (off != 0 || q + 1 < W / 4) z = splitmix64_at(seed, (first >> 2) + q + 1);
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

// What an epilogue warp keeps of its boxes between tiles.
template <int PLANES>
struct Boxes {
  uint8_t* box;        // [kBoxes][4 KB]
  uint64_t* loaded;    // [kBoxes]
  uint32_t phase;      // bit b: parity of the next load into box b
  uint32_t flying;     // bit b: a load into box b has not been waited for
  uint32_t turn;       // of stores that take the boxes in turn
};
// The next box to store from, without a residual: the last store from it has been read.
template <int PLANES>
__device__ __forceinline__ uint8_t* next_box(Boxes<PLANES>& b) {
  constexpr int kBoxes = LinearTiles<PLANES>::kBoxes;
  if ((threadIdx.x & 31) == 0) {
    if (kBoxes == 1) bulk_wait_read();
    else bulk_wait_read_but_one();
  }
  __syncwarp();
  return b.box + (b.turn++ & (kBoxes - 1)) * LinearTiles<PLANES>::kBoxBytes;
}

// One lane's row of a half tile: x[j] = C[m][n0 + j], j < 128.  m0: row of lane 0.
template <int MODE, int PLANES>
__device__ __forceinline__ bool linear_epilogue(const LinearGemm& g, const LinearTile& t, int m0, int n0, uint64_t seed,
                                                float (&x)[kHalf], Boxes<PLANES>& b, const CUtensorMap* map_y,
                                                const CUtensorMap* map_z, const CUtensorMap* map_r) {
  using T = typename std::conditional<PLANES == 1, __nv_bfloat16, float>::type;
  constexpr int W = 128 / sizeof(T), kBoxes = LinearTiles<PLANES>::kBoxes;
  const int lane = threadIdx.x & 31, m = m0 + lane;
  if (m0 >= g.m) return true;
  if (g.sum != nullptr) {
    if (m >= g.m) return true;
    float* out = g.sum + t.split * g.sum_split + m * g.lds + n0;
    const int cols = min(static_cast<int>(g.lds) - n0, g.tile_n);
#pragma unroll
    for (int j = 0; j < kHalf; j += 8) {
      if (j < cols) {
        uint32_t u[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) u[q] = __float_as_uint(x[j + q]);
        st_v8(out + j, u);
      }
    }
    return true;
  }
  const int rows = min(g.m - m0, 32);
#pragma unroll
  for (int h = 0; h < kHalf / W; ++h) {
    const int n = n0 + h * W, left = g.n - n;
    if (left <= 0 || h * W >= g.tile_n) continue;
    const int at = h & (kBoxes - 1);  // the box of the residual, where y takes its place
    uint8_t* box = b.box + at * LinearTiles<PLANES>::kBoxBytes;
    float* v = x + h * W;
    if (MODE == kForward) {
      if (g.bias != nullptr) add_bias<T, W>(static_cast<const T*>(g.bias) + n, g.bias_wide, left, v);
      if (g.z != nullptr) {
        uint8_t* zbox = next_box<PLANES>(b);
        box_put<T>(zbox, v);
        if (g.mapped) {
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) tensor_s2g(map_z, n, m0, 0, zbox);
        } else {
          box_rows<T, false>(zbox, static_cast<T*>(g.z) + m0 * g.ldz + n, g.ldz, rows, left);
        }
      }
      apply_act<W, PLANES == 1>(g.act, v);
      if (g.drop.level > 0) apply_drop<W>(g.drop, seed, static_cast<uint64_t>(m) * g.n + n, v);
      if (g.residual != nullptr) {
        if (g.mapped) {
          if (!(b.flying >> at & 1)) {
            if (lane == 0) {
              bulk_wait_read();
              mbar_arrive_expect_tx(&b.loaded[at], LinearTiles<PLANES>::kBoxBytes);
              tensor_g2s_own(box, map_r, n, m0, 0, smem_addr(&b.loaded[at]));
            }
            b.flying |= 1u << at;
          }
          const bool ok = mbar_wait_bounded(&b.loaded[at], b.phase >> at & 1, g.spin_limit, g.status);
          if (!__all_sync(kFull, ok)) return false;
          b.phase ^= 1u << at;
          b.flying &= ~(1u << at);
        } else {
          box_rows<T, true>(box, const_cast<T*>(static_cast<const T*>(g.residual)) + m0 * g.ldr + n, g.ldr, rows, left);
        }
        box_add<T>(box, v);
      } else {
        box = next_box<PLANES>(b);
      }
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) v[j] = fmul(v[j], g.drop.scale);
      box = next_box<PLANES>(b);
    }
    box_put<T>(box, v);
    if (g.mapped) {
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tensor_s2g(map_y, n, m0, 0, box);
    } else {
      box_rows<T, false>(box, static_cast<T*>(g.y) + m0 * g.ldy + n, g.ldy, rows, left);
    }
  }
  return true;
}

template <int MODE, int PLANES>
__global__ void __launch_bounds__(kGemmThreads, 1)
    linear_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                       const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_z,
                       const __grid_constant__ CUtensorMap map_r, const __grid_constant__ LinearGemm g) {
  constexpr bool A_MN = MODE == kDw, B_MN = MODE != kForward;
  constexpr int stages = LinearTiles<PLANES>::kStages, kBoxes = LinearTiles<PLANES>::kBoxes;
  extern __shared__ uint8_t raw[];
  // full and taken are used in the first CTA, for both; empty and done in each
  __shared__ uint64_t full[stages], empty[stages], done[2], taken[2], drain, loaded[kEpiWarps * kBoxes];
  __shared__ uint32_t tmem;
  uint8_t* stage0 = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = static_cast<int>(cluster_rank());
  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&done[i], 1);
      mbar_init(&taken[i], 2 * kEpiWarps);
    }
    for (int i = 0; i < kEpiWarps * kBoxes; ++i) mbar_init(&loaded[i], 1);
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
  const int total = g.m_tiles * g.n_tiles * g.splits;
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (warp == 0) {
    if (lane == 0) {
      fence_proxy_async_all();  // operands that earlier kernels wrote
      uint32_t it = 0;
      bool ok = true;
      // a CTA's rows of B in a stage: half the tile's, in blocks of 64 where they are columns
      const int b_blocks = (g.tile_n / 2 + 63) / 64;
      const uint32_t bytes = 2 * PLANES * (kBytesA + (B_MN ? b_blocks * kK * 128 : g.tile_n / 2 * kK * 2));
      for (int i = pair; i < total && ok; i += pairs) {
        const LinearTile t = linear_tile(g, i);
        const int m0 = t.m0 + rank * kM, n0 = t.n0 + rank * (tile_cols(g.n, t.n0, g.tile_n) / 2);
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
              for (int q = 0; q < b_blocks; ++q) tensor_g2s(b + q * kK * 128, &map_b, n0 + q * 64, kb * kK, p, bar);
            } else {
              tensor_g2s(b, &map_b, kb * kK, n0, p, bar);
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
        const LinearTile t = linear_tile(g, i);
        const uint32_t idesc = mma_desc(kPair, tile_cols(g.n, t.n0, g.tile_n), A_MN, B_MN);
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
    const uint64_t seed = MODE == kForward && g.drop.level > 0 ? drop_seed(g.drop) : 0;
    Boxes<PLANES> boxes = {stage0 + stages * PLANES * kStageBytes + (warp - 2) * kBoxes * LinearTiles<PLANES>::kBoxBytes,
                           loaded + (warp - 2) * kBoxes, 0u, 0u, 0u};
    constexpr int W = 64 * PLANES / (PLANES == 1 ? 1 : 6);  // columns of a box: 64 or 32
    if (MODE == kForward && lane == 0) fence_proxy_async_all();  // a residual that earlier kernels wrote
    uint32_t n = 0;
    bool ok = true;
    for (int i = pair; i < total; i += pairs) {
      const LinearTile t = linear_tile(g, i);
      const int m0 = t.m0 + rank * kM + quad * 32, n0 = t.n0 + half * kHalf;
      // the residual's first boxes come while the products run
      if (MODE == kForward && g.residual != nullptr && g.z == nullptr && g.mapped && g.sum == nullptr && m0 < g.m &&
          half * kHalf < g.tile_n) {
        if (lane == 0) bulk_wait_read();
#pragma unroll
        for (int q = 0; q < kBoxes; ++q) {
          if (n0 + q * W < g.n && half * kHalf + q * W < g.tile_n) {
            if (lane == 0) {
              mbar_arrive_expect_tx(&boxes.loaded[q], LinearTiles<PLANES>::kBoxBytes);
              tensor_g2s_own(boxes.box + q * LinearTiles<PLANES>::kBoxBytes, &map_r, n0 + q * W, m0, 0,
                             smem_addr(&boxes.loaded[q]));
            }
            boxes.flying |= 1u << q;
          }
        }
      }
      float x[kHalf];
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
      ok = linear_epilogue<MODE, PLANES>(g, t, m0, n0, seed, x, boxes, &map_y, &map_z, &map_r);
      if (!ok) break;
    }
    // no copy of this warp is in flight when it leaves
    if (lane == 0) {
      for (int q = 0; q < kBoxes; ++q)
        if (boxes.flying >> q & 1) mbar_wait_bounded(&boxes.loaded[q], boxes.phase >> q & 1, kDrainPolls, g.status);
      bulk_wait();
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

}  // namespace
}  // namespace mpc
