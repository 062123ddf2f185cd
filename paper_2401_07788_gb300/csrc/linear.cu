// linear.cu -- linear layer with bias, activation, dropout and residual, and its gradient.
//
//   z = x w^T + b;   y = r + drop(act(z))
//   dz = drop(dy) act'(z);   dx = dz w;   dw = dz^T x;   db = sum_rows dz
//
// Operands go to the matrix units as bf16 planes (gemm_tiles.cuh): a bf16 operand whose rows
// start on 16 bytes as it is, another one through a copy, an fp32 one split in three.  The
// epilogue of the products (linear_gemm.cuh) does what is done to z; where tiles are cut
// along K, because whole ones would leave SMs without work, linear_finish_kernel adds the parts and
// does it there.  A few rows go another way (linear_few.cu).
//
// Rounded to fewer bits in bf16: z as it is kept for the backward pass (up to 2^-8 of it, which
// moves act' by 0.8 of that at most), and dz for the two products (an error of the size of
// the result's own rounding: dx and dw are 2.4e-3 off 64 bits, where one rounding makes 1.7e-3).
// Dropout's factor stays out of dz: it scales the fp32 sums of dx, dw and db, so a dz without an
// activation is dy's own bits.
//
// What bounds it: the products.  Measured on one GB300: 8192^3 in bf16 558 us (1.97 PFLOP/s;
// cuBLAS 546), 4096^3 in fp32 454 us (six plane products, 1.82 PFLOP/s); training 8192 x 4096 x
// 1024 with dropout and residual 146 to 159 us over several GPUs, 1000 x 777 x 2051 in fp32 with gelu 96.  fp32 of 9 to
// 100 rows splits all of w in every call: 9 x 4096 x 4096 69 us, 64 rows 71, 100 rows 73 (8 rows in linear_few.cu 36).
#include <algorithm>

#include "launch_util.h"
#include "linear_gemm.cuh"

namespace mpc {
namespace {

// ---------------------------------------------------------------------------
// Operands.  One launch: dz with its column sums, and what of x and w is not read in place.
// ---------------------------------------------------------------------------
template <typename E>
struct Operand {
  const E* p;
  int64_t ld, rows, cols, padded;  // padded: columns of a plane's row, a multiple of 8
  int wide;                        // rows on 16 bytes
  uint16_t* out;                   // nullptr: read in place
  unsigned blocks;
};

// Rows of a CTA's part of dz, of 256 columns: up to 128 (8 threads a column group, 16 rows each),
// fewer where that would leave SMs without work (1000 x 2051 in fp32 with gelu took 34 us).
int64_t dz_rows(int64_t rows, int64_t out) {
  int64_t r = 128;
  while (r > 8 && (rows + r - 1) / r * ((out + 255) / 256) < 608) r /= 2;
  return r;
}

template <typename E>
struct Prepare {
  Operand<E> x, w, dy;     // dy.out: the planes of dz, or nullptr where dz is dy itself
  const E* z;
  int64_t ldz;
  int wide_z, act;
  Drop drop;
  float* part;             // column sums of every dz_rows rows, or nullptr
  int dz_rows;
  unsigned dz_cols;        // CTAs along the columns
};

template <typename E, int P>
__device__ __forceinline__ void copy_planes(unsigned block, const Operand<E>& o) {
  const int groups = static_cast<int>(o.padded / 8);
  for (int64_t q = block * int64_t{256} + threadIdx.x; q < o.rows * groups; q += o.blocks * int64_t{256}) {
    const int64_t r = q / groups;
    const int c = static_cast<int>(q - r * groups) * 8;
    E x[8];
    uint16_t p[8][3];
    load8(o.p + r * o.ld + c, static_cast<int>(min64(o.cols - c, 8)), o.wide, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) planes_of<E>(x[j], p[j]);
    store_planes8<P>(o.out + r * o.padded + c, o.rows * o.padded, p);
  }
}

// Eight columns a thread, 32 threads along the columns, 8 along the rows.
template <typename E, int P>
__device__ __forceinline__ void make_dz(unsigned block, const Prepare<E>& f) {
  __shared__ float sums[8][256 + 8];
  const Operand<E>& o = f.dy;
  const int tc = threadIdx.x & 31, tr = threadIdx.x >> 5;
  const int c = static_cast<int>(block % f.dz_cols) * 256 + tc * 8;
  const int64_t chunk = block / f.dz_cols, first = chunk * f.dz_rows;
  const int64_t end = min64(o.rows, first + f.dz_rows);
  const int left = static_cast<int>(o.cols - c);
  const uint64_t seed = f.drop.level > 0 ? drop_seed(f.drop) : 0;
  float sum[8] = {};
  if (left > 0) {
#pragma unroll 2
    for (int64_t r = first + tr; r < end; r += 8) {
      E x[8], zs[8];
      load8(o.p + r * o.ld + c, left, o.wide, x);
      if (f.act != MPC_ACT_NONE) load8(f.z + r * f.ldz + c, left, f.wide_z, zs);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = to_float(x[j]);
      if (f.act != MPC_ACT_NONE) {
#define MPC_EACH(A) \
  case A:           \
    _Pragma("unroll") for (int j = 0; j < 8; ++j) v[j] = fmul(v[j], act_slope<P == 1>(A, to_float(zs[j]))); \
    break
        switch (f.act) {
          MPC_EACH(MPC_ACT_RELU);
          MPC_EACH(MPC_ACT_GELU);
          MPC_EACH(MPC_ACT_GELU_TANH);
          MPC_EACH(MPC_ACT_SILU);
          default: break;
        }
#undef MPC_EACH
        if (left < 8) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j >= left) v[j] = 0.0f;
        }
      }
      if (f.drop.level > 0) {  // last: what z holds in a dropped place reaches nothing
        const uint64_t at = static_cast<uint64_t>(r) * o.cols + c;
        const int off = static_cast<int>(at & 3) * 16;
        Draws draws(seed, at >> 2);
        uint64_t d = draws.next();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint64_t use = d;
          if (off != 0 || q == 0) d = draws.next();
          if (off != 0) use = (use >> off) | (d << (64 - off));
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (!kept(use, k, f.drop.level)) v[4 * q + k] = 0.0f;
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] = fadd(sum[j], v[j]);
      if (o.out != nullptr) {
        uint16_t p[8][3];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (P == 1) p[j][0] = __bfloat16_as_ushort(__float2bfloat16_rn(v[j]));
          else split(v[j], p[j]);
        }
        store_planes8<P>(o.out + r * o.padded + c, o.rows * o.padded, p);
      }
    }
  }
  if (f.part == nullptr) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sums[tr][tc * 8 + j] = sum[j];
  __syncthreads();
  const int64_t col = static_cast<int64_t>(block % f.dz_cols) * 256 + threadIdx.x;
  if (col < o.cols) {
    float v = sums[0][threadIdx.x];
#pragma unroll
    for (int r = 1; r < 8; ++r) v = fadd(v, sums[r][threadIdx.x]);
    f.part[chunk * o.cols + col] = v;
  }
}

template <typename E, int P>
__global__ void __launch_bounds__(256) linear_prepare_kernel(const Prepare<E> f) {
  pdl_begin();
  pdl_end();
  unsigned block = blockIdx.x;
  if (block < f.dy.blocks) {
    make_dz<E, P>(block, f);
    return;
  }
  block -= f.dy.blocks;
  if (block < f.x.blocks) {
    copy_planes<E, P>(block, f.x);
    return;
  }
  copy_planes<E, P>(block - f.x.blocks, f.w);
}

// db from the column sums: 32 columns a CTA, 8 rows of threads.
template <typename E>
struct Bias {
  const float* part;
  int64_t parts, out;
  float scale;
  E* db;
  unsigned blocks;
};
template <typename E>
__device__ __forceinline__ void sum_bias(unsigned block, const Bias<E>& b) {
  __shared__ float sums[8][33];
  const int64_t col = block * int64_t{32} + (threadIdx.x & 31);
  const int r = threadIdx.x >> 5;
  float v = 0.0f;
  if (col < b.out) {
#pragma unroll 8
    for (int64_t p = r; p < b.parts; p += 8) v = fadd(v, b.part[p * b.out + col]);
  }
  sums[r][threadIdx.x & 31] = v;
  __syncthreads();
  if (r == 0 && col < b.out) {
#pragma unroll
    for (int p = 1; p < 8; ++p) v = fadd(v, sums[p][threadIdx.x]);
    put(b.db + col, fmul(v, b.scale));
  }
}

// Four entries that start at a multiple of four of a row on 16 bytes.
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&v)[4]) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
}

// The tiles that were formed in parts of K, four columns a thread, and what the epilogue would have
// done.
struct Finish {
  LinearGemm g;
  unsigned blocks;  // 0: every tile was whole
};
template <typename E, bool FORWARD>
__device__ __forceinline__ void finish_tiles(unsigned block, const Finish& f) {
  const LinearGemm& g = f.g;
  const int rest = g.m_tiles * g.n_tiles - g.whole, groups = g.tile_n / 4;
  const int64_t part = static_cast<int64_t>(rest) * kPair * g.tile_n;
  const uint64_t seed = FORWARD && g.drop.level > 0 ? drop_seed(g.drop) : 0;
  for (int64_t q = block * int64_t{256} + threadIdx.x; q < static_cast<int64_t>(rest) * kPair * groups;
       q += f.blocks * int64_t{256}) {
    const int row = static_cast<int>(q / groups), col = static_cast<int>(q - static_cast<int64_t>(row) * groups) * 4;
    int m0, n0;
    place_tile(g, g.whole + row / kPair, &m0, &n0);
    const int64_t m = m0 + row % kPair;
    const int n = n0 + col, left = min(g.n - n, 4);
    if (m >= g.m || left <= 0) continue;
    const float* from = g.sum + static_cast<int64_t>(row) * g.tile_n + col;
    float4 s = *reinterpret_cast<const float4*>(from);
#pragma unroll 4
    for (int p = 1; p < g.splits; ++p) {
      const float4 a = *reinterpret_cast<const float4*>(from + p * part);
      s = make_float4(fadd(s.x, a.x), fadd(s.y, a.y), fadd(s.z, a.z), fadd(s.w, a.w));
    }
    float v[4] = {s.x, s.y, s.z, s.w};
    auto store = [&](void* base, int64_t ld) {
      E* p = static_cast<E*>(base) + m * ld + n;
      if (g.wide != 0 && left == 4) {
        store4(p, v);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < left) put(p + j, v[j]);
      }
    };
    if (FORWARD) {
      if (g.bias != nullptr) add_bias<E, 4>(static_cast<const E*>(g.bias) + n, false, left, v);
      if (g.z != nullptr) store(g.z, g.ldz);
      apply_act<4, sizeof(E) == 2>(g.act, v);
      if (g.drop.level > 0) apply_drop<4>(g.drop, seed, static_cast<uint64_t>(m) * g.n + n, v);
      if (g.residual != nullptr) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j < left) v[j] = fadd(as_float(static_cast<const E*>(g.residual)[m * g.ldr + n + j]), v[j]);
      }
    } else if (g.drop.level > 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = fmul(v[j], g.drop.scale);
    }
    store(g.y, g.ldy);
  }
}

// One launch for what a call has left to add: db, and the tiles in parts of its products.
template <typename E, bool FORWARD>
__global__ void __launch_bounds__(256) linear_finish_kernel(const Bias<E> bias, const Finish a, const Finish b) {
  pdl_begin();
  pdl_end();
  unsigned block = blockIdx.x;
  if (block < bias.blocks) {
    sum_bias<E>(block, bias);
    return;
  }
  block -= bias.blocks;
  if (block < a.blocks) finish_tiles<E, FORWARD>(block, a);
  else finish_tiles<E, FORWARD>(block - a.blocks, b);
}
template <typename E, bool FORWARD>
cudaError_t launch_finish(const Bias<E>& bias, const Finish& a, const Finish& b, cudaStream_t s) {
  const unsigned blocks = bias.blocks + a.blocks + b.blocks;
  if (blocks == 0) return cudaSuccess;
  return launch_kernel(linear_finish_kernel<E, FORWARD>, dim3(blocks), dim3(256), 0, s, 0u, bias, a, b);
}

// ---------------------------------------------------------------------------
// Workspace and launches
// ---------------------------------------------------------------------------
// Tile width and parts of K.  All pairs of SMs form whole tiles as long as there is one for each
// of them; what is left over can be cut into parts along K, which then fill the pairs once
// more, at the price of their sums, written and read, and of a launch.  Estimated in cycles:
// a K block of a tile takes its products (512 for 256 columns in bf16, six times that in
// fp32) or its copies from L2 (about 55 bytes a cycle an SM) and a little more; what is
// exposed at the ends is the first copies and the last tile's epilogue.
struct Cut {
  int tile_n, splits;
  int64_t whole;  // tiles in one piece
};
constexpr int kMostSplits = 32;

Cut best_cut(int64_t m, int64_t n, int64_t blocks, int planes) {
  Cut best = {kN, 1, 0};
  double least = 1e300;
  const int64_t mt = (m + kPair - 1) / kPair;
  for (int tn = kN; tn >= 64; tn -= 64) {
    const int64_t nt = (n + tn - 1) / tn, tiles = mt * nt, full = tiles / kPairs * kPairs, rest = tiles - full;
    const double copies = planes * (kBytesA + tn / 2 * kK * 2) / 55.0, products = (planes == 1 ? 2.0 : 12.0) * tn;
    const double step = std::max(copies, products) + 20.0, end = 3000.0 + 4000.0 * tn / kN;
    const double tile = std::max(blocks * step, 2500.0 + 3500.0 * tn / kN);  // or its epilogue
    for (int s = 1; s <= kMostSplits && s <= blocks; ++s) {
      if (s > 1 && rest == 0) break;
      double cost = tiles / kPairs * tile + end;
      if (s == 1) {
        cost += rest > 0 ? tile : 0.0;
      } else {
        const int64_t waves = (rest * s + kPairs - 1) / kPairs;
        cost += waves * (((blocks + s - 1) / s) * step + 500.0) + 6000.0 +
                static_cast<double>(rest) * s * kPair * tn * 8.0 / 3500.0;
      }
      if (cost < 0.98 * least) {
        least = cost;
        best = Cut{tn, s, s == 1 ? tiles : full};
      }
    }
  }
  return best;
}
// The estimate weighs up to 128 candidates, and a call asks for it three times (for the size of its
// workspace, to check that, and to launch): 15 us of the host for a backward call.  So each thread
// keeps the answers for the sizes it asked for last.
Cut cut_tiles(int64_t m, int64_t n, int64_t blocks, int planes) {
  struct Known {
    int64_t m, n, blocks;
    int planes;
    Cut cut;
  };
  static thread_local Known known[32] = {};
  const uint64_t key = static_cast<uint64_t>(m) * 0x9E3779B97F4A7C15ull ^ static_cast<uint64_t>(n) * 0xBF58476D1CE4E5B9ull ^
                       static_cast<uint64_t>(blocks * 4 + planes) * 0x94D049BB133111EBull;
  Known& k = known[key >> 59];
  if (k.m != m || k.n != n || k.blocks != blocks || k.planes != planes) k = Known{m, n, blocks, planes, best_cut(m, n, blocks, planes)};
  return k.cut;
}
// Bytes of the sums.
size_t cut_bytes(const Cut& c, int64_t m, int64_t n) {
  if (c.splits == 1) return 0;
  const int64_t tiles = (m + kPair - 1) / kPair * ((n + c.tile_n - 1) / c.tile_n);
  return static_cast<size_t>((tiles - c.whole) * c.splits) * kPair * c.tile_n * 4;
}

struct Layout {
  size_t x, w, dz, part, sum, dw_sum, total;
  bool pack_x, pack_w, pack_dy;  // dy: where nothing else makes a dz of it
  int64_t Kp, Np;
  Cut forward, dx, dw;
};

Layout layout(int64_t rows, int64_t in, int64_t out, bool bf16, int pass, int64_t ldx, int64_t ldw, int64_t lddy) {
  Layout l = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t p = at;
    at += up(bytes);
    return p;
  };
  const int planes = bf16 ? 1 : 3;
  l.Kp = round_up(in, 8);
  l.Np = round_up(out, 8);
  l.pack_x = !bf16 || ldx < in || ldx % 8 != 0;
  l.pack_w = !bf16 || ldw < in || ldw % 8 != 0;
  l.pack_dy = !bf16 || lddy < out || lddy % 8 != 0;
  l.x = take(l.pack_x ? static_cast<size_t>(planes) * rows * l.Kp * 2 : 0);
  l.w = take(l.pack_w ? static_cast<size_t>(planes) * out * l.Kp * 2 : 0);
  if (pass == MPC_LINEAR_FORWARD) {
    l.forward = cut_tiles(rows, out, (in + kK - 1) / kK, planes);
    l.sum = take(cut_bytes(l.forward, rows, out));
  } else {
    // plain: dz is dy itself where it is read in place
    l.dz = take(pass == MPC_LINEAR_BACKWARD_PLAIN && !l.pack_dy ? 0 : static_cast<size_t>(planes) * rows * l.Np * 2);
    l.part = take((rows + dz_rows(rows, out) - 1) / dz_rows(rows, out) * out * 4);
    l.dx = cut_tiles(rows, in, (out + kK - 1) / kK, planes);
    l.dw = cut_tiles(out, in, (rows + kK - 1) / kK, planes);
    l.sum = take(cut_bytes(l.dx, rows, in));
    l.dw_sum = take(cut_bytes(l.dw, out, in));
  }
  l.total = at;
  return l;
}

bool on16(const void* p, int64_t ld, int size) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * size % 16 == 0; }

#define LIN_TRY(...)                      \
  do {                                    \
    const cudaError_t e_ = (__VA_ARGS__); \
    if (e_ != cudaSuccess) return e_;     \
  } while (0)

// One matrix of a product: its planes and how they lie.
struct Matrix {
  const void* p;
  int64_t rows, cols, ld;
};

template <int MODE, typename E>
cudaError_t product(LinearGemm g, const Matrix& a, const Matrix& b, int64_t m, int64_t n, int64_t k, const Cut& cut,
                    float* sum, int num_sms, cudaStream_t s, Finish* finish) {
  constexpr int P = sizeof(E) == 2 ? 1 : 3, size = static_cast<int>(sizeof(E));
  const int64_t mt = (m + kPair - 1) / kPair, nt = (n + cut.tile_n - 1) / cut.tile_n;
  const int64_t rest = mt * nt - cut.whole, units = cut.whole + rest * cut.splits;
  if (units > 0x7fffffff - num_sms || rest * kPair > 0x7fffffff) return cudaErrorInvalidValue;
  g.m = static_cast<int>(m);
  g.n = static_cast<int>(n);
  g.blocks = static_cast<int>((k + kK - 1) / kK);
  g.m_tiles = static_cast<int>(mt);
  g.n_tiles = static_cast<int>(nt);
  g.whole = static_cast<int>(cut.whole);
  g.splits = cut.splits;
  g.tile_n = cut.tile_n;
  g.group = static_cast<int>(std::min<int64_t>(8, mt));
  const int64_t over = mt % g.group;
  g.band = divisor(static_cast<uint32_t>(g.group * nt));
  g.rows = divisor(static_cast<uint32_t>(g.group));
  g.last_rows = divisor(static_cast<uint32_t>(over > 0 ? over : g.group));
  g.chunk = P == 1 ? 128 : 2;
  g.sum = sum;
  auto on = [&](uintptr_t bytes) {
    auto fits = [&](const void* q, int64_t ld) {
      return q == nullptr || (reinterpret_cast<uintptr_t>(q) % bytes == 0 && ld * size % static_cast<int64_t>(bytes) == 0);
    };
    return fits(g.y, g.ldy) && fits(g.z, g.ldz) && fits(g.residual, g.ldr);
  };
  g.wide = on(32) ? 2 : on(16) ? 1 : 0;
  CUtensorMap ma, mb;
  LIN_TRY(make_map(&ma, a.p, a.cols, a.rows, P, a.ld, a.rows * a.ld, MODE == kDw ? kK : kM));
  LIN_TRY(make_map(&mb, b.p, b.cols, b.rows, P, b.ld, b.rows * b.ld, MODE == kForward ? cut.tile_n / 2 : kK));
  const bool one = P == 1 && g.blocks <= g.chunk;
  const auto kernel = one ? linear_gemm_kernel<MODE, P, P == 1> : linear_gemm_kernel<MODE, P, false>;
  constexpr int smem = LinearTiles<P>::kSmem;
  LIN_TRY(ensure_dynamic_smem(kernel, smem));
  const unsigned grid = static_cast<unsigned>(2 * std::min<int64_t>(units, num_sms / 2));
  LIN_TRY(launch_kernel(kernel, dim3(grid), dim3(kLinearThreads), smem, s, 2u, ma, mb, g));
  finish->g = g;
  finish->blocks = static_cast<unsigned>(std::min<int64_t>(rest * (kPair / 4) * cut.tile_n / 256, int64_t{num_sms} * 16));
  return cudaSuccess;
}

template <typename E>
Operand<E> operand(const void* p, int64_t ld, int64_t rows, int64_t cols, int64_t padded, uint16_t* out, int num_sms) {
  Operand<E> o = {static_cast<const E*>(p), ld, rows, cols, padded, on16(p, ld, sizeof(E)), out, 0};
  if (out != nullptr) o.blocks = static_cast<unsigned>(std::min<int64_t>((rows * (padded / 8) + 255) / 256, int64_t{num_sms} * 32));
  return o;
}

template <typename E>
cudaError_t forward(const LinearArgs& a, int num_sms, cudaStream_t s) {
  constexpr int P = sizeof(E) == 2 ? 1 : 3;
  const Layout l = layout(a.rows, a.in, a.out, P == 1, MPC_LINEAR_FORWARD, on16(a.x, 0, 1) ? a.ldx : 0, on16(a.w, 0, 1) ? a.ldw : 0, 0);
  char* ws = static_cast<char*>(a.ws);
  Prepare<E> f = {};
  if (l.pack_x) f.x = operand<E>(a.x, a.ldx, a.rows, a.in, l.Kp, reinterpret_cast<uint16_t*>(ws + l.x), num_sms);
  if (l.pack_w) f.w = operand<E>(a.w, a.ldw, a.out, a.in, l.Kp, reinterpret_cast<uint16_t*>(ws + l.w), num_sms);
  if (f.x.blocks + f.w.blocks > 0)
    LIN_TRY(launch_kernel(linear_prepare_kernel<E, P>, dim3(f.x.blocks + f.w.blocks), dim3(256), 0, s, 0u, f));
  LinearGemm g = {};
  g.bias = a.bias;
  g.bias_wide = on16(a.bias, 0, 1);
  g.residual = a.residual;
  g.ldr = a.ldr;
  g.y = a.y;
  g.ldy = a.ldy;
  g.z = a.z;
  g.ldz = a.ldz;
  g.act = a.act;
  g.drop = make_drop(a.p, a.seed, a.step);
  g.spin_limit = a.spin_limit;
  g.status = a.status;
  const Matrix x = {l.pack_x ? ws + l.x : a.x, a.rows, a.in, l.pack_x ? l.Kp : a.ldx};
  const Matrix w = {l.pack_w ? ws + l.w : a.w, a.out, a.in, l.pack_w ? l.Kp : a.ldw};
  Finish finish = {};
  LIN_TRY(product<kForward, E>(g, x, w, a.rows, a.out, a.in, l.forward, reinterpret_cast<float*>(ws + l.sum), num_sms, s, &finish));
  return launch_finish<E, true>(Bias<E>{}, finish, Finish{}, s);
}

template <typename E>
cudaError_t backward(const LinearArgs& a, int num_sms, cudaStream_t s) {
  constexpr int P = sizeof(E) == 2 ? 1 : 3;
  const Layout l = layout(a.rows, a.in, a.out, P == 1, linear_backward_pass(a), on16(a.x, 0, 1) ? a.ldx : 0,
                          on16(a.w, 0, 1) ? a.ldw : 0, on16(a.dy, 0, 1) ? a.lddy : 0);
  char* ws = static_cast<char*>(a.ws);
  float* part = reinterpret_cast<float*>(ws + l.part);
  const bool products = a.dx != nullptr || a.dw != nullptr;
  Prepare<E> f = {};
  f.drop = make_drop(a.p, a.seed, a.step);
  f.act = a.act;
  f.z = static_cast<const E*>(a.z_in);
  f.ldz = a.ldz;
  f.wide_z = on16(a.z_in, a.ldz, sizeof(E));
  const bool make = products && (l.pack_dy || linear_backward_pass(a) == MPC_LINEAR_BACKWARD);
  f.dy = operand<E>(a.dy, a.lddy, a.rows, a.out, l.Np, make ? reinterpret_cast<uint16_t*>(ws + l.dz) : nullptr, num_sms);
  f.part = a.dbias != nullptr ? part : nullptr;
  f.dz_rows = static_cast<int>(dz_rows(a.rows, a.out));
  const int64_t chunks = (a.rows + f.dz_rows - 1) / f.dz_rows, cols = (a.out + 255) / 256;
  if (chunks * cols > 0x3fffffff) return cudaErrorInvalidValue;
  f.dz_cols = static_cast<unsigned>(cols);
  f.dy.blocks = make || a.dbias != nullptr ? static_cast<unsigned>(chunks * cols) : 0;
  if (l.pack_x && a.dw != nullptr) f.x = operand<E>(a.x, a.ldx, a.rows, a.in, l.Kp, reinterpret_cast<uint16_t*>(ws + l.x), num_sms);
  if (l.pack_w && a.dx != nullptr) f.w = operand<E>(a.w, a.ldw, a.out, a.in, l.Kp, reinterpret_cast<uint16_t*>(ws + l.w), num_sms);
  const unsigned blocks = f.dy.blocks + f.x.blocks + f.w.blocks;
  if (blocks > 0) LIN_TRY(launch_kernel(linear_prepare_kernel<E, P>, dim3(blocks), dim3(256), 0, s, 0u, f));
  Bias<E> bias = {};
  if (a.dbias != nullptr)
    bias = {part, chunks, a.out, f.drop.scale, static_cast<E*>(a.dbias), static_cast<unsigned>((a.out + 31) / 32)};
  Finish dx = {}, dw = {};
  LinearGemm g = {};
  g.drop = f.drop;
  g.spin_limit = a.spin_limit;
  g.status = a.status;
  float* sum = reinterpret_cast<float*>(ws + l.sum);
  const Matrix dz = {make ? ws + l.dz : a.dy, a.rows, a.out, make ? l.Np : a.lddy};
  if (a.dx != nullptr) {
    const Matrix w = {l.pack_w ? ws + l.w : a.w, a.out, a.in, l.pack_w ? l.Kp : a.ldw};
    g.y = a.dx;
    g.ldy = a.lddx;
    LIN_TRY(product<kDx, E>(g, dz, w, a.rows, a.in, a.out, l.dx, sum, num_sms, s, &dx));
  }
  if (a.dw != nullptr) {
    const Matrix x = {l.pack_x ? ws + l.x : a.x, a.rows, a.in, l.pack_x ? l.Kp : a.ldx};
    g.y = a.dw;
    g.ldy = a.lddw;
    LIN_TRY(product<kDw, E>(g, dz, x, a.out, a.in, a.rows, l.dw, reinterpret_cast<float*>(ws + l.dw_sum), num_sms, s, &dw));
  }
  return launch_finish<E, false>(bias, dx, dw, s);
}

}  // namespace

size_t linear_workspace_bytes(int64_t rows, int64_t in, int64_t out, int bf16, int pass, int64_t ldx, int64_t ldw, int64_t lddy) {
  if (pass == MPC_LINEAR_FORWARD && linear_few_fits(rows, in, bf16, ldx, ldw)) return 0;
  return layout(rows, in, out, bf16 != 0, pass, ldx, ldw, lddy).total;
}
int linear_backward_pass(const LinearArgs& a) {
  return a.act == MPC_ACT_NONE && make_drop(a.p, 0, nullptr).level == 0 ? MPC_LINEAR_BACKWARD_PLAIN : MPC_LINEAR_BACKWARD;
}
cudaError_t launch_linear_forward(const LinearArgs& a, int num_sms, cudaStream_t s) {
  if (linear_few_fits(a.rows, a.in, a.bf16, on16(a.x, 0, 1) ? a.ldx : 0, on16(a.w, 0, 1) ? a.ldw : 0))
    return launch_linear_few(a, num_sms, s);
  return a.bf16 ? forward<__nv_bfloat16>(a, num_sms, s) : forward<float>(a, num_sms, s);
}
cudaError_t launch_linear_backward(const LinearArgs& a, int num_sms, cudaStream_t s) {
  return a.bf16 ? backward<__nv_bfloat16>(a, num_sms, s) : backward<float>(a, num_sms, s);
}

}  // namespace mpc
