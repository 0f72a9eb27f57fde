// Matrix products of the dense maps (the affine map, and the gated map whose two products share a
// kernel): C[M, N] = sum_k A(m, k) B(n, k) with an epilogue, each operand stored either with the
// contraction index fastest ("row" form) or with the output index fastest ("column" form). The bf16
// matrix cores multiply, float32 tensors as three bf16 parts; sums, bias, activation and what follows
// are float32, rounded once to the storage type.
#pragma once
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "dense.hpp"
#include "dense_common.hpp"
#include "gemm_common.hpp"

namespace bsa {
namespace {

// ---- activations ----

// Normal distribution function Phi(z) and e^(-z^2 / 2). f32 tensors take the library's erfc (f32
// accurate in the lower tail as well). bf16 tensors take Abramowitz and Stegun 7.1.26, erfc(x) =
// (a1 t + .. + a5 t^5) e^(-x^2), t = 1 / (1 + p x), x >= 0, off by at most 1.5e-7: 2^-14 of a
// bf16 step at 1. erfc's branches took longer than the products: at 65536 x 512 -> 2048 channels
// the forward with GELU ran 427 us, the dz pass 253.
template <typename T>
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  e = __expf(-0.5f * z * z);
  if constexpr (sizeof(T) == 4) return 0.5f * erfcf(-z * 0.70710678118654752f);
  const float x = fabsf(z) * 0.70710678118654752f;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.0f));
  float p = fmaf(1.061405429f, t, -1.453152027f);
  p = fmaf(p, t, 1.421413741f);
  p = fmaf(p, t, -0.284496736f);
  p = fmaf(p, t, 0.254829592f);
  const float tail = 0.5f * p * t * e;
  return z > 0.f ? 1.0f - tail : tail;
}

template <typename T>
__device__ __forceinline__ float act_fwd(float z, int act) {
  switch (act) {
    case kActRelu: return z > 0.f ? z : z != z ? z : 0.f;
    case kActGelu: {
      float e;
      return z * normal_cdf<T>(z, e);
    }
    case kActSilu: return z * sigmoid(z);
    default: return z;
  }
}
template <typename T>
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case kActRelu: return z > 0.f ? 1.f : 0.f;
    case kActGelu: {
      float e;
      const float cdf = normal_cdf<T>(z, e);
      return fmaf(z * e, 0.39894228040143268f, cdf);
    }
    case kActSilu: {
      const float s = sigmoid(z);
      return s * fmaf(z, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}

// ---- epilogue ----

template <typename T>
struct Epi {
  long long M;
  int N;
  T* out;
  long long ldo;
  const T* bias;      // [N] or NULL
  const T* res;       // [M, ldr] or NULL
  long long ldr;
  T* pre;             // [M, N] or NULL: z in the storage type
  int act;
  float* part;        // not NULL: the bare sums go to part[split][M][N] instead
};

// Four consecutive columns of a row at element alignment.
__device__ __forceinline__ void load4u(const float* p, float (&v)[4]) { __builtin_memcpy(v, p, 16); }
__device__ __forceinline__ void load4u(const bf16_t* p, float (&v)[4]) {
  uint2 u;
  __builtin_memcpy(&u, p, 8);
  v[0] = __uint_as_float(u.x << 16);
  v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16);
  v[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ void store4u(float* p, const float (&v)[4]) { __builtin_memcpy(p, v, 16); }
__device__ __forceinline__ void store4u(bf16_t* p, const float (&v)[4]) {
  const uint2 u = make_uint2((uint32_t)f2bf(v[0]) | ((uint32_t)f2bf(v[1]) << 16), (uint32_t)f2bf(v[2]) | ((uint32_t)f2bf(v[3]) << 16));
  __builtin_memcpy(p, &u, 8);
}

// Four consecutive columns n.. of row m.
template <typename T>
__device__ __forceinline__ void epi_store4(const Epi<T>& o, long long m, int n, float (&v)[4], int split) {
  if (m >= o.M || n >= o.N) return;
  if (n + 4 <= o.N) {
    if (o.part) {
      store4u(o.part + ((long long)split * o.M + m) * o.N + n, v);
      return;
    }
    float t[4];
    if (o.bias) {
      load4u(o.bias + n, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += t[e];
    }
    if (o.pre) store4u(o.pre + m * o.N + n, v);
    if (o.act != kActNone) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = act_fwd<T>(v[e], o.act);
    }
    if (o.res) {
      load4u(o.res + m * o.ldr + n, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += t[e];
    }
    store4u(o.out + m * o.ldo + n, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e) {   // the row ends inside
    if (n + e >= o.N) break;
    if (o.part) {
      o.part[((long long)split * o.M + m) * o.N + n + e] = v[e];
      continue;
    }
    float z = v[e];
    if (o.bias) z += to_f32<T>(o.bias[n + e]);
    if (o.pre) o.pre[m * o.N + n + e] = from_f32<T>(z);
    z = act_fwd<T>(z, o.act);
    if (o.res) z += to_f32<T>(o.res[m * o.ldr + n + e]);
    o.out[m * o.ldo + n + e] = from_f32<T>(z);
  }
}

// Gated: four consecutive columns of both maps, g of the first and u of the second, out = act(g) u. bias,
// pre and part hold the first map's N columns and behind them the second's.
template <typename T>
__device__ __forceinline__ void gated_store4(const Epi<T>& o, long long m, int n, float (&g)[4], float (&u)[4], int split) {
  if (m >= o.M || n >= o.N) return;
  if (n + 4 <= o.N) {
    if (o.part) {
      float* p = o.part + ((long long)split * o.M + m) * 2 * o.N + n;
      store4u(p, g);
      store4u(p + o.N, u);
      return;
    }
    if (o.bias) {
      float t[4];
      load4u(o.bias + n, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) g[e] += t[e];
      load4u(o.bias + o.N + n, t);
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] += t[e];
    }
    if (o.pre) {
      store4u(o.pre + m * 2 * o.N + n, g);
      store4u(o.pre + m * 2 * o.N + o.N + n, u);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] *= act_fwd<T>(g[e], o.act);
    store4u(o.out + m * o.ldo + n, u);
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e) {   // the row ends inside
    if (n + e >= o.N) break;
    const long long at = m * 2 * o.N + n + e;
    if (o.part) {
      float* p = o.part + (long long)split * o.M * 2 * o.N + at;
      p[0] = g[e];
      p[o.N] = u[e];
      continue;
    }
    float zg = g[e], zu = u[e];
    if (o.bias) {
      zg += to_f32<T>(o.bias[n + e]);
      zu += to_f32<T>(o.bias[o.N + n + e]);
    }
    if (o.pre) {
      o.pre[at] = from_f32<T>(zg);
      o.pre[at + o.N] = from_f32<T>(zu);
    }
    o.out[m * o.ldo + n + e] = from_f32<T>(act_fwd<T>(zg, o.act) * zu);
  }
}

// ---- products, any shape: tiles staged through registers ----

// A stored matrix (rows x cols, leading dimension ld); in column form its rows are the
// contraction index.
template <typename T>
struct Mat {
  const T* p;
  long long ld;
  long long rows;
  int cols;
};

// Gated products (G): the stored rows of B are two maps of n = rows / 2 rows, and the operand rows take 16
// of the first and 16 of the second in turn, so that a wave holds both sums of an output and joins them
// in registers. Operand row v is output column (v / 32) 16 + v % 16 (behind the last column: that one again).
__device__ __forceinline__ int gated_col(int v) { return ((v >> 5) << 4) + (v & 15); }
template <bool G, typename T>
__device__ __forceinline__ long long stored_row(const Mat<T>& m, long long v) {
  if constexpr (G) {
    const long long n = m.rows / 2;
    return min((long long)gated_col((int)v), n - 1) + (v & 16 ? n : 0);
  } else {
    return v;
  }
}

template <typename T>
__device__ __forceinline__ uint4 load_piece(const Mat<T>& m, long long r, int c) {
  constexpr int E = 16 / (int)sizeof(T);
  if (r >= m.rows || c >= m.cols) return make_uint4(0, 0, 0, 0);
  const T* p = m.p + r * m.ld + c;
  return c + E <= m.cols ? load16u(p) : load_partial(p, m.cols - c);
}

// A product's operands as bf16 tiles in LDS: bf16 tensors are copied; a float32 value enters as the
// sum of three bf16 values (P = 3 planes), x1 = bf16(x), x2 = bf16(x - x1), x3 = bf16(x - x1 - x2),
// which holds its 24 bits (of values below 2^-110: to 2^-134, half the smallest bf16 step), and a
// product as the six of nine part products that reach 2^-24 of it (x2 y3, x3 y2, x3 y3 are left out,
// 2^-24 at most in all), accumulated in float32. That is 6 bf16
// matrix instructions where the f32 ones take 16 times a bf16 one.
struct Parts {
  uint2 p[3];   // four values of each part
};
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}
// top: the largest magnitude split so far. Magnitudes of kNoSplit and above (what rounds to bf16
// infinity, and infinity) do not split: a tile that holds one is formed again (plain_tile). NaN
// splits into itself and NaN.
constexpr float kNoSplit = 3.3895314e38f;   // the largest bf16 value
__device__ __forceinline__ Parts split_parts(uint4 u, float& top) {
  float v[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
  top = fmaxf(fmaxf(top, fabsf(v[0])), fabsf(v[1]));
  top = fmaxf(fmaxf(top, fabsf(v[2])), fabsf(v[3]));
  Parts r;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    r.p[k] = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    v[0] -= __uint_as_float(r.p[k].x << 16);
    v[1] -= __uint_as_float(r.p[k].x & 0xffff0000u);
    v[2] -= __uint_as_float(r.p[k].y << 16);
    v[3] -= __uint_as_float(r.p[k].y & 0xffff0000u);
  }
  return r;
}

// A piece moved up by n elements (n < 0 or past its end: anything).
template <typename T>
__device__ __forceinline__ uint4 shift_piece(uint4 v, int n) {
  const uint64_t lo = (uint64_t)v.x | (uint64_t)v.y << 32, hi = (uint64_t)v.z | (uint64_t)v.w << 32;
  const int bits = n * 8 * (int)sizeof(T);
  const uint64_t a = bits == 0 ? lo : bits < 64 ? lo >> bits | hi << (64 - bits) : bits < 128 ? hi >> (bits - 64) : 0;
  const uint64_t b = bits < 64 ? hi >> bits : 0;
  return make_uint4((uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32));
}

// Tile of R operand rows x 32 contraction indices staged through registers, in the operand's own
// order (row form [R][32], column form [32][R]); pieces outside the matrix are zero.
template <typename T, bool TR, bool MIX, int R, bool G = false>
struct RegTile {
  static_assert(!(G && TR), "gated rows are in row form");
  static constexpr int E = 16 / (int)sizeof(T), P = sizeof(T) == 4 ? 3 : 1;
  static constexpr int COLS = TR ? R : 32, ROWS = TR ? 32 : R, CPR = COLS / E;
  static constexpr int NV = ROWS * CPR / 256, SIZE = R * 32;
  static_assert(NV * 256 == ROWS * CPR, "tile / thread split");

  const T* at[NV];   // this thread's pieces at contraction index 0; rows behind the matrix repeat its last
  int shift[NV];     // column form: a piece that ends behind the row is loaded that many elements earlier

  // o0: first operand row of the tile
  __device__ __forceinline__ void init(const Mat<T>& m, long long o0) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int i = threadIdx.x + 256 * u, row = i / CPR, c = (i % CPR) * E;
      if constexpr (TR) {
        const int col = (int)o0 + c, in = max(min(col, m.cols - E), 0);
        shift[u] = col - in;
        at[u] = m.p + row * m.ld + in;
      } else {
        shift[u] = 0;
        at[u] = m.p + (G ? stored_row<G>(m, o0 + row) : o0 + row < m.rows ? o0 + row : m.rows - 1) * m.ld + c;
      }
    }
  }
  // whole tiles: no branch lies between the loads and their use
  __device__ __forceinline__ void load(uint4 (&v)[NV], const Mat<T>& m, long long k0) const {
    const long long k = TR ? k0 * m.ld : k0;
#pragma unroll
    for (int u = 0; u < NV; ++u) v[u] = load16u(at[u] + k);
  }
  __device__ __forceinline__ void settle(uint4 (&v)[NV], const Mat<T>& m, long long o0) const {
    if constexpr (TR) {
      if (o0 + R > m.cols) {   // uniform
#pragma unroll
        for (int u = 0; u < NV; ++u) v[u] = shift_piece<T>(v[u], shift[u]);
      }
    }
  }
  // the contraction's last, partial tile (k0: its first index)
  __device__ __forceinline__ static void load_tail(uint4 (&v)[NV], const Mat<T>& m, long long o0, long long k0) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int i = threadIdx.x + 256 * u, row = i / CPR, c = (i % CPR) * E;
      v[u] = TR ? load_piece(m, k0 + row, (int)o0 + c) : load_piece(m, stored_row<G>(m, o0 + row), (int)k0 + c);
    }
  }
  __device__ __forceinline__ static void store(const uint4 (&v)[NV], bf16_t* t, float& top) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int i = threadIdx.x + 256 * u, row = i / CPR, c = (i % CPR) * E;
      bf16_t* p = t + row * COLS + 8 * ((c >> 3) ^ tile_swz<COLS, TR && MIX>(row)) + (c & 7);
      if constexpr (P == 1) {
        *reinterpret_cast<uint4*>(p) = v[u];
      } else {
        const Parts s = split_parts(v[u], top);
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<uint2*>(p + k * SIZE) = s.p[k];
      }
    }
  }
};

// The NF fragments of operand rows r0 + 16 i of a staged tile at contraction step ks; TR: the tile
// is in column form, COLS operand rows wide; MIX: the partner is in the other form.
template <bool TR, bool MIX, int BK, int COLS, int NF>
struct Frags {
  __device__ __forceinline__ static void read(const bf16_t* t, int r0, int ks, int lane, bf16x8 (&f)[NF]) {
    if constexpr (!TR) {
#pragma unroll
      for (int i = 0; i < NF; ++i) f[i] = frag_row<BK>(t, r0 + 16 * i + (lane & 15), 4 * ks + (lane >> 4));
    } else if constexpr (NF % 4 == 0) {
#pragma unroll
      for (int i = 0; i < NF; i += 4)
        tr_frags4<COLS, MIX>(t, 32 * ks, r0 + 16 * i, lane, *reinterpret_cast<bf16x8(*)[4]>(&f[i]));
    } else {
#pragma unroll
      for (int i = 0; i < NF; i += 2)
        tr_frags2<COLS, MIX>(t, 32 * ks, r0 + 16 * i, lane, *reinterpret_cast<bf16x8(*)[2]>(&f[i]));
    }
  }
};

// Accumulators of a float32 wave tile by f32 matrix instructions, straight from memory: for tiles
// with values that do not split into bf16 parts.
template <bool TA, bool TB, int FI, int FJ, bool G>
__device__ __forceinline__ void plain_tile(const Mat<float>& a, const Mat<float>& b, long long m0, long long n0, long long k0,
                                        long long k1, int lane, f32x4 (&acc)[FI][FJ]) {
  const int r = lane & 15, j = lane >> 4;
  auto at = [](const Mat<float>& m, bool tr, long long o, long long k) {
    const long long row = tr ? k : o, col = tr ? o : k;
    return row < m.rows && col < m.cols ? m.p[row * m.ld + col] : 0.f;
  };
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int jj = 0; jj < FJ; ++jj) acc[i][jj] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (long long k = k0; k < k1; k += 4) {
    float x[FI], y[FJ];
#pragma unroll
    for (int i = 0; i < FI; ++i) x[i] = k + j < k1 ? at(a, TA, m0 + 16 * i + r, k + j) : 0.f;
#pragma unroll
    for (int i = 0; i < FJ; ++i) y[i] = k + j < k1 ? at(b, TB, stored_row<G>(b, n0 + 16 * i + r), k + j) : 0.f;
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int jj = 0; jj < FJ; ++jj) acc[i][jj] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[jj], x[i], acc[i][jj], 0, 0, 0);
  }
}

// Schedule of an iteration with VALU instructions of splitting beside 6 MF matrix instructions: the
// former between the latter, so that both pipes work in one wave.
template <int P, int MF, int VALU>
__device__ __forceinline__ void interleave() {
  constexpr int N = 6 * MF, per = (VALU + N - 1) / N;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x2, per, 0);
  }
}

// 4 waves in a 2 x 2 arrangement. Tiles pass from memory through registers (two in flight) into
// one of two LDS buffers: the next tile is split and stored while the current one is multiplied,
// and an iteration has one barrier, without a fence (that of __syncthreads would wait for the
// tiles in flight). float32 at 4096^3: 770 us, 178 TFLOP/s (f32 matrix instructions reach 151);
// the matrix cores are busy 45% of the time, the VALU (splitting) 42%.
// Accumulator lane L holds C[m + L % 16][n + 4 (L / 16) + e] (B's fragment comes first).
template <typename T, bool TA, bool TB, int BM, int BN, bool G>
__global__ void __launch_bounds__(256, (BM * BN <= 8192 ? 2 : 1)) product_kernel(Mat<T> a, Mat<T> b, long long K, int ntn, long long kt_per, Epi<T> o) {
  constexpr int BK = 32, FI = BM / 32, FJ = BN / 32;
  typedef RegTile<T, TA, TA != TB, BM> LA;
  typedef RegTile<T, TB, TA != TB, BN, G> LB;
  constexpr int P = LA::P;
  __shared__ __attribute__((aligned(1024))) bf16_t as[2][P * LA::SIZE], bs[2][P * LB::SIZE];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, wm = wid >> 1, wn = wid & 1;
  const int tm = blockIdx.x / ntn, tn = blockIdx.x - tm * ntn;
  const long long m0 = (long long)tm * BM;
  const int n0 = tn * BN;
  const long long nkt = (K + BK - 1) / BK;
  // whole tiles; none where a column-form operand is narrower than a piece
  const long long nwhole = (TA && a.cols < LA::E) || (TB && b.cols < LB::E) ? 0 : K / BK;
  const long long kt0 = min(blockIdx.y * kt_per, nkt), kt1 = min(kt0 + kt_per, nkt), kw = min(kt1, nwhole);
  f32x4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  LA la;
  LB lb;
  la.init(a, m0);
  lb.init(b, n0);
  float top = 0.f;
  uint4 av[2][LA::NV], bv[2][LB::NV];
  auto load = [&](int d, long long kt) {
    la.load(av[d], a, kt * BK);
    lb.load(bv[d], b, kt * BK);
  };
  auto store = [&](int d, int buf) {
    la.settle(av[d], a, m0);
    lb.settle(bv[d], b, n0);
    LA::store(av[d], as[buf], top);
    LB::store(bv[d], bs[buf], top);
  };
  bf16x8 af[P][FI], bf[P][FJ];
  auto frags = [&](int buf) {
#pragma unroll
    for (int k = 0; k < P; ++k) {
      Frags<TA, TA != TB, BK, BM, FI>::read(as[buf] + k * LA::SIZE, wm * (BM / 2), 0, lane, af[k]);
      Frags<TB, TA != TB, BK, BN, FJ>::read(bs[buf] + k * LB::SIZE, wn * (BN / 2), 0, lane, bf[k]);
    }
  };
  auto multiply_parts = [&](int ka, int kb) {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) acc[i][j] = mma(bf[kb][j], af[ka][i], acc[i][j]);
  };
  auto multiply = [&]() {
    if constexpr (P == 3) {   // the small part products first
      multiply_parts(2, 0);
      multiply_parts(0, 2);
      multiply_parts(1, 1);
      multiply_parts(1, 0);
      multiply_parts(0, 1);
    }
    multiply_parts(0, 0);
  };
  if (kt0 < kw) {
    load(0, kt0);
    load(1, min(kt0 + 1, kw - 1));
    store(0, 0);
    load(0, min(kt0 + 2, kw - 1));
  }
  // loads past the last whole tile repeat it (never used), so that no branch surrounds them
  auto iterate = [&](long long kt, int d) {
    // tile kt lies in buffer d, kt + 1 in register set 1 - d, kt + 2 in set d
    lgkm_drain();
    lds_barrier();   // tile kt is visible; every wave has its fragments of kt - 1
    frags(d);
    store(1 - d, 1 - d);
    load(1 - d, min(kt + 3, kw - 1));
    multiply();
    if constexpr (P == 3) interleave<P, FI * FJ, (LA::NV + LB::NV) * 30>();
  };
  long long t = kt0;
  for (; t + 1 < kw; t += 2) {
    iterate(t, 0);
    iterate(t + 1, 1);
  }
  if (t < kw) iterate(t, 0);
  for (long long kt = max(kt0, kw); kt < kt1; ++kt) {
    LA::load_tail(av[0], a, m0, kt * BK);
    LB::load_tail(bv[0], b, n0, kt * BK);
    __syncthreads();
    LA::store(av[0], as[0], top);
    LB::store(bv[0], bs[0], top);
    __syncthreads();
    frags(0);
    multiply();
  }
  if constexpr (P == 3) {
    __shared__ int again;
    if (threadIdx.x == 0) again = 0;
    __syncthreads();
    if (top >= kNoSplit) again = 1;
    __syncthreads();
    if (again)
      plain_tile<TA, TB, FI, FJ, G>(a, b, m0 + wm * (BM / 2), n0 + wn * (BN / 2), kt0 * BK, min(kt1 * BK, K), lane, acc);
  }
#pragma unroll
  for (int i = 0; i < FI; ++i) {
    const long long m = m0 + wm * (BM / 2) + 16 * i + (lane & 15);
#pragma unroll
    for (int j = 0; j < FJ; j += G ? 2 : 1) {
      const int n = n0 + wn * (BN / 2) + 16 * j + 4 * (lane >> 4);
      float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
      if constexpr (G) {
        float u[4] = {acc[i][j + 1][0], acc[i][j + 1][1], acc[i][j + 1][2], acc[i][j + 1][3]};
        gated_store4(o, m, gated_col(n), v, u, blockIdx.y);
      } else {
        epi_store4(o, m, n, v, blockIdx.y);
      }
    }
  }
}

// ---- bf16 products of aligned operands: tiles loaded straight into LDS ----

// Loads of a ROWS x COLS tile of a stored matrix (row form: operand rows x contraction; column
// form: contraction x operand rows) by NW waves: a wave instruction fills 1 KB of consecutive
// LDS, and each lane fetches the 16-byte piece that the swizzle puts there. Operand rows behind
// the matrix repeat its last ones (their products are not stored); the contraction's last,
// partial tile is staged through registers (tail), zeros behind its end.
// G: a wave instruction's 8 or 16 rows are of one map; the second lies `up` bytes behind the first.
template <bool TR, bool MIX, int ROWS, int COLS, int NW, bool G = false>
struct DmaTile {
  static_assert(!(G && TR), "gated rows are in row form");
  static constexpr int CPR = COLS / 8, NU = ROWS * CPR / (64 * NW);
  static_assert(NU * 64 * NW == ROWS * CPR, "tile / wave split");
  const char* base;       // the operand block's first element (uniform)
  uint32_t off[NU];       // bytes from there at contraction index 0 (the launcher bounds ld)
  long long up;

  __device__ __forceinline__ void init(const Mat<bf16_t>& m, long long o0, int wid, int lane) {
    if constexpr (G) {
      const long long n = m.rows / 2, c0 = o0 / 2;      // o0: a multiple of 32
      base = reinterpret_cast<const char*>(m.p + c0 * m.ld);
      up = 2 * n * m.ld;
      const int last = (int)(n - 1 - c0 < (1 << 20) ? n - 1 - c0 : 1 << 20);
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const int i = (wid * NU + u) * 64 + lane, row = i / CPR;
        const int c = 8 * ((i % CPR) ^ tile_swz<COLS, false>(row));
        off[u] = 2u * ((uint32_t)min(gated_col(row), last) * (uint32_t)m.ld + c);
      }
      return;
    }
    base = reinterpret_cast<const char*>(m.p + (TR ? o0 : o0 * m.ld));
    const int last = (int)((TR ? m.cols - 8 : m.rows - 1) - o0 < (1 << 20) ? (TR ? m.cols - 8 : m.rows - 1) - o0 : 1 << 20);
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int i = (wid * NU + u) * 64 + lane, row = i / CPR;
      const int c = 8 * ((i % CPR) ^ tile_swz<COLS, TR && MIX>(row));
      off[u] = 2u * (TR ? (uint32_t)row * (uint32_t)m.ld + min(c, last) : (uint32_t)min(row, last) * (uint32_t)m.ld + c);
    }
  }
  // more: bytes to a matrix of the same shape behind this one
  __device__ __forceinline__ void issue(bf16_t* lds, const Mat<bf16_t>& m, long long k0, int wid, long long more = 0) const {
    const char* p = base + 2 * (TR ? k0 * m.ld : k0) + more;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const bool second = G && ((wid * NU + u) * (64 / CPR) & 16);
      load_lds16(p + (second ? up : 0) + off[u], lds + (wid * NU + u) * 512);
    }
  }
  __device__ __forceinline__ void tail(bf16_t* lds, const Mat<bf16_t>& m, long long o0, long long k0, int wid,
                                       int lane) const {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int i = (wid * NU + u) * 64 + lane, row = i / CPR;
      const int c = 8 * ((i % CPR) ^ tile_swz<COLS, TR && MIX>(row));
      *reinterpret_cast<uint4*>(lds + 8 * i) = TR ? load_piece(m, k0 + row, (int)o0 + c) : load_piece(m, stored_row<G>(m, o0 + row), (int)k0 + c);
    }
  }
};

// Eight consecutive columns of a row: whole 16-byte pieces unless the row ends inside.
__device__ __forceinline__ void epi_store8(const Epi<bf16_t>& o, long long m, int n, float (&v)[8], int split) {
  if (n + 8 > o.N || o.part) {
    float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
    epi_store4(o, m, n, a, split);
    epi_store4(o, m, n + 4, b, split);
    return;
  }
  if (m >= o.M) return;
  if (o.bias) {
    float b[8];
    unpack16<bf16_t>(load16u(o.bias + n), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[e];
  }
  if (o.pre) store16u(o.pre + m * o.N + n, pack16<bf16_t>(v));
  if (o.act != kActNone) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = act_fwd<bf16_t>(v[e], o.act);
  }
  if (o.res) {
    float r[8];
    unpack16<bf16_t>(load16u(o.res + m * o.ldr + n), r);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += r[e];
  }
  store16u(o.out + m * o.ldo + n, pack16<bf16_t>(v));
}

// A store past the caches' retention, of 16 bytes at element alignment.
__device__ __forceinline__ void store16_stream(bf16_t* p, uint4 v) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(2)));
  __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p));
}

__device__ __forceinline__ void store16_past(bf16_t* p, uint4 v, bool stream) {
  if (stream)
    store16_stream(p, v);
  else
    store16u(p, v);
}

// Eight consecutive columns of both maps of a gated product. The outputs are larger than the operands and do not
// push them out of the caches: 65536 x 512 -> 2 x 2048 with [g | u] kept 461 us, so 428; 8192 x 4096 -> 2 x 8192 965 and 897.
// Where rows do not end with a line of 64 bytes the caches have to join the pieces: 47687 x 88 -> 2 x 3208 742 us past
// them, through them 339; -> 2 x 3201 866 and 358; 4015 x 136 -> 2 x 6683 173 and 65.
__device__ __forceinline__ void gated_store8(const Epi<bf16_t>& o, long long m, int n, float (&g)[8], float (&u)[8], int split) {
  if (n + 8 > o.N || o.part) {
    float g0[4] = {g[0], g[1], g[2], g[3]}, g1[4] = {g[4], g[5], g[6], g[7]};
    float u0[4] = {u[0], u[1], u[2], u[3]}, u1[4] = {u[4], u[5], u[6], u[7]};
    gated_store4(o, m, n, g0, u0, split);
    gated_store4(o, m, n + 4, g1, u1, split);
    return;
  }
  if (m >= o.M) return;
  if (o.bias) {
    float t[8];
    unpack16<bf16_t>(load16u(o.bias + n), t);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] += t[e];
    unpack16<bf16_t>(load16u(o.bias + o.N + n), t);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] += t[e];
  }
  const bool lines = !((o.N | o.ldo) & 31);
  if (o.pre) {
    store16_past(o.pre + m * 2 * o.N + n, pack16<bf16_t>(g), lines);
    store16_past(o.pre + m * 2 * o.N + o.N + n, pack16<bf16_t>(u), lines);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] *= act_fwd<bf16_t>(g[e], o.act);
  store16_past(o.out + m * o.ldo + n, pack16<bf16_t>(u), lines);
}

// Workgroup tile BM x BN of WM x WN waves, contraction tiles of BK in a ring of NS LDS stages,
// NS - 1 of them in flight while one feeds the matrix cores.
template <bool TA, bool TB, int BM, int BN, int WM, int WN, int BK, int NS, bool G>
__global__ void __launch_bounds__(64 * WM * WN) product_dma_kernel(Mat<bf16_t> a, Mat<bf16_t> b, long long K, int ntm,
                                                                   int ntn, int kt_per, Epi<bf16_t> o) {
  constexpr int NW = WM * WN, TMW = BM / WM, TNW = BN / WN, FI = TMW / 16, FJ = TNW / 16;
  static_assert(NS >= 2 && NS <= 4 && (BK == 32 || BK == 64), "pipeline");
  constexpr int AE = BM * BK, BE = BN * BK;
  __shared__ __attribute__((aligned(1024))) bf16_t as0[AE], bs0[BE], as1[AE], bs1[BE];
  __shared__ __attribute__((aligned(1024))) bf16_t as2[NS > 2 ? AE : 8], bs2[NS > 2 ? BE : 8];
  __shared__ __attribute__((aligned(1024))) bf16_t as3[NS > 3 ? AE : 8], bs3[NS > 3 ? BE : 8];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int wm = wid / WN, wn = wid % WN;
  // workgroups are dealt to the 8 XCDs round-robin; each XCD gets a contiguous run of tiles, in
  // bands of 8 tile rows walked column by column, so the tiles it holds at a time share operands
  const int nt = ntm * ntn;
  int id = blockIdx.x;
  if ((nt & 7) == 0) id = (id & 7) * (nt >> 3) + (id >> 3);
  const int band = id / (8 * ntn), in = id - band * 8 * ntn, bh = min(8, ntm - 8 * band);
  const int tm = 8 * band + in % bh, tn = in / bh;
  const long long m0 = (long long)tm * BM, n0 = (long long)tn * BN;
  const int nkt = (int)(K / BK);     // whole tiles
  const int kt0 = min((int)blockIdx.y * kt_per, nkt), kt1 = min(kt0 + kt_per, nkt);
  const bool tail = (blockIdx.y == gridDim.y - 1) && K > (long long)nkt * BK;

  DmaTile<TA, TA != TB, TA ? BK : BM, TA ? BM : BK, NW> la;
  DmaTile<TB, TA != TB, TB ? BK : BN, TB ? BN : BK, NW, G> lb;
  la.init(a, m0, wid, lane);
  lb.init(b, n0, wid, lane);
  constexpr int PER = decltype(la)::NU + decltype(lb)::NU;   // wave load instructions per tile
  bf16_t* const AS[4] = {as0, as1, as2, as3};
  bf16_t* const BS[4] = {bs0, bs1, bs2, bs3};
  auto issue = [&](int kt, int st) {
    la.issue(AS[st], a, (long long)kt * BK, wid);
    lb.issue(BS[st], b, (long long)kt * BK, wid);
  };
  f32x4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  bf16x8 af[FI], bfr[FJ];
  auto read = [&](const bf16_t* as, const bf16_t* bs, int ks) {
    Frags<TA, TA != TB, BK, BM, FI>::read(as, wm * TMW, ks, lane, af);
    Frags<TB, TA != TB, BK, BN, FJ>::read(bs, wn * TNW, ks, lane, bfr);
  };
  auto multiply = [&]() {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) acc[i][j] = mma(bfr[j], af[i], acc[i][j]);
  };

#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (kt0 + s < kt1) issue(kt0 + s, s);
  if constexpr (NW == 8 && NS == 4) {
    // One workgroup to a CU: two waves share a SIMD; the second four waves run one phase behind the first four, so one
    // wave of each SIMD multiplies while the other reads its fragments. Phases end with a
    // barrier; group 0 reads tile t in phase 2t and multiplies in 2t + 1, group 1 one phase
    // later. Stage (t - 1) % NS is last read in phase 2t - 1, so tile t + NS - 1 may be loaded
    // into it from phase 2t on; tile t + 1 is first read in phase 2t + 2, so every wave waits for
    // its part of it before the barrier that ends phase 2t + 1.
    static_assert(BK == 32 && NS == 4, "one fragment depth per phase");
    const int n = kt1 - kt0, grp = wid >> 2;
    auto landed = [&](int t) {   // tile t + 1, with at most tiles t + 2 and t + 3 in flight
      if (t + 3 < n)
        vm_wait<2 * PER>();
      else if (t + 2 < n)
        vm_wait<PER>();
      else
        vm_drain();
    };
    landed(-1);
    lds_barrier();
    if (grp == 1) lds_barrier();
    for (int t0 = 0; t0 < n; t0 += NS) {
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int t = t0 + s;
        if (t < n) {
          if (t + NS - 1 < n) issue(kt0 + t + NS - 1, (s + NS - 1) % NS);
          read(AS[s], BS[s], 0);
          lgkm_drain();
          if (grp == 1) landed(t);
          lds_barrier();
          __builtin_amdgcn_s_setprio(1);
          multiply();
          __builtin_amdgcn_s_setprio(0);
          if (grp == 0) landed(t);
          lds_barrier();
        }
      }
    }
    if (grp == 0) lds_barrier();
  } else {
    for (int kt = kt0; kt < kt1; kt += NS) {
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int t = kt + s;
        if (t < kt1) {
          // tile t has landed once at most the NS - 2 tiles issued after it are in flight
          if (t + NS - 2 < kt1)
            vm_wait<(NS - 2) * PER>();
          else
            vm_drain();
          lds_barrier();     // every wave's loads of tile t are visible; stage s - 1 is free
          if (t + NS - 1 < kt1) issue(t + NS - 1, (s + NS - 1) % NS);
#pragma unroll
          for (int ks = 0; ks < BK / 32; ++ks) {
            read(AS[s], BS[s], ks);
            multiply();
          }
        }
      }
    }
  }
  if (tail) {
    __syncthreads();
    la.tail(as0, a, m0, (long long)nkt * BK, wid, lane);
    lb.tail(bs0, b, n0, (long long)nkt * BK, wid, lane);
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < BK / 32; ++ks) {
      read(as0, bs0, ks);
      multiply();
    }
  }

  // Epilogue through LDS (the stages are free by then), RP rows of the wave's tile at a time in
  // f32, so that stores are runs of whole lines; 16-byte chunk c of row x sits at c ^ (x mod 16).
  constexpr int AB = 2 * (AE < BE ? AE : BE);
  constexpr int RP = epi_rows(AB, TMW, TNW, NW);
  constexpr int WPA = AB / (RP * TNW * 4);                             // waves per stage array
  static_assert(WPA >= 1 && 4 * WPA >= NW && RP % 16 == 0, "epilogue regions");
  constexpr int SM = TNW >= 64 ? 15 : 7;
  lds_barrier();   // every wave has read the last tile
  bf16_t* const arr = wid / WPA == 0 ? as0 : wid / WPA == 1 ? bs0 : wid / WPA == 2 ? as1 : bs1;
  float* const reg = reinterpret_cast<float*>(arr) + (wid % WPA) * RP * TNW;
  auto at = [&](int row, int chunk) { return reinterpret_cast<f32x4*>(reg + row * TNW + 4 * (chunk ^ (row & SM))); };
  constexpr int LPR = TNW / (G ? 16 : 8), RPI = 64 / LPR;   // lanes to a row's outputs, eight each
#pragma unroll
  for (int i0 = 0; i0 < FI; i0 += RP / 16) {
#pragma unroll
    for (int i = 0; i < RP / 16; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) *at(16 * i + (lane & 15), 4 * j + (lane >> 4)) = acc[i0 + i][j];
    wave_sync();
    const long long mw = m0 + wm * TMW + 16 * i0;
    const int c = 8 * (lane % LPR), n = (int)n0 + wn * TNW + c;
#pragma unroll 2
    for (int x0 = 0; x0 < RP; x0 += RPI) {
      const int x = x0 + lane / LPR;
      if constexpr (G) {
        static_assert(RPI <= RP, "rows of a step");
        const int h = 8 * (c >> 4) + 2 * ((c >> 3) & 1);   // chunks h, h + 1 and, of the second map, h + 4, h + 5
        const f32x4 a0 = *at(x, h), a1 = *at(x, h + 1), b0 = *at(x, h + 4), b1 = *at(x, h + 5);
        float g[8] = {a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
        float v[8] = {b0[0], b0[1], b0[2], b0[3], b1[0], b1[1], b1[2], b1[3]};
        gated_store8(o, mw + x, ((int)n0 + wn * TNW) / 2 + c, g, v, blockIdx.y);
        continue;
      }
      const f32x4 u = *at(x, c / 4), w = *at(x, c / 4 + 1);
      float v[8] = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
      epi_store8(o, mw + x, n, v, blockIdx.y);
    }
    wave_sync();
  }
}

// ---- few rows: the weight is streamed once ----

// y of up to 16 MB rows of x: a workgroup owns 16 output columns (rows of w) and its NW waves split
// the contraction, 128 indices at a time in turn. Weights go from memory into the matrix
// instructions' operand (the weight's 16 rows first, x's rows the columns), no LDS on the way;
// x comes from the caches. The waves' sums meet in LDS, added in order. Bound by the weight's
// bytes: 4 rows, 4096 -> 8192 channels (67 MB) take 14.6 us, 4.6 TB/s; with the tiles above 24.
// Gated: the workgroup's 16 columns of both maps (NM = 2).
// WORDS: bf16 rows of an odd length (load16_words; 3 rows, 4263 -> 2 x 4371: 30 us, 48 without; 6 rows, 5355 -> 2 x 2311: 20
// and 37).
template <typename T, int MB, int NW, int NM, bool WORDS>
__global__ void __launch_bounds__(64 * NW) few_rows_kernel(Mat<T> x, Mat<T> w, int K, Epi<T> o) {
  typedef typename Chunk<T>::type CT;
  __shared__ __attribute__((aligned(16))) float part[NW][NM][MB][256];
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6, r = lane & 15, j = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const int ncol = (int)w.rows / NM;
  const T* wp[NM];
#pragma unroll
  for (int h = 0; h < NM; ++h) wp[h] = w.p + ((long long)h * ncol + min(n0 + r, ncol - 1)) * w.ld + 8 * j;
  const T* xp[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) xp[b] = x.p + min((long long)(16 * b + r), x.rows - 1) * x.ld + 8 * j;
  f32x4 acc[NM][MB];
#pragma unroll
  for (int h = 0; h < NM; ++h)
#pragma unroll
    for (int b = 0; b < MB; ++b) acc[h][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int whole = K / 128;
#pragma unroll 2
  for (int g = wid; g < whole; g += NW) {
    CT wf[NM][4], xf[MB][4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
#pragma unroll
      for (int h = 0; h < NM; ++h) {
        if constexpr (WORDS)
          wf[h][c] = __builtin_bit_cast(CT, load16_words(wp[h] + 128 * g + 32 * c));
        else
          wf[h][c] = load_chunk_u(wp[h] + 128 * g + 32 * c);
      }
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        if constexpr (WORDS)
          xf[b][c] = __builtin_bit_cast(CT, load16_words(xp[b] + 128 * g + 32 * c));
        else
          xf[b][c] = load_chunk_u(xp[b] + 128 * g + 32 * c);
      }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int b = 0; b < MB; ++b)
#pragma unroll
        for (int h = 0; h < NM; ++h) acc[h][b] = mma(wf[h][c], xf[b][c], acc[h][b]);
  }
  if (wid == whole % NW) {   // the rest of the contraction
    for (int k = 128 * whole; k < K; k += 32) {
      CT wf[NM];
#pragma unroll
      for (int h = 0; h < NM; ++h) wf[h] = load_chunk_to(wp[h] + k, K - k - 8 * j);
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        const CT xf = load_chunk_to(xp[b] + k, K - k - 8 * j);
#pragma unroll
        for (int h = 0; h < NM; ++h) acc[h][b] = mma(wf[h], xf, acc[h][b]);
      }
    }
  }
#pragma unroll
  for (int h = 0; h < NM; ++h)
#pragma unroll
    for (int b = 0; b < MB; ++b) *reinterpret_cast<f32x4*>(&part[wid][h][b][4 * lane]) = acc[h][b];
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * MB; i += 64 * NW) {
    const int b = i / 64, l = i % 64;
    float v[NM][4];
#pragma unroll
    for (int h = 0; h < NM; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[h][e] = part[0][h][b][4 * l + e];
#pragma unroll
        for (int q = 1; q < NW; ++q) v[h][e] += part[q][h][b][4 * l + e];
      }
    if constexpr (NM == 2)
      gated_store4(o, 16 * b + (l & 15), n0 + 4 * (l >> 4), v[0], v[1], 0);
    else
      epi_store4(o, 16 * b + (l & 15), n0 + 4 * (l >> 4), v[0], 0);
  }
}

// y = epilogue(sum over the splits, in order), four columns per thread (gated, NM = 2: of both maps)
template <typename T, int NM>
__global__ void __launch_bounds__(256) split_sum_kernel(const float* __restrict__ part, int S, Epi<T> o) {
  const int nq = (o.N + 3) / 4;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= o.M * nq) return;
  const long long m = i / nq;
  const int n = (int)(i - m * nq) * 4;
  float v[NM][4];
#pragma unroll
  for (int h = 0; h < NM; ++h) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[h][e] = 0.f;
#pragma unroll 4
    for (int s = 0; s < S; ++s) {
      const float* p = part + ((long long)s * o.M + m) * NM * o.N + h * o.N + n;
      float t[4] = {0.f, 0.f, 0.f, 0.f};
      if (n + 4 <= o.N) {
        load4u(p, t);
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (n + e < o.N) t[e] = p[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) v[h][e] += t[e];
    }
  }
  if constexpr (NM == 2)
    gated_store4(o, m, n, v[0], v[1], 0);
  else
    epi_store4(o, m, n, v[0], 0);
}

// ---- sums of partial column sums ----

// out = sum over P rows of part [P][n], in the storage type: wave w takes rows w, w + 16, ...
template <typename T>
__global__ void __launch_bounds__(1024) db_sum_kernel(const float* __restrict__ part, int P, int n, T* __restrict__ out) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < n) {
#pragma unroll 8
    for (int i = w; i < P; i += 16) s += part[(long long)i * n + c];
  }
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < n) {
#pragma unroll
    for (int k = 1; k < 16; ++k) s += red[k][lane];
    out[c] = from_f32<T>(s);
  }
}

// ---- host ----

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// How a product runs: tile side (workgroup tile T x T) and splits of the contraction.
struct Plan {
  int T, S;
};

// The contraction is split, in powers of two, while the tiles leave CUs idle: each split writes and reads
// its sums once more and takes a second launch, which 256 indices (512 of the larger tiles) pay for.
//
// bf16, us with the one and the other tile:
// - 256 x 256 (8 waves, one workgroup per CU) where there are 192 of them (3586 x 4096 x 4096, 240 tiles: 107, 128 x 128
//   115; contraction 512: 23.7 and 23.6), or where the splits of a long contraction fill the CUs in one round (65536 rows,
//   dW of 1024 x 1024: 137 and 236, 2048 x 2048: 483 and 836, with 8192 rows: 81 and 91, forward 81 and 76), or in two
//   where 128 x 128 tiles, two to a CU, take two as well (dW of 2560 x 3584: 65536 rows 1631 and 1977, 24576 rows 622
//   and 716, 16384 rows 430 and 391). Else they lose: 2048 x 2048 x 2048 43 and 24, 2560 columns (80 tiles) 62 and 31.
// - 128 x 128 where there are 256 of them (2048 x 1024 x 2048: 14.9, 64 x 64 16.8), or where a contraction of 4096 and
//   more is split over them (1280 x 4096 x 1792: 38 and 49; 2048, no split of 64 x 64: 1024 x 2048 x 1024: 18.6 and 12.2).
// float32: 128 x 128 where there are 512 of them (2560 x 2048 -> 3584, 560 tiles: 286 and 286; 2304 x 3200, 450
// tiles: 213, 128 x 64 193), else 64 rows fewer or both (product()): also for contractions up to 1024, where more
// workgroups to a CU write while others multiply (128 x 128 and 128 x 64; 65536 x 256 -> 512: 173 and 131, 65536 x 1024 ->
// 1024: 897 and 886, 8192 x 1024 -> 2048: 221 and 208, dW of 4096 x 2048 with 512 rows 88 and 79, of 8192 x 4096 with 32
// rows 76 and 59; 4096 x 2048 -> 4096: 402 and 422).
Plan plan_product(bool bf16, long long M, int N, long long K) {
  auto tiles = [&](int T) { return ((M + T - 1) / T) * ((N + T - 1) / T); };
  auto plan = [&](int T, int want) {
    Plan p{T, 1};
    while (tiles(T) * p.S < want && K / (2 * p.S) >= (T == 64 ? 256 : 512) && p.S < 64) p.S *= 2;
    return p;
  };
  // 128 x 64 tiles of a very long and narrow product would be more workgroups than a launch holds
  const bool narrow = (M + 127) / 128 * ((N + 63) / 64) >= 1 << 24;
  if (!bf16) return plan((tiles(128) >= 512 && K > 1024) || narrow ? 128 : 64, 512);
  if (tiles(256) >= 192) return Plan{256, 1};
  if (K >= 16384 && tiles(256) >= 12) {
    const Plan p = plan(256, 192);
    if (tiles(256) * p.S <= 256 || (K >= 24576 && tiles(128) > 512)) return p;
  }
  if (tiles(128) >= 256 || (K >= 4096 && tiles(128) * (K / 512) >= 256)) return plan(128, 256);
  return plan(64, 256);
}

size_t plan_bytes(const Plan& p, long long M, long long N) { return p.S > 1 ? sizeof(float) * (size_t)p.S * M * N : 0; }

// Whether the forward streams the weight through few_rows_kernel: up to 16 rows, and up to 64 where the
// contraction is too short to pay for a split product's second launch. (bf16, 64 rows, 1024 -> 1024
// channels: 9.2 us, split 13.0; 4096 -> 4096: 21.3 us, split 15.6, as every 16 columns read all of x.)
bool few_rows_ok(long long m, int k) { return m <= 16 || (m <= 64 && k <= 1024); }

template <typename T, int NW, int NM, bool WORDS>
void few_rows_nw(int MB, dim3 grid, const Mat<T>& x, const Mat<T>& w, int K, const Epi<T>& o, hipStream_t st) {
  if (MB == 1)
    few_rows_kernel<T, 1, NW, NM, WORDS><<<grid, 64 * NW, 0, st>>>(x, w, K, o);
  else if (MB == 2)
    few_rows_kernel<T, 2, NW, NM, WORDS><<<grid, 64 * NW, 0, st>>>(x, w, K, o);
  else
    few_rows_kernel<T, 4, NW, NM, WORDS><<<grid, 64 * NW, 0, st>>>(x, w, K, o);
}

template <typename T, int NM, bool WORDS>
void few_rows_run(const Mat<T>& x, const Mat<T>& w, long long M, int N, int K, const Epi<T>& o, hipStream_t st) {
  const int MB = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  const dim3 grid((N + 15) / 16);
  // waves per workgroup: about two per SIMD of the chip, at most one per 128 indices
  const long long wg = grid.x;
  if (wg >= 512 || K <= 512)
    few_rows_nw<T, 4, NM, WORDS>(MB, grid, x, w, K, o, st);
  else if (wg >= 256 || K <= 1024)
    few_rows_nw<T, 8, NM, WORDS>(MB, grid, x, w, K, o, st);
  else    // longer contractions come with up to 16 rows (few_rows_ok)
    few_rows_kernel<T, 1, 16, NM, WORDS><<<grid, 64 * 16, 0, st>>>(x, w, K, o);
}

// The forward of a map of N columns by few_rows_kernel (few_rows_ok).
template <typename T, int NM>
hipError_t few_rows(const Mat<T>& x, const Mat<T>& w, long long M, int N, int K, const Epi<T>& o, hipStream_t st) {
  if constexpr (sizeof(T) == 2) {
    if (w.ld % 2 && !(((uintptr_t)w.p | (uintptr_t)x.p) & 2)) {
      few_rows_run<T, NM, true>(x, w, M, N, K, o, st);
      return hipGetLastError();
    }
  }
  few_rows_run<T, NM, false>(x, w, M, N, K, o, st);
  return hipGetLastError();
}

bool dma_ok(const Mat<bf16_t>& m, bool tr) {
  const bool whole = !tr || (m.cols % 8 == 0 && m.cols >= 8);    // a row's last piece is loaded as a part of one
  // a tile's byte offsets fit 32 bits: 256 rows of at most 2^22 elements
  return whole && m.ld % 8 == 0 && m.ld <= (1 << 22) && ((uintptr_t)m.p & 15) == 0;
}
bool dma_ok(const Mat<float>&, bool) { return false; }

// C = A B^T with the epilogue; S > 1: partial sums in part, joined by split_sum_kernel. G: a gated product,
// N outputs from 2 N stored rows of B.
template <typename T, bool TA, bool TB, bool G = false>
hipError_t product(const Mat<T>& a, const Mat<T>& b, long long M, int N, long long K, Plan p, float* part, Epi<T> o,
                   hipStream_t st) {
  o.part = p.S > 1 ? part : nullptr;
  const bool dma = dma_ok(a, TA) && dma_ok(b, TB);
  const int side = !dma && p.T == 256 ? 128 : p.T;
  const int cols = G ? side / 2 : side;    // outputs of a tile's row
  const int ntm = (int)((M + side - 1) / side), ntn = (N + cols - 1) / cols;
  const dim3 grid((unsigned)((long long)ntm * ntn), (unsigned)p.S);
  if constexpr (sizeof(T) == 2 && G) {
    // A gated tile's epilogue is long: over short contractions 256 x 128 tiles, two to a CU, let one write while the other
    // multiplies (65536 x 512 -> 2 x 2048: 338 us, 256 x 256 350; 65536 x 256 -> 2 x 512: 57 and 65; 16384 x 1024 -> 2 x 1024: 77 and 71).
    const int nn = (N + 63) / 64;
    if (dma && side == 256 && K <= 512 && p.S == 1 && (long long)ntm * nn < 1 << 23) {
      product_dma_kernel<TA, TB, 256, 128, 4, 2, 32, 3, G><<<(unsigned)((long long)ntm * nn), 512, 0, st>>>(a, b, K, ntm, nn, (int)(K / 32), o);
      return hipGetLastError();
    }
  }
  if constexpr (sizeof(T) == 2) {
    if (dma) {
      const int bk = side == 256 ? 32 : 64;
      const int per = (int)((K / bk + p.S - 1) / p.S);
      if (side == 256)
        product_dma_kernel<TA, TB, 256, 256, 4, 2, 32, 4, G><<<grid, 512, 0, st>>>(a, b, K, ntm, ntn, per, o);
      else if (side == 128)
        product_dma_kernel<TA, TB, 128, 128, 2, 2, 64, 2, G><<<grid, 256, 0, st>>>(a, b, K, ntm, ntn, per, o);
      else
        product_dma_kernel<TA, TB, 64, 64, 2, 2, 64, 4, G><<<grid, 256, 0, st>>>(a, b, K, ntm, ntn, per, o);
    }
  }
  if (!dma) {
    const long long per = ((K + 31) / 32 + p.S - 1) / p.S;
    // float32: 64 x 64 tiles lie three to a CU. While they do so in one round they are faster than 128 x 64 (2816 x 512
    // -> 1024, 704 tiles: 28.0 us and 30.3; 1536 x 2048 -> 2048, 768: 90 and 95); beyond, those split a quarter less
    // (3000 x 515 -> 1029, 799: 39.7 and 34.8; 2048 x 2048 -> 2048, 1024: 119 and 102), unless there is no second row of
    // them to share with (30 rows, 3116 -> 2 x 6976: 59 and 93; 42 rows, 7138 -> 2 x 3080: 65 and 100).
    if (side == 128)
      product_kernel<T, TA, TB, 128, 128, G><<<grid, 256, 0, st>>>(a, b, K, ntn, per, o);
    else if (sizeof(T) == 2 || ntm == 1 || (long long)ntm * ntn * p.S <= 768)
      product_kernel<T, TA, TB, 64, 64, G><<<grid, 256, 0, st>>>(a, b, K, ntn, per, o);
    else if constexpr (sizeof(T) == 4)
      product_kernel<T, TA, TB, 128, 64, G><<<dim3((unsigned)((M + 127) / 128 * ntn), (unsigned)p.S), 256, 0, st>>>(a, b, K, ntn, per, o);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.S == 1) return e;
  o.part = nullptr;
  const long long n4 = M * ((N + 3) / 4);
  split_sum_kernel<T, G ? 2 : 1><<<(unsigned)((n4 + 255) / 256), 256, 0, st>>>(part, p.S, o);
  return hipGetLastError();
}

}  // namespace
}  // namespace bsa
