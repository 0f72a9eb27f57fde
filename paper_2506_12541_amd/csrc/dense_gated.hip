// Gated map and its gradients: with [g | u] = x w^T + bias, w [2n, k],
//   y = act(g) u;   dg = dy u act'(g), du = dy act(g), dz = [dg | du], dx = dz w, dw = dz^T x,
//   db = sum dz.
// The forward is one product whose workgroups hold the same columns of both maps, so g and u meet in
// registers (dense_product.hpp) and only y is written (and, for the backward, [g | u]). The backward's two
// products are the affine map's over the 2n columns of dz. float32 operands of large products are split into
// their bf16 parts once, in a pass before (planes, below).
// Bound by the matrix cores from a few hundred rows on, below by the weight's bytes.
#include "dense_product.hpp"

namespace bsa {
namespace {

// 32 column pieces x 8 rows at a time; workgroup (x, y) takes rows y rpg .. and leaves the sums of its
// columns of dg and du in part[y][2n] (NULL: not formed).
template <typename T>
__global__ void __launch_bounds__(256) gated_dz_kernel(const T* __restrict__ dy, long long lddy, const T* __restrict__ pre,
                                                       int act, long long m, int n, long long rpg, T* __restrict__ dz,
                                                       long long lddz, float* __restrict__ part) {
  constexpr int E = 16 / (int)sizeof(T);
  __shared__ float red[8][2][32 * E + 4];
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
  const int c = (blockIdx.x * 32 + cx) * E;
  const long long r0 = blockIdx.y * rpg, r1 = r0 + rpg < m ? r0 + rpg : m;
  float s[2][E];
#pragma unroll
  for (int e = 0; e < E; ++e) s[0][e] = s[1][e] = 0.f;
  if (c < n) {
    const Mat<T> my{dy, lddy, m, n}, mg{pre, 2LL * n, m, n}, mu{pre + n, 2LL * n, m, n};
#pragma unroll 2
    for (long long r = r0 + ry; r < r1; r += 8) {
      float y[E], g[E], u[E];
      unpack16<T>(load_piece(my, r, c), y);
      unpack16<T>(load_piece(mg, r, c), g);
      unpack16<T>(load_piece(mu, r, c), u);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float z = g[e];
        g[e] = y[e] * u[e] * act_slope<T>(z, act);
        u[e] = y[e] * act_fwd<T>(z, act);
        s[0][e] += g[e];
        s[1][e] += u[e];
      }
      T* const p = dz + r * lddz + c;
      if (c + E <= n) {
        store16u(p, pack16<T>(g));
        store16u(p + n, pack16<T>(u));
      } else {
        store_partial(p, pack16<T>(g), n - c);
        store_partial(p + n, pack16<T>(u), n - c);
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < E; ++e) red[ry][h][cx * E + e] = s[h][e];
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * 32 * E; i += 256) {
    const int h = i / (32 * E), x = i % (32 * E);
    float v = red[0][h][x];
#pragma unroll
    for (int k = 1; k < 8; ++k) v += red[k][h][x];
    const int col = blockIdx.x * 32 * E + x;
    if (col < n) part[(long long)blockIdx.y * 2 * n + h * n + col] = v;
  }
}

// ---- float32: operands split into their parts once ----
//
// A float32 value enters a product as three bf16 parts (dense_product.hpp). Formed in the product's tiles, the parts
// of a value are formed again for every tile of the other side; with 64 x 64 tiles, which odd middle sizes end up with,
// that takes longer than multiplying. Here a pass before writes them as three bf16 matrices ("planes", [3][rows][cols], both
// rounded up to 32 with zeros, so that no tile of the contraction is partial), and the product loads its tiles
// straight into LDS. A value past the largest bf16 is cut there and its rest is in the other parts; infinities, whose
// parts would meet zeros, are noted (flags) and send every tile through parts_plain.

constexpr long long up32(long long x) { return (x + 31) / 32 * 32; }

__device__ __forceinline__ void split3(float x, bf16_t (&p)[3], bool& inf) {
  const float top = 3.3895314e38f;     // the largest bf16 value
  const bool endless = fabsf(x) == __builtin_huge_valf();
  inf |= endless;
  float x1 = bf2f(f2bf(x));
  if (fabsf(x1) > top && !endless) x1 = copysignf(top, x);
  const float r = endless ? 0.f : x - x1, x2 = bf2f(f2bf(r));
  p[0] = f2bf(x1);
  p[1] = f2bf(x2);
  p[2] = f2bf(r - x2);
}

struct Planes {
  const float* src;
  long long ld, rows;
  int cols;
  bf16_t* to;          // [3][up32(rows)][up32(cols)]
  int* flags;          // one for each workgroup: it met an infinity
};
constexpr int kSplitBlocks = 512;

// Two matrices (blockIdx.y), four columns to a thread.
__global__ void __launch_bounds__(256) split_planes_kernel(Planes p0, Planes p1) {
  const Planes p = blockIdx.y ? p1 : p0;
  const long long R = up32(p.rows), plane = R * up32(p.cols);
  const int C4 = (int)(up32(p.cols) / 4);
  bool inf = false;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < R * C4; i += 256LL * kSplitBlocks) {
    const long long r = i / C4;
    const int c = (int)(i - r * C4) * 4;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (r < p.rows) {
      const float* s = p.src + r * p.ld + c;
      if (c + 4 <= p.cols) {
        load4u(s, v);
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (c + e < p.cols) v[e] = s[e];
      }
    }
    bf16_t q[4][3];
#pragma unroll
    for (int e = 0; e < 4; ++e) split3(v[e], q[e], inf);
#pragma unroll
    for (int k = 0; k < 3; ++k)
      *reinterpret_cast<ushort4*>(p.to + k * plane + r * 4 * C4 + c) = make_ushort4(q[0][k], q[1][k], q[2][k], q[3][k]);
  }
  const int any = __syncthreads_or(inf);
  if (threadIdx.x == 0) p.flags[blockIdx.x] = any;
}

// A matrix of planes: Mat of the first, elements to the next.
struct PlaneMat {
  Mat<bf16_t> m;
  long long plane;
  __device__ __forceinline__ float at(long long r, long long c) const {
    const bf16_t* p = m.p + r * m.ld + c;
    return bf2f(p[0]) + (bf2f(p[plane]) + bf2f(p[2 * plane]));
  }
};

// Accumulators of a wave tile by f32 matrix instructions from the sums of the parts, which are the values.
template <bool TA, bool TB, bool G, int FI, int FJ>
__device__ __forceinline__ void parts_plain(const PlaneMat& a, const PlaneMat& b, long long m0, long long n0, long long k0,
                                            long long k1, int lane, f32x4 (&acc)[FI][FJ]) {
  const int r = lane & 15, j = lane >> 4;
  auto at = [](const PlaneMat& m, bool tr, long long o, long long k) {
    const bool in = tr ? o < m.m.cols : o < m.m.rows;
    return in ? (tr ? m.at(k, o) : m.at(o, k)) : 0.f;
  };
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int jj = 0; jj < FJ; ++jj) acc[i][jj] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (long long k = k0; k < k1; k += 4) {     // k1 - k0: a multiple of 32
    float x[FI], y[FJ];
#pragma unroll
    for (int i = 0; i < FI; ++i) x[i] = at(a, TA, m0 + 16 * i + r, k + j);
#pragma unroll
    for (int i = 0; i < FJ; ++i) y[i] = at(b, TB, stored_row<G>(b.m, n0 + 16 * i + r), k + j);
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int jj = 0; jj < FJ; ++jj) acc[i][jj] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[jj], x[i], acc[i][jj], 0, 0, 0);
  }
}

// BM x 128 tiles of 8 waves, contraction tiles of 32: BM = 256, waves of 64 x 64 and two LDS stages of 72 KB, or BM = 128,
// waves of 64 x 32 (more LDS reads for a product) and three stages of 48 KB. One workgroup to a CU, two waves to a SIMD
// (4 waves of 64 x 64 on 128 x 128 tiles read less, but nothing runs while one waits: 14 % slower). 16384 x 1024 -> 2 x 2048: 713 us
// with 256 rows (193 TFLOP/s), 767 with 128; 3586 x 515 -> 2 x 1029: 57 and 62 of the forward's 61 and 67.
template <bool TA, bool TB, bool G, int BM>
__global__ void __launch_bounds__(512, 2) parts_kernel(PlaneMat a, PlaneMat b, int nkt, int ntm, int ntn, int kt_per,
                                                       const int* fa, int nfa, const int* fb, int nfb, Epi<float> o) {
  constexpr int BN = 128, BK = 32, NS = BM == 256 ? 2 : 3, WN = BM == 256 ? 2 : 4, FI = 4, FJ = 8 / WN;
  constexpr int AT = BM * BK, BT = BN * BK;
  // a stage is an array of its own: reads of one stage do not wait for loads into another
  __shared__ __attribute__((aligned(1024))) bf16_t st0[3 * (AT + BT)], st1[3 * (AT + BT)], st2[NS == 3 ? 3 * (AT + BT) : 8];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wid / WN, wn = wid % WN;
  // XCDs take contiguous runs of tiles, in bands of 8 tile rows walked column by column (product_dma_kernel)
  const int nt = ntm * ntn;
  int id = blockIdx.x;
  if ((nt & 7) == 0) id = (id & 7) * (nt >> 3) + (id >> 3);
  const int band = id / (8 * ntn), in = id - band * 8 * ntn, bh = min(8, ntm - 8 * band);
  const int tm = 8 * band + in % bh, tn = in / bh;
  const long long m0 = (long long)tm * BM, n0 = (long long)tn * BN;
  const int kt0 = min((int)blockIdx.y * kt_per, nkt), kt1 = min(kt0 + kt_per, nkt);
  DmaTile<TA, TA != TB, TA ? BK : BM, TA ? BM : BK, 8> la;
  DmaTile<TB, TA != TB, TB ? BK : BN, TB ? BN : BK, 8, G> lb;
  la.init(a.m, m0, wid, lane);
  lb.init(b.m, n0, wid, lane);
  constexpr int PER = 3 * (decltype(la)::NU + decltype(lb)::NU);
  auto issue = [&](int kt, bf16_t* st, int k) __attribute__((always_inline)) {
    la.issue(st + k * AT, a.m, (long long)kt * BK, wid, 2 * k * a.plane);
    lb.issue(st + 3 * AT + k * BT, b.m, (long long)kt * BK, wid, 2 * k * b.plane);
  };
  f32x4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 af[3][FI], bf[3][FJ];
  auto read_a = [&](const bf16_t* st, int k) __attribute__((always_inline)) {
    Frags<TA, TA != TB, BK, BM, FI>::read(st + k * AT, wm * 64, 0, lane, af[k]);
  };
  auto read_b = [&](const bf16_t* st, int k) __attribute__((always_inline)) {
    Frags<TB, TA != TB, BK, BN, FJ>::read(st + 3 * AT + k * BT, wn * 16 * FJ, 0, lane, bf[k]);
  };
  auto multiply = [&](int ka, int kb) {
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) acc[i][j] = mma(bf[kb][j], af[ka][i], acc[i][j]);
  };
  // tile t lies in stage c; the stage `free` has been read. NS - 2 tiles stay in flight while t is waited for
  auto step = [&](int t, const bf16_t* c, bf16_t* free) __attribute__((always_inline)) {
    if (NS == 3 && t + 1 < kt1)
      vm_wait<PER>();
    else
      vm_drain();
    lds_barrier();     // every wave's loads of tile t are visible, and it has its fragments of t - 1
    const int next = t + NS - 1;
    // the small part products first; the next loads between the products, so that no wave queues for all of them
    const bool more = next < kt1;
    read_a(c, 2);
    read_b(c, 0);
    multiply(2, 0);
    if (more) issue(next, free, 0);
    read_a(c, 0);
    read_b(c, 2);
    multiply(0, 2);
    if (more) issue(next, free, 1);
    read_a(c, 1);
    read_b(c, 1);
    multiply(1, 1);
    if (more) issue(next, free, 2);
    multiply(1, 0);
    multiply(0, 1);
    multiply(0, 0);
    lgkm_drain();
  };
#pragma unroll
  for (int u = 0; u < NS - 1; ++u)
    if (kt0 + u < kt1) {
#pragma unroll
      for (int k = 0; k < 3; ++k) issue(kt0 + u, u ? st1 : st0, k);
    }
  if constexpr (NS == 3) {
    for (int kt = kt0; kt < kt1; kt += 3) {
      step(kt, st0, st2);
      if (kt + 1 < kt1) step(kt + 1, st1, st0);
      if (kt + 2 < kt1) step(kt + 2, st2, st1);
    }
  } else {
    for (int kt = kt0; kt < kt1; kt += 2) {
      step(kt, st0, st1);
      if (kt + 1 < kt1) step(kt + 1, st1, st0);
    }
  }
  int odd = 0;
  for (int i = threadIdx.x; i < nfa; i += 512) odd |= fa[i];
  for (int i = threadIdx.x; i < nfb; i += 512) odd |= fb[i];
  if (__syncthreads_or(odd))
    parts_plain<TA, TB, G, FI, FJ>(a, b, m0 + wm * 64, n0 + wn * 16 * FJ, (long long)kt0 * BK, (long long)kt1 * BK, lane, acc);
#pragma unroll
  for (int i = 0; i < FI; ++i) {
    const long long m = m0 + wm * 64 + 16 * i + (lane & 15);
#pragma unroll
    for (int j = 0; j < FJ; j += G ? 2 : 1) {
      const int n = (int)n0 + wn * 16 * FJ + 16 * j + 4 * (lane >> 4);
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

// dz as planes [3][up32(m)][up32(2n)] and its partial column sums; otherwise as gated_dz_kernel. The last
// workgroups also clear the rows and columns behind dz. flags: one for each workgroup.
__global__ void __launch_bounds__(256) gated_dz_planes_kernel(const float* __restrict__ dy, long long lddy,
                                                              const float* __restrict__ pre, int act, long long m, int n,
                                                              long long rpg, bf16_t* __restrict__ dz, float* __restrict__ part,
                                                              int* __restrict__ flags) {
  __shared__ float red[8][2][132];
  const long long R = up32(m), C = up32(2LL * n), plane = R * C;
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5, c = (blockIdx.x * 32 + cx) * 4;
  const long long r0 = blockIdx.y * rpg, r1 = r0 + rpg < m ? r0 + rpg : m;
  bool inf = false;
  float s[2][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) s[0][e] = s[1][e] = 0.f;
  if (c < n) {
    const Mat<float> my{dy, lddy, m, n}, mg{pre, 2LL * n, m, n}, mu{pre + n, 2LL * n, m, n};
#pragma unroll 2
    for (long long r = r0 + ry; r < r1; r += 8) {
      float y[4], v[2][4];
      unpack16<float>(load_piece(my, r, c), y);
      unpack16<float>(load_piece(mg, r, c), v[0]);
      unpack16<float>(load_piece(mu, r, c), v[1]);
      bf16_t q[2][4][3];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float z = v[0][e];
        const float dg = y[e] * v[1][e] * act_slope<float>(z, act), du = y[e] * act_fwd<float>(z, act);
        s[0][e] += dg;
        s[1][e] += du;
        split3(dg, q[0][e], inf);
        split3(du, q[1][e], inf);
      }
#pragma unroll
      for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16_t* const p = dz + k * plane + r * C + h * n + c;
          const ushort4 w = make_ushort4(q[h][0][k], q[h][1][k], q[h][2][k], q[h][3][k]);
          if (c + 4 <= n) {
            __builtin_memcpy(p, &w, 8);
          } else {
            p[0] = w.x;
            if (c + 1 < n) p[1] = w.y;
            if (c + 2 < n) p[2] = w.z;
          }
        }
    }
  }
  if (blockIdx.x == 0) {       // the columns behind, of this workgroup's rows
    const int w = (int)(C - 2 * n);
    for (long long i = threadIdx.x; i < (r1 - r0) * w; i += 256)
      for (int k = 0; k < 3; ++k) dz[k * plane + (r0 + i / w) * C + 2 * n + i % w] = 0;
  }
  if (blockIdx.y == gridDim.y - 1) {   // the rows behind
    for (long long i = blockIdx.x * 256LL + threadIdx.x; i < (R - m) * C; i += 256LL * gridDim.x)
      for (int k = 0; k < 3; ++k) dz[k * plane + m * C + i] = 0;
  }
  const int any = __syncthreads_or(inf);
  if (threadIdx.x == 0) flags[blockIdx.y * gridDim.x + blockIdx.x] = any;
  if (!part) return;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[ry][h][cx * 4 + e] = s[h][e];
  __syncthreads();
  for (int i = threadIdx.x; i < 256; i += 256) {
    const int h = i / 128, x = i % 128;
    float v = red[0][h][x];
#pragma unroll
    for (int k = 1; k < 8; ++k) v += red[k][h][x];
    const int col = blockIdx.x * 128 + x;
    if (col < n) part[(long long)blockIdx.y * 2 * n + h * n + col] = v;
  }
}

// ---- bf16 rows that do not begin on 16 bytes ----
//
// The products load 16-byte pieces straight into LDS where rows begin on 16 bytes. Others are copied so that they do,
// zeros behind their ends.

struct PadJob {
  const bf16_t* src;
  long long ld, rows;
  bf16_t* dst;
};

// 32 column pieces x 8 rows at a time
__global__ void __launch_bounds__(256) pad_rows_kernel(PadJob j0, PadJob j1, int cols, int pitch) {
  const PadJob j = blockIdx.z ? j1 : j0;
  const int c = 8 * (blockIdx.x * 32 + (threadIdx.x & 31));
  if (c >= cols) return;
  const bool words = !((uintptr_t)j.src & 2);
  const Mat<bf16_t> m{j.src, j.ld, j.rows, cols};
#pragma unroll 2
  for (long long r = blockIdx.y * 8LL + (threadIdx.x >> 5); r < j.rows; r += 8LL * gridDim.y)
    *reinterpret_cast<uint4*>(j.dst + r * pitch + c) = words && c + 8 <= cols ? load16_words(j.src + r * j.ld + c) : load_piece(m, r, c);
}

// ---- gradients of few rows: the weight is read, and its gradient written, once ----
//
// Float32 with few rows is no work for the matrix cores: 16 multiply-adds for a value of w, or of dw, keep up with
// memory. A lane holds 16 bytes of columns; a row's dz are the same for all lanes and come from LDS. MR: rows that are
// computed (m of them are there). Both kernels are bound by memory: 2 rows and w of 10880 x 7168, which takes 60 us at
// a copy's rate, dx 64 us and dw 58, each with the launches before and behind it.

constexpr int kFewChunk = 64;    // rows of w whose dz are staged at a time

// zs[j][i] = dz[i][r0 + j], 0 behind the ends.
template <int MR>
__device__ __forceinline__ void stage_dz(float (&zs)[kFewChunk][MR], const float* dz, int m, int n2, int r0, int r1) {
  for (int i = threadIdx.x; i < kFewChunk * MR; i += 256) {
    const int row = i / kFewChunk, j = i % kFewChunk;
    zs[j][row] = row < m && r0 + j < r1 ? dz[(long long)row * n2 + r0 + j] : 0.f;
  }
}

// dx = dz w: the workgroup's columns 64 E blockIdx.x .. of the rows [r0, r1) of w that blockIdx.y takes; its waves
// take them in turn and are joined in order.
template <int MR>
__global__ void __launch_bounds__(256) few_dx_kernel(const float* __restrict__ dz, const float* __restrict__ w, long long ldw, int m,
                                                     int k, int n2, int per, Epi<float> o) {
  constexpr int E = 4, U = 4;
  __shared__ __attribute__((aligned(16))) float zs[kFewChunk][MR], red[4][64 * E + 4];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (blockIdx.x * 64 + lane) * E, left = k - c;
  const int r0 = blockIdx.y * per, r1 = min(r0 + per, n2);
  float acc[MR][E];
#pragma unroll
  for (int i = 0; i < MR; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) acc[i][e] = 0.f;
  for (int b = r0; b < r1; b += kFewChunk) {
    __syncthreads();
    stage_dz<MR>(zs, dz, m, n2, b, r1);
    __syncthreads();
    for (int j = wid; j < kFewChunk && b + j < r1; j += 4 * U) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {     // rows behind the last repeat its loads and are left out below
        const float* p = w + (long long)min(b + j + 4 * u, r1 - 1) * ldw + c;
        v[u] = left >= E ? load16u(p) : left > 0 ? load_partial(p, left) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (b + j + 4 * u < r1) {
          float x[E];
          unpack16<float>(v[u], x);
#pragma unroll
          for (int i = 0; i < MR; ++i) {
            const float z = zs[j + 4 * u][i];
#pragma unroll
            for (int e = 0; e < E; ++e) acc[i][e] = fmaf(z, x[e], acc[i][e]);
          }
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < MR; ++i) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) red[wid][lane * E + e] = acc[i][e];
    __syncthreads();
    if (i < m && threadIdx.x < 16 * E) {
      const int x = 4 * threadIdx.x;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = red[0][x + e] + red[1][x + e] + red[2][x + e] + red[3][x + e];
      epi_store4(o, i, blockIdx.x * 64 * E + x, v, blockIdx.y);
    }
  }
}

// dw = dz^T x: kFewChunk rows of dw by 256 columns, its waves in turn; cols workgroups share the rows.
template <int MR>
__global__ void __launch_bounds__(256) few_dw_kernel(const float* __restrict__ dz, const float* __restrict__ x, long long ldx, int m,
                                                     int k, int n2, int cols, float* __restrict__ dw) {
  constexpr int E = 4;
  __shared__ __attribute__((aligned(16))) float zs[kFewChunk][MR];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (blockIdx.x % cols * 64 + lane) * E, left = k - c, r0 = blockIdx.x / cols * kFewChunk;
  float xs[MR][E];
#pragma unroll
  for (int i = 0; i < MR; ++i) {
    const float* p = x + min(i, m - 1) * ldx + c;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (i < m) v = left >= E ? load16u(p) : left > 0 ? load_partial(p, left) : v;
    unpack16<float>(v, xs[i]);
  }
  stage_dz<MR>(zs, dz, m, n2, r0, n2);
  __syncthreads();
  if (left <= 0) return;
  for (int j = wid; j < kFewChunk && r0 + j < n2; j += 4) {
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = 0.f;
#pragma unroll
    for (int i = 0; i < MR; ++i) {
      const float z = zs[j][i];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = fmaf(z, xs[i][e], v[e]);
    }
    float* const to = dw + (long long)(r0 + j) * k + c;
    if (left >= E)
      store16u(to, pack16<float>(v));
    else
      store_partial(to, pack16<float>(v), left);
  }
}

// ---- host ----

// The forward's product has 2n columns.
Plan fwd_plan(const GatedArgs& a) { return plan_product(a.bf16, a.m, 2 * a.n, a.k); }

int up8(int x) { return (x + 7) / 8 * 8; }
// dz belongs to this file: its rows begin on 16 bytes, and what lies behind them may be read.
long long dz_pitch(const GatedArgs& a) { return a.bf16 ? up8(2 * a.n) : 2LL * a.n; }
LinearArgs rows_of(const GatedArgs& a) {
  return LinearArgs{a.m, a.k, 2 * a.n, a.bf16, kActNone, a.ldx, a.ldw, 0, 0, dz_pitch(a), 0, (int)dz_pitch(a)};
}

// Whether bf16 operands whose rows do not begin on 16 bytes (backward: or end inside of them) are copied first: where
// the products are long enough for it. us (forward, backward) with copies and without: 8191 x 1023 -> 2 x 2047 105, 228
// and 157, 290; 47687 x 84 -> 2 x 3201 376, 859 and 526, 866; 65536 x 511 -> 2 x 257 94, 322 and 139, 320; 4015 x 133 ->
// 2 x 6683 67, 212 and 103, 245; 2048 x 2047 -> 2 x 1023 46, 92 and 41, 100; 1954 x 1331 -> 2 x 824 41, 83 and 45, 82;
// 1000 x 707 -> 2 x 300 20, 48 and 17, 43; 64 x 8191 -> 2 x 4096 106, 181 and 40, 144.
struct Pads {
  bool x, w;
  size_t x_bytes, w_bytes;
};
Pads pads(const GatedArgs& a, bool backward) {
  if (!a.bf16 || a.m * a.n < (3LL << 30) / a.k || a.m < 1024) return Pads{};
  Pads p{};
  p.x = a.ldx % 8 || (backward && a.k % 8);
  p.w = a.ldw % 8 || (backward && a.k % 8);
  p.x_bytes = p.x ? align256(sizeof(bf16_t) * (size_t)a.m * up8(a.k)) : 0;
  p.w_bytes = p.w ? align256(sizeof(bf16_t) * (size_t)2 * a.n * up8(a.k)) : 0;
  return p;
}

// Copies of x and w, those that p names, behind one another at `to`, as their places in a.
hipError_t pad(GatedArgs& a, const Pads& p, const void*& x, const void*& w, char* to, hipStream_t st) {
  PadJob j[2]{};
  int n = 0;
  if (p.x) j[n++] = PadJob{(const bf16_t*)x, a.ldx, a.m, (bf16_t*)to}, x = to, a.ldx = up8(a.k), to += p.x_bytes;
  if (p.w) j[n++] = PadJob{(const bf16_t*)w, a.ldw, 2LL * a.n, (bf16_t*)to}, w = to, a.ldw = up8(a.k);
  if (n == 0) return hipSuccess;
  const unsigned gx = (unsigned)((a.k + 255) / 256);
  const long long rows = std::max(j[0].rows, j[1].rows), gy = std::min<long long>((rows + 15) / 16, std::max(2048 / gx, 1u));
  pad_rows_kernel<<<dim3(gx, (unsigned)gy, n), 256, 0, st>>>(j[0], j[1], a.k, up8(a.k));
  return hipGetLastError();
}

// Whether float32 products go through planes: where both sides of a product have several tiles that share them, and
// the forward's one product is long enough for the pass before it. us (forward, backward) by planes and without:
// 3586 x 515 -> 2 x 1029: 61, 156 and 76, 255; 2000 x 2048 -> 2 x 2048: 169, 352 and 200, 475; 8192 x 1024 -> 2 x 2048: 343, 693 and
// 423, 981; 65536 x 256 -> 2 x 1024: 582, 1049 and 568, 1391; 1024 x 1024 -> 2 x 1024: 40, 89 and 42, 115; 2048 x 512 -> 2 x 1024:
// 38, 91 and 40, 116; 800 x 256 -> 2 x 512: 12 (none), 49 and 13, 44; 20000 x 256 -> 2 x 256: 56, 134 and 52, 138; 300 x 4096 ->
// 2 x 4096: 218, 378 and 212, 447; 65536 x 64 -> 2 x 1024: 275, 728 and 271, 707.
bool bwd_planes(const GatedArgs& a) {
  const long long most = 1LL << 35;     // launches of fewer than 2^23 workgroups
  return !a.bf16 && a.m >= 768 && a.n >= 512 && a.k >= 256 && a.k <= (1 << 22) && a.n <= (1 << 21) && a.m * a.n <= most &&
         a.m * a.k <= most && (long long)a.n * a.k <= most;
}
bool fwd_planes(const GatedArgs& a) { return bwd_planes(a) && a.m * a.n >= (3LL << 29) / a.k; }
size_t planes_bytes(long long rows, long long cols) { return align256(3 * sizeof(bf16_t) * (size_t)(up32(rows) * up32(cols))); }

// Rows of a tile and splits of the contraction.
struct PartsPlan {
  int BM, S;
};
// What ends first, in units of 0.1 us: each of 256 CUs takes 1.2 us for a tile of 128 x 128 x 32, 1.9 for 256 x 128 x 32, 4 and 6
// for a workgroup's start and end, and the splits' sums are written and read at 4 TB/s behind another launch of 4 us.
PartsPlan parts_plan(long long M, long long N, long long K, int outs) {
  const long long nkt = (K + 31) / 32;
  long long best = 0;
  PartsPlan p{128, 1};
  for (int BM : {128, 256})
    for (long long S = 1; S <= 16 && S <= nkt; ++S) {
      const long long tiles = (M + BM - 1) / BM * ((N * outs + 127) / 128);
      const long long t = (tiles * S + 255) / 256 * ((nkt + S - 1) / S * (BM == 128 ? 12 : 19) + (BM == 128 ? 40 : 60)) +
                          (S > 1 ? 40 + S * M * N * outs / 50000 : 0);
      if (best == 0 || t < best) best = t, p = PartsPlan{BM, (int)S};
    }
  return p;
}

// Whether float32 gradients of few rows go through few_dw_kernel and few_dx_kernel. The products' tiles would be mostly
// empty rows. dw, us by the kernel and by tiles: 16 rows, w of 8192 x 4096 39 and 73, 4096 x 2048 19 and 27, 2048 x 1024
// 18 and 17; 32 rows 64 and 78, 25 and 29, 22 and 16. dx reads all splits once more to join them, which weighs when k is
// short: 8 rows, w of 10880 x 7168 74 and 110, 8192 x 4096 44 and 50, 4096 x 2048 23 and 22, 16384 x 512 34 and 28; 2 rows
// 64 and 114, 40 and 52, 19 and 21, 29 and 27; 16 rows 92 and 112, 53 and 52, 30 and 23, 44 and 29.
bool few_dw(const GatedArgs& a) { return !a.bf16 && a.m <= 16; }
bool few_dx(const GatedArgs& a) { return !a.bf16 && a.m <= 8 && a.k >= 1024 && 2LL * a.n * a.k >= 1 << 24; }
// Splits of dx, in chunks of kFewChunk rows of w: about two workgroups to a CU.
int few_splits(const GatedArgs& a) {
  const int cols = (a.k + 255) / 256, chunks = (2 * a.n + kFewChunk - 1) / kFewChunk;
  return std::max(1, std::min(std::min(512 / cols, chunks), 64));
}

template <int MR>
void few_dw_rows(const GatedArgs& a, const float* x, const float* dz, float* dw, hipStream_t st) {
  const int cols = (a.k + 255) / 256, chunks = (2 * a.n + kFewChunk - 1) / kFewChunk;
  few_dw_kernel<MR><<<(unsigned)((long long)cols * chunks), 256, 0, st>>>(dz, x, a.ldx, (int)a.m, a.k, 2 * a.n, cols, dw);
}
hipError_t few_dw_run(const GatedArgs& a, const float* x, const float* dz, float* dw, hipStream_t st) {
  (a.m <= 4 ? few_dw_rows<4> : a.m <= 8 ? few_dw_rows<8> : few_dw_rows<16>)(a, x, dz, dw, st);
  return hipGetLastError();
}

template <int MR>
void few_dx_rows(const GatedArgs& a, const float* w, const float* dz, int S, const Epi<float>& o, hipStream_t st) {
  const int cols = (a.k + 255) / 256, chunks = (2 * a.n + kFewChunk - 1) / kFewChunk, per = (chunks + S - 1) / S * kFewChunk;
  few_dx_kernel<MR><<<dim3(cols, S), 256, 0, st>>>(dz, w, a.ldw, (int)a.m, a.k, 2 * a.n, per, o);
}
hipError_t few_dx_run(const GatedArgs& a, const float* w, const float* dz, float* dx, float* part, hipStream_t st) {
  const int S = few_splits(a);
  Epi<float> o{a.m, a.k, dx, a.k, nullptr, nullptr, 0, nullptr, kActNone, S > 1 ? part : nullptr};
  (a.m <= 4 ? few_dx_rows<4> : few_dx_rows<8>)(a, w, dz, S, o, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || S == 1) return e;
  o.part = nullptr;
  const long long n4 = a.m * ((a.k + 3) / 4);
  split_sum_kernel<float, 1><<<(unsigned)((n4 + 255) / 256), 256, 0, st>>>(part, S, o);
  return hipGetLastError();
}

struct GatedBwdWs {
  size_t dz, dbp, rest, total;
  size_t w, x, flags;        // planes of w and x, and the flags of w, x and dz
  int P;
  long long rpg;
  PartsPlan px, pw;          // of dx and dw
  Pads pads;                 // x and w copied, at x
};
GatedBwdWs gated_bwd_layout(const GatedArgs& a) {
  GatedBwdWs L{};
  const size_t esz = a.bf16 ? 2 : 4;
  const int E = 16 / (int)esz;
  // row groups of the dz pass: about 1024 workgroups, at least 32 rows each
  const long long gx = (a.n + 32 * E - 1) / (32 * E);
  long long P = std::min<long long>(std::max<long long>(1024 / gx, 1), (a.m + 31) / 32);
  P = std::max<long long>(std::min<long long>(P, 256), 1);
  L.rpg = (a.m + P - 1) / P;
  L.P = (int)(L.rpg ? (a.m + L.rpg - 1) / L.rpg : 1);
  size_t off = 0;
  auto put = [&](size_t b) { const size_t o = off; off += align256(b); return o; };
  L.dbp = put(sizeof(float) * (size_t)L.P * 2 * a.n);
  if (bwd_planes(a)) {
    L.dz = put(planes_bytes(a.m, 2LL * a.n));
    L.w = put(planes_bytes(2LL * a.n, a.k));
    L.x = put(planes_bytes(a.m, a.k));
    L.flags = put(sizeof(int) * (2 * kSplitBlocks + (size_t)gx * L.P));
    L.px = parts_plan(a.m, a.k, 2LL * a.n, 1);
    L.pw = parts_plan(2LL * a.n, a.k, a.m, 1);
    auto part = [](int S, long long M, long long N) { return S > 1 ? sizeof(float) * (size_t)S * M * N : 0; };
    L.rest = put(std::max(part(L.px.S, a.m, a.k), part(L.pw.S, 2LL * a.n, a.k)));
  } else {
    L.dz = put(esz * (size_t)a.m * dz_pitch(a));
    L.pads = pads(a, true);
    L.x = put(L.pads.x_bytes + L.pads.w_bytes);
    const size_t own = few_dx(a) ? sizeof(float) * (size_t)few_splits(a) * a.m * a.k : 0;
    L.rest = put(few_dx(a) && few_dw(a) ? own : std::max(own, linear_bwd_ws_bytes(rows_of(a))));
  }
  L.total = off;
  return L;
}

Planes planes_of(const float* src, long long ld, long long rows, int cols, void* to, int* flags) {
  return Planes{src, ld, rows, cols, (bf16_t*)to, flags};
}
// The planes as an operand. In column form the zeros behind a row are columns of it.
PlaneMat plane_mat(const void* p, long long rows, long long cols, bool column) {
  const long long C = up32(cols), R = up32(rows);
  return PlaneMat{Mat<bf16_t>{(const bf16_t*)p, C, column ? R : rows, (int)C}, R * C};
}

// C = A B^T of planes; S > 1: partial sums in part, joined by split_sum_kernel
template <bool TA, bool TB, bool G>
hipError_t parts_product(const PlaneMat& a, const PlaneMat& b, long long M, int N, long long K, PartsPlan p, float* part, const int* fa,
                         int nfa, const int* fb, int nfb, Epi<float> o, hipStream_t st) {
  const int S = p.S;
  o.part = S > 1 ? part : nullptr;
  const int nkt = (int)(up32(K) / 32), ntm = (int)((M + p.BM - 1) / p.BM), ntn = G ? (N + 63) / 64 : (N + 127) / 128;
  const dim3 grid((unsigned)((long long)ntm * ntn), (unsigned)S);
  const int per = (nkt + S - 1) / S;
  if (p.BM == 256)
    parts_kernel<TA, TB, G, 256><<<grid, 512, 0, st>>>(a, b, nkt, ntm, ntn, per, fa, nfa, fb, nfb, o);
  else
    parts_kernel<TA, TB, G, 128><<<grid, 512, 0, st>>>(a, b, nkt, ntm, ntn, per, fa, nfa, fb, nfb, o);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || S == 1) return e;
  o.part = nullptr;
  const long long n4 = M * ((N + 3) / 4);
  split_sum_kernel<float, G ? 2 : 1><<<(unsigned)((n4 + 255) / 256), 256, 0, st>>>(part, S, o);
  return hipGetLastError();
}

struct GatedFwdWs {
  size_t x, w, flags, part, total;
  PartsPlan p;
  Pads pads;
};
GatedFwdWs gated_fwd_layout(const GatedArgs& a) {
  GatedFwdWs L{};
  size_t off = 0;
  auto put = [&](size_t b) { const size_t o = off; off += align256(b); return o; };
  if (fwd_planes(a)) {
    L.p = parts_plan(a.m, a.n, a.k, 2);
    L.x = put(planes_bytes(a.m, a.k));
    L.w = put(planes_bytes(2LL * a.n, a.k));
    L.flags = put(sizeof(int) * 2 * kSplitBlocks);
    L.part = put(L.p.S > 1 ? sizeof(float) * (size_t)L.p.S * a.m * 2 * a.n : 0);
  } else if (!few_rows_ok(a.m, a.k)) {
    L.part = put(plan_bytes(fwd_plan(a), a.m, 2LL * a.n));
    L.pads = pads(a, false);
    L.x = put(L.pads.x_bytes + L.pads.w_bytes);
  }
  L.total = off;
  return L;
}

hipError_t split_two(const Planes& p, const Planes& q, hipStream_t st) {
  split_planes_kernel<<<dim3(kSplitBlocks, 2), 256, 0, st>>>(p, q);
  return hipGetLastError();
}

hipError_t planes_fwd(const GatedArgs& a, const void* x, const void* w, const Epi<float>& o, char* ws, hipStream_t st) {
  const GatedFwdWs L = gated_fwd_layout(a);
  int* const flags = (int*)(ws + L.flags);
  const hipError_t e = split_two(planes_of((const float*)x, a.ldx, a.m, a.k, ws + L.x, flags),
                                 planes_of((const float*)w, a.ldw, 2LL * a.n, a.k, ws + L.w, flags + kSplitBlocks), st);
  if (e != hipSuccess) return e;
  return parts_product<false, false, true>(plane_mat(ws + L.x, a.m, a.k, false), plane_mat(ws + L.w, 2LL * a.n, a.k, false), a.m, a.n,
                                           a.k, L.p, (float*)(ws + L.part), flags, kSplitBlocks, flags + kSplitBlocks, kSplitBlocks,
                                           o, st);
}

hipError_t planes_bwd(const GatedArgs& a, const GatedBwdWs& L, const void* x, const void* w, const void* pre, const void* dy,
                      void* dx, void* dw, float* dbp, char* ws, hipStream_t st) {
  const int gx = (a.n + 127) / 128;
  int *const fw = (int*)(ws + L.flags), *const fx = fw + kSplitBlocks, *const fz = fx + kSplitBlocks;
  gated_dz_planes_kernel<<<dim3(gx, L.P), 256, 0, st>>>((const float*)dy, a.lddy, (const float*)pre, a.act, a.m, a.n, L.rpg,
                                                       (bf16_t*)(ws + L.dz), dbp, fz);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (!dx && !dw)) return e;
  const Planes pw = planes_of((const float*)w, a.ldw, 2LL * a.n, a.k, ws + L.w, fw);
  const Planes px = planes_of((const float*)x, a.ldx, a.m, a.k, ws + L.x, fx);
  const Planes none_w{nullptr, 0, 0, 0, nullptr, fw}, none_x{nullptr, 0, 0, 0, nullptr, fx};   // not asked for: no rows
  e = split_two(dx ? pw : none_w, dw ? px : none_x, st);
  if (e != hipSuccess) return e;
  if (dx) {
    const Epi<float> o{a.m, a.k, (float*)dx, a.k, nullptr, nullptr, 0, nullptr, kActNone, nullptr};
    e = parts_product<false, true, false>(plane_mat(ws + L.dz, a.m, 2LL * a.n, false), plane_mat(ws + L.w, 2LL * a.n, a.k, true), a.m,
                                          a.k, 2LL * a.n, L.px, (float*)(ws + L.rest), fz, gx * L.P, fw, kSplitBlocks, o, st);
    if (e != hipSuccess) return e;
  }
  if (dw) {
    const Epi<float> o{2LL * a.n, a.k, (float*)dw, a.k, nullptr, nullptr, 0, nullptr, kActNone, nullptr};
    e = parts_product<true, true, false>(plane_mat(ws + L.dz, a.m, 2LL * a.n, true), plane_mat(ws + L.x, a.m, a.k, true), 2LL * a.n,
                                         a.k, a.m, L.pw, (float*)(ws + L.rest), fz, gx * L.P, fx, kSplitBlocks, o, st);
  }
  return e;
}

template <typename T>
hipError_t gated_fwd(GatedArgs a, const void* x, const void* w, const void* bias, void* y, void* pre, void* ws,
                     hipStream_t st) {
  const Epi<T> o{a.m, a.n, (T*)y, a.ldy, (const T*)bias, nullptr, 0, (T*)pre, a.act, nullptr};
  if (few_rows_ok(a.m, a.k))
    return few_rows<T, 2>(Mat<T>{(const T*)x, a.ldx, a.m, a.k}, Mat<T>{(const T*)w, a.ldw, 2LL * a.n, a.k}, a.m, a.n, a.k, o, st);
  if constexpr (sizeof(T) == 4) {
    if (fwd_planes(a)) return planes_fwd(a, x, w, o, (char*)ws, st);
  }
  const GatedFwdWs L = gated_fwd_layout(a);
  const hipError_t e = pad(a, L.pads, x, w, (char*)ws + L.x, st);
  if (e != hipSuccess) return e;
  return product<T, false, false, true>(Mat<T>{(const T*)x, a.ldx, a.m, a.k}, Mat<T>{(const T*)w, a.ldw, 2LL * a.n, a.k}, a.m, a.n,
                                        a.k, fwd_plan(a), (float*)((char*)ws + L.part), o, st);
}

template <typename T>
hipError_t gated_bwd(const GatedArgs& a, const void* x, const void* w, const void* pre, const void* dy, void* dx, void* dw,
                     void* db, void* ws, hipStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  const GatedBwdWs L = gated_bwd_layout(a);
  char* const c = (char*)ws;
  T* const dz = (T*)(c + L.dz);
  float* const dbp = db && a.m > 0 ? (float*)(c + L.dbp) : nullptr;
  const bool planes = a.m > 0 && bwd_planes(a);
  if (planes) {
    const hipError_t e = planes_bwd(a, L, x, w, pre, dy, dx, dw, dbp, c, st);
    if (e != hipSuccess) return e;
  } else if (a.m > 0) {
    gated_dz_kernel<T><<<dim3((a.n + 32 * E - 1) / (32 * E), L.P), 256, 0, st>>>((const T*)dy, a.lddy, (const T*)pre, a.act,
                                                                                 a.m, a.n, L.rpg, dz, dz_pitch(a), dbp);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (sizeof(T) == 4 && a.m > 0) {
    if (dw && few_dw(a)) {
      const hipError_t e = few_dw_run(a, (const float*)x, (const float*)dz, (float*)dw, st);
      if (e != hipSuccess) return e;
      dw = nullptr;
    }
    if (dx && few_dx(a)) {
      const hipError_t e = few_dx_run(a, (const float*)w, (const float*)dz, (float*)dx, (float*)(c + L.rest), st);
      if (e != hipSuccess) return e;
      dx = nullptr;
    }
  }
  if (!planes && (dx || dw || a.m == 0)) {    // without rows this also clears db
    LinearArgs r = rows_of(a);
    // the operands of the gradients that are formed; the other one's pointer may be NULL (8191 x 1023 -> 2 x 2047: dw alone
    // 154.5 us, 157 with a copy of w; dx alone 136 and 142)
    Pads pads = L.pads;
    pads.x = pads.x && dw && a.m > 0;
    pads.w = pads.w && dx && a.m > 0;
    if (pads.x || pads.w) {
      GatedArgs p = a;
      const hipError_t e = pad(p, pads, x, w, c + L.x, st);
      if (e != hipSuccess) return e;
      r.ldx = p.ldx, r.ldw = p.ldw, r.readable_k = up8(a.k);
    }
    const hipError_t e = launch_linear_bwd(r, x, w, nullptr, dz, dx, dw, a.m > 0 ? nullptr : db, c + L.rest, st);
    if (e != hipSuccess) return e;
  }
  if (!dbp) return hipSuccess;
  db_sum_kernel<T><<<(2 * a.n + 63) / 64, 1024, 0, st>>>(dbp, L.P, 2 * a.n, (T*)db);
  return hipGetLastError();
}

}  // namespace

size_t gated_fwd_ws_bytes(const GatedArgs& a) { return gated_fwd_layout(a).total; }

hipError_t launch_gated_fwd(const GatedArgs& a, const void* x, const void* w, const void* bias, void* y, void* pre, void* ws,
                            hipStream_t st) {
  if (a.m == 0) return hipSuccess;
  return a.bf16 ? gated_fwd<bf16_t>(a, x, w, bias, y, pre, ws, st) : gated_fwd<float>(a, x, w, bias, y, pre, ws, st);
}

size_t gated_bwd_ws_bytes(const GatedArgs& a) { return gated_bwd_layout(a).total; }

hipError_t launch_gated_bwd(const GatedArgs& a, const void* x, const void* w, const void* pre, const void* dy, void* dx,
                            void* dw, void* db, void* ws, hipStream_t st) {
  return a.bf16 ? gated_bwd<bf16_t>(a, x, w, pre, dy, dx, dw, db, ws, st) : gated_bwd<float>(a, x, w, pre, dy, dx, dw, db, ws, st);
}

}  // namespace bsa
