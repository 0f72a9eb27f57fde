// Gated map and its gradients: with [g | u] = x w^T + bias, w [2n, k],
//   y = act(g) u;   dg = dy u act'(g), du = dy act(g), dz = [dg | du], dx = dz w, dw = dz^T x,
//   db = sum dz.
// The forward is one product whose workgroups hold the same columns of both maps, so g and u meet in
// registers (dense_product.hpp) and only y is written (and, for the backward, [g | u]). The backward's two
// products are the affine map's over the 2n columns of dz.
// Bound by the matrix cores from a few hundred rows on, below by the weight's bytes.
#include "dense_product.hpp"

namespace bsa {
namespace {

// 32 column pieces x 8 rows at a time; workgroup (x, y) takes rows y rpg .. and leaves the sums of its
// columns of dg and du in part[y][2n] (NULL: not formed).
template <typename T>
__global__ void __launch_bounds__(256) gated_dz_kernel(const T* __restrict__ dy, long long lddy, const T* __restrict__ pre,
                                                       int act, long long m, int n, long long rpg, T* __restrict__ dz,
                                                       float* __restrict__ part) {
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
      T* const p = dz + r * 2 * n + c;
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

// ---- host ----

// The forward's product has 2n columns.
Plan fwd_plan(const GatedArgs& a) { return plan_product(a.bf16, a.m, 2 * a.n, a.k); }

LinearArgs rows_of(const GatedArgs& a) { return LinearArgs{a.m, a.k, 2 * a.n, a.bf16, kActNone, a.ldx, a.ldw, 0, 0, 2LL * a.n}; }

struct GatedBwdWs {
  size_t dz, dbp, rest, total;
  int P;
  long long rpg;
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
  L.dz = put(esz * (size_t)a.m * 2 * a.n);
  L.dbp = put(sizeof(float) * (size_t)L.P * 2 * a.n);
  L.rest = put(linear_bwd_ws_bytes(rows_of(a)));
  L.total = off;
  return L;
}

template <typename T>
hipError_t gated_fwd(const GatedArgs& a, const void* x, const void* w, const void* bias, void* y, void* pre, void* ws,
                     hipStream_t st) {
  const Epi<T> o{a.m, a.n, (T*)y, a.ldy, (const T*)bias, nullptr, 0, (T*)pre, a.act, nullptr};
  const Mat<T> mx{(const T*)x, a.ldx, a.m, a.k}, mw{(const T*)w, a.ldw, 2LL * a.n, a.k};
  if (few_rows_ok(a.m, a.k)) return few_rows<T, 2>(mx, mw, a.m, a.n, a.k, o, st);
  return product<T, false, false, true>(mx, mw, a.m, a.n, a.k, fwd_plan(a), (float*)ws, o, st);
}

template <typename T>
hipError_t gated_bwd(const GatedArgs& a, const void* x, const void* w, const void* pre, const void* dy, void* dx, void* dw,
                     void* db, void* ws, hipStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  const GatedBwdWs L = gated_bwd_layout(a);
  char* const c = (char*)ws;
  T* const dz = (T*)(c + L.dz);
  float* const dbp = db && a.m > 0 ? (float*)(c + L.dbp) : nullptr;
  if (a.m > 0) {
    gated_dz_kernel<T><<<dim3((a.n + 32 * E - 1) / (32 * E), L.P), 256, 0, st>>>((const T*)dy, a.lddy, (const T*)pre, a.act,
                                                                                 a.m, a.n, L.rpg, dz, dbp);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // without rows this also clears db
  const hipError_t e = launch_linear_bwd(rows_of(a), x, w, nullptr, dz, dx, dw, a.m > 0 ? nullptr : db, c + L.rest, st);
  if (e != hipSuccess || !dbp) return e;
  db_sum_kernel<T><<<(2 * a.n + 63) / 64, 1024, 0, st>>>(dbp, L.P, 2 * a.n, (T*)db);
  return hipGetLastError();
}

}  // namespace

size_t gated_fwd_ws_bytes(const GatedArgs& a) {
  return few_rows_ok(a.m, a.k) ? 0 : plan_bytes(fwd_plan(a), a.m, 2LL * a.n);
}

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
