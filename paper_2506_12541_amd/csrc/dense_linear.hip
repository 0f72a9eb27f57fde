// Affine map with an epilogue and its gradients:
//   z = x w^T + bias, y = act(z) + res;   dz = dy act'(z), dx = dz w, dw = dz^T x, db = sum dz.
// The three products (dense_product.hpp) have x and w of the forward and dz of dx in row form, w of dx and
// both operands of dw in column form.
#include "dense_product.hpp"

namespace bsa {
namespace {

// ---- dz = dy act'(z) and the partial column sums of dz ----

// 32 column pieces x 8 rows at a time; workgroup (x, y) takes rows y rpg .. and leaves the sums
// of its columns in part[y][n]. dz == NULL: only the sums; part == NULL: only dz.
template <typename T>
__global__ void __launch_bounds__(256) dz_kernel(const T* __restrict__ dy, long long lddy, const T* __restrict__ pre,
                                                 int act, long long m, int n, long long rpg, T* __restrict__ dz,
                                                 float* __restrict__ part) {
  constexpr int E = 16 / (int)sizeof(T);
  __shared__ float red[8][32 * E + 4];
  const int cx = threadIdx.x & 31, ry = threadIdx.x >> 5;
  const int c = (blockIdx.x * 32 + cx) * E;
  const long long r0 = blockIdx.y * rpg, r1 = r0 + rpg < m ? r0 + rpg : m;
  float s[E];
#pragma unroll
  for (int e = 0; e < E; ++e) s[e] = 0.f;
  if (c < n) {
    const Mat<T> my{dy, lddy, m, n}, mz{pre, n, m, n};
#pragma unroll 2
    for (long long r = r0 + ry; r < r1; r += 8) {
      float v[E];
      unpack16<T>(load_piece(my, r, c), v);
      if (dz) {
        float z[E];
        unpack16<T>(load_piece(mz, r, c), z);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= act_slope<T>(z[e], act);
        T* p = dz + r * n + c;
        if (c + E <= n)
          store16u(p, pack16<T>(v));
        else
          store_partial(p, pack16<T>(v), n - c);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) s[e] += v[e];
    }
  }
  if (!part) return;
#pragma unroll
  for (int e = 0; e < E; ++e) red[ry][cx * E + e] = s[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 32 * E; i += 256) {
    float v = red[0][i];
#pragma unroll
    for (int k = 1; k < 8; ++k) v += red[k][i];
    const int col = blockIdx.x * 32 * E + i;
    if (col < n) part[(long long)blockIdx.y * n + col] = v;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) fill_zero_kernel(T* p, long long n) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += 256LL * gridDim.x) p[i] = from_f32<T>(0.f);
}

// ---- host ----

struct LinBwdWs {
  size_t dz, dbp, part, total;
  Plan dx, dw;
  int P;
  long long rpg;
};
LinBwdWs linear_bwd_layout(const LinearArgs& a) {
  LinBwdWs L{};
  const size_t esz = a.bf16 ? 2 : 4;
  const int E = 16 / (int)esz;
  size_t off = 0;
  auto put = [&](size_t b) { const size_t o = off; off += align256(b); return o; };
  L.dx = plan_product(a.bf16, a.m, a.k, a.n);
  L.dw = plan_product(a.bf16, a.n, a.k, a.m);
  // row groups of the dz pass: about 1024 workgroups, at least 32 rows each
  const long long gx = (a.n + 32 * E - 1) / (32 * E);
  long long P = std::min<long long>(std::max<long long>(1024 / gx, 1), (a.m + 31) / 32);
  P = std::max<long long>(std::min<long long>(P, 256), 1);
  L.rpg = (a.m + P - 1) / P;
  L.P = (int)(L.rpg ? (a.m + L.rpg - 1) / L.rpg : 1);
  L.dz = put(a.act == kActNone ? 0 : esz * (size_t)a.m * a.n);
  L.dbp = put(sizeof(float) * (size_t)L.P * a.n);
  L.part = put(std::max(plan_bytes(L.dx, a.m, a.k), plan_bytes(L.dw, a.n, a.k)));
  L.total = off;
  return L;
}

template <typename T>
hipError_t linear_fwd(const LinearArgs& a, const void* x, const void* w, const void* bias, const void* res, void* y,
                      void* pre, void* ws, hipStream_t st) {
  const Epi<T> o{a.m, a.n, (T*)y, a.ldy, (const T*)bias, (const T*)res, a.ldr, (T*)pre, a.act, nullptr};
  const Mat<T> mx{(const T*)x, a.ldx, a.m, a.k}, mw{(const T*)w, a.ldw, a.n, a.k};
  if (few_rows_ok(a.m, a.k)) return few_rows<T, 1>(mx, mw, a.m, a.n, a.k, o, st);
  return product<T, false, false>(mx, mw, a.m, a.n, a.k, plan_product(a.bf16, a.m, a.n, a.k), (float*)ws, o, st);
}

template <typename T>
hipError_t zero(T* p, long long n, hipStream_t st) {
  fill_zero_kernel<T><<<(unsigned)std::min<long long>((n + 255) / 256, 1 << 16), 256, 0, st>>>(p, n);
  return hipGetLastError();
}

template <typename T>
hipError_t linear_bwd(const LinearArgs& a, const void* x, const void* w, const void* pre, const void* dy, void* dx,
                      void* dw, void* db, void* ws, hipStream_t st) {
  if (a.m == 0) {   // empty sums
    hipError_t e = hipSuccess;
    if (dw) e = zero((T*)dw, (long long)a.n * a.k, st);
    if (e == hipSuccess && db) e = zero((T*)db, a.n, st);
    return e;
  }
  constexpr int E = 16 / (int)sizeof(T);
  const LinBwdWs L = linear_bwd_layout(a);
  char* c = (char*)ws;
  T* const dz = a.act == kActNone ? nullptr : (T*)(c + L.dz);
  float* const dbp = db ? (float*)(c + L.dbp) : nullptr;
  if (dz || dbp) {
    dz_kernel<T><<<dim3((a.n + 32 * E - 1) / (32 * E), L.P), 256, 0, st>>>((const T*)dy, a.lddy, (const T*)pre, a.act,
                                                                           a.m, a.n, L.rpg, dz, dbp);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  Mat<T> mz{dz ? dz : (const T*)dy, dz ? a.n : a.lddy, a.m, a.n};
  const int k = std::max(a.k, a.readable_k);
  if (dx) {
    Epi<T> o{a.m, a.k, (T*)dx, a.k, nullptr, nullptr, 0, nullptr, kActNone, nullptr};
    hipError_t e = product<T, false, true>(mz, Mat<T>{(const T*)w, a.ldw, a.n, k}, a.m, a.k, a.n, L.dx,
                                             (float*)(c + L.part), o, st);
    if (e != hipSuccess) return e;
  }
  if (dw) {
    Epi<T> o{a.n, a.k, (T*)dw, a.k, nullptr, nullptr, 0, nullptr, kActNone, nullptr};
    mz.cols = std::max(a.n, a.readable_n);
    hipError_t e = product<T, true, true>(mz, Mat<T>{(const T*)x, a.ldx, a.m, k}, a.n, a.k, a.m, L.dw,
                                          (float*)(c + L.part), o, st);
    if (e != hipSuccess) return e;
  }
  if (db) {
    db_sum_kernel<T><<<(a.n + 63) / 64, 1024, 0, st>>>(dbp, L.P, a.n, (T*)db);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace

size_t linear_fwd_ws_bytes(const LinearArgs& a) {
  return few_rows_ok(a.m, a.k) ? 0 : plan_bytes(plan_product(a.bf16, a.m, a.n, a.k), a.m, a.n);
}

hipError_t launch_linear_fwd(const LinearArgs& a, const void* x, const void* w, const void* bias, const void* res,
                             void* y, void* pre, void* ws, hipStream_t st) {
  if (a.m == 0) return hipSuccess;
  return a.bf16 ? linear_fwd<bf16_t>(a, x, w, bias, res, y, pre, ws, st)
                : linear_fwd<float>(a, x, w, bias, res, y, pre, ws, st);
}

size_t linear_bwd_ws_bytes(const LinearArgs& a) { return linear_bwd_layout(a).total; }

hipError_t launch_linear_bwd(const LinearArgs& a, const void* x, const void* w, const void* pre, const void* dy,
                             void* dx, void* dw, void* db, void* ws, hipStream_t st) {
  return a.bf16 ? linear_bwd<bf16_t>(a, x, w, pre, dy, dx, dw, db, ws, st)
                : linear_bwd<float>(a, x, w, pre, dy, dx, dw, db, ws, st);
}

}  // namespace bsa
