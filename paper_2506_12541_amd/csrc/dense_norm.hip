// Layer norm, forward and backward:
//   y = xh gain + bias, xh = (x - mean) rstd, rstd = 1 / sqrt(var + eps) over the columns;
//   dx = rstd (g - mean(g) - xh mean(g xh)), g = dy gain;   dgain = sum dy xhat, dbias = sum dy
// over the rows. A row is held in registers by a group of L lanes (16, 64, 256 or 1024, NV
// 16-byte vectors a lane), so x is read once and the variance is the mean of squared
// deviations (no cancellation). Everything is bound by HBM: the forward reads x and writes y,
// the backward reads x and dy and writes dx; statistics and sums are float32.
#include <algorithm>

#include "common.hpp"
#include "dense.hpp"
#include "dense_common.hpp"

namespace bsa {
namespace {

// Sum over the 16 lanes of a lane group, in every lane (row rotations: no LDS traffic).
template <int CTRL>
__device__ __forceinline__ float row_rot(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum16(float x) {
  x += row_rot<0x128>(x);
  x += row_rot<0x124>(x);
  x += row_rot<0x122>(x);
  return x + row_rot<0x121>(x);
}

// Sums over a group of L lanes of NS values at once; groups wider than a wave meet in LDS
// (red: NS floats per wave; every wave of the workgroup calls this together).
template <int L, int NS>
__device__ __forceinline__ void group_sum(float (&s)[NS], float* red) {
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    s[i] = sum16(s[i]);
    if constexpr (L >= 64) s[i] = col_sum(s[i]);
  }
  if constexpr (L > 64) {
    constexpr int W = L / 64;
    const int wid = threadIdx.x >> 6, w0 = wid / W * W;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < NS; ++i) red[wid * NS + i] = s[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      s[i] = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) s[i] += red[(w0 + w) * NS + i];
    }
    __syncthreads();
  }
}

template <typename T> struct NormVec {
  static constexpr int E = 16 / (int)sizeof(T);
};

// Vector idx of a row (columns [E idx, E idx + E)); columns past the row are zero.
template <typename T>
__device__ __forceinline__ uint4 norm_load(const T* row, int idx, int cols) {
  constexpr int E = NormVec<T>::E;
  const int c = idx * E;
  if (c + E <= cols) return load16u(row + c);
  uint4 v = make_uint4(0, 0, 0, 0);
  if (c < cols) v = load_partial(row + c, cols - c);
  return v;
}
template <typename T>
__device__ __forceinline__ void norm_store(T* row, int idx, int cols, const float* v) {
  constexpr int E = NormVec<T>::E;
  const int c = idx * E;
  if (c + E <= cols)
    store16u(row + c, pack16<T>(v));
  else if (c < cols)
    store_partial(row + c, pack16<T>(v), cols - c);
}
// Gain or bias of vector idx's columns (fill: without p, and behind the row).
template <int E>
__device__ __forceinline__ void norm_params(const float* p, int idx, int cols, float fill, float* out) {
#pragma unroll
  for (int e = 0; e < E; e += 4) {
    const int c = idx * E + e;
    float4 v = make_float4(fill, fill, fill, fill);
    if (p) {
      if (c + 4 <= cols) {
        __builtin_memcpy(&v, p + c, 16);
      } else {
        if (c < cols) v.x = p[c];
        if (c + 1 < cols) v.y = p[c + 1];
        if (c + 2 < cols) v.z = p[c + 2];
      }
    }
    out[e] = v.x;
    out[e + 1] = v.y;
    out[e + 2] = v.z;
    out[e + 3] = v.w;
  }
}

template <typename T, int L, int NV, int NT>
__global__ void __launch_bounds__(NT) layernorm_fwd_kernel(const T* __restrict__ x, const float* __restrict__ gain,
                                                           const float* __restrict__ bias, NormArgs a,
                                                           T* __restrict__ y, float* __restrict__ mean,
                                                           float* __restrict__ rstd) {
  constexpr int E = NormVec<T>::E, GPW = NT / L;   // groups (rows at a time) per workgroup
  __shared__ float red[2 * NT / 64];
  const int l = threadIdx.x % L;
  // gain and bias stay in registers over the rows while they are few (wide rows: read again)
  constexpr bool KEEP = NV * E <= 16;
  float g[KEEP ? NV : 1][E], b[KEEP ? NV : 1][E];
  if constexpr (KEEP) {
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      norm_params<E>(gain, l + L * t, a.cols, 1.f, g[t]);
      norm_params<E>(bias, l + L * t, a.cols, 0.f, b[t]);
    }
  }
  // every group of a workgroup makes the same number of steps (they meet in group_sum); the next
  // row is on its way while this one is reduced
  const long long step = (long long)gridDim.x * GPW;
  uint4 u[NV];
  auto fetch = [&](long long row) {
#pragma unroll
    for (int t = 0; t < NV; ++t) u[t] = row < a.rows ? norm_load(x + row * a.ldx, l + L * t, a.cols) : make_uint4(0, 0, 0, 0);
  };
  fetch((long long)blockIdx.x * GPW + threadIdx.x / L);
  for (long long r0 = (long long)blockIdx.x * GPW; r0 < a.rows; r0 += step) {
    const long long row = r0 + threadIdx.x / L;
    const bool on = row < a.rows;
    float v[NV][E];
    float s[1] = {0.f};
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      unpack16<T>(u[t], v[t]);
#pragma unroll
      for (int e = 0; e < E; ++e) s[0] += v[t][e];
    }
    if (r0 + step < a.rows) fetch(row + step);
    group_sum<L>(s, red);
    const float mu = s[0] / (float)a.cols;
    // the deviations' own mean is the rounding error of mu: it is taken out of them again, so
    // rows far from zero lose nothing
    float q[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < NV; ++t)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[t][e] = (l + L * t) * E + e < a.cols ? v[t][e] - mu : 0.f;
        q[0] += v[t][e];
        q[1] = fmaf(v[t][e], v[t][e], q[1]);
      }
    group_sum<L>(q, red);
    const float d = q[0] / (float)a.cols;
    const float var = q[1] / (float)a.cols - d * d;
    const float rs = 1.0f / sqrtf((var < 0.f ? 0.f : var) + a.eps);   // NaN stays (a row that is not finite)
    if (on) {
#pragma unroll
      for (int t = 0; t < NV; ++t) {
        constexpr int K = KEEP ? 1 : 0;
        if constexpr (!KEEP) {
          norm_params<E>(gain, l + L * t, a.cols, 1.f, g[0]);
          norm_params<E>(bias, l + L * t, a.cols, 0.f, b[0]);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) v[t][e] = fmaf((v[t][e] - d) * rs, g[K * t][e], b[K * t][e]);
        norm_store(y + row * a.ldy, l + L * t, a.cols, v[t]);
      }
      if (l == 0) {
        mean[row] = fabsf(mu) < __builtin_huge_valf() ? mu + d : mu;   // infinite: d is NaN
        rstd[row] = rs;
      }
    }
  }
}

// A row is read whole before it is written: dx may be x or dy.
// Workgroup b takes rows b GPW .. in steps of the grid; the column sums of its rows go to
// part[b][2][cols] (dgain, dbias): each lane sums its own columns over its rows, then the
// groups are added in order through LDS.
template <typename T, int L, int NV, int NT>
__global__ void __launch_bounds__(NT) layernorm_bwd_kernel(const T* x, const float* __restrict__ gain,
                                                           const float* __restrict__ mean,
                                                           const float* __restrict__ rstd, const T* dy, NormArgs a, T* dx,
                                                           float* __restrict__ part, float* __restrict__ part_b,
                                                           long long part_ld) {
  constexpr int E = NormVec<T>::E, GPW = NT / L;
  __shared__ __attribute__((aligned(16))) float sums[GPW > 1 ? NT * 2 * E : 2 * NT / 64];
  const int l = threadIdx.x % L, grp = threadIdx.x / L;
  const float inv = 1.0f / (float)a.cols;
  float g[NV][E], ag[NV][E], ab[NV][E];
#pragma unroll
  for (int t = 0; t < NV; ++t) {
    norm_params<E>(gain, l + L * t, a.cols, 0.f, g[t]);
#pragma unroll
    for (int e = 0; e < E; ++e) ag[t][e] = ab[t][e] = 0.f;
  }
  for (long long r0 = (long long)blockIdx.x * GPW; r0 < a.rows; r0 += (long long)gridDim.x * GPW) {
    const long long row = r0 + grp;
    const bool on = row < a.rows;
    uint4 xu[NV], du[NV];
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      xu[t] = on ? norm_load(x + row * a.ldx, l + L * t, a.cols) : make_uint4(0, 0, 0, 0);
      du[t] = on ? norm_load(dy + row * a.lddy, l + L * t, a.cols) : make_uint4(0, 0, 0, 0);
    }
    const float mu = on ? mean[row] : 0.f, rs = on ? rstd[row] : 0.f;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      float xv[E], dv[E];
      unpack16<T>(xu[t], xv);
      unpack16<T>(du[t], dv);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        // columns past the row: gain and dy are zero there, so every term is
        const float xh = (xv[e] - mu) * rs, gd = dv[e] * g[t][e];
        s[0] += gd;
        s[1] = fmaf(gd, xh, s[1]);
        ag[t][e] = fmaf(dv[e], xh, ag[t][e]);
        ab[t][e] += dv[e];
      }
    }
    group_sum<L>(s, sums);
    const float m0 = s[0] * inv, m1 = s[1] * inv;
    if (on) {
#pragma unroll
      for (int t = 0; t < NV; ++t) {
        float xv[E], dv[E];
        unpack16<T>(xu[t], xv);
        unpack16<T>(du[t], dv);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float xh = (xv[e] - mu) * rs;
          xv[e] = rs * (fmaf(dv[e], g[t][e], -m0) - xh * m1);
        }
        norm_store(dx + row * a.lddx, l + L * t, a.cols, xv);
      }
    }
  }
  float* const pg = part + blockIdx.x * part_ld;
  float* const pb = part_b ? part_b + blockIdx.x * part_ld : nullptr;
#pragma unroll
  for (int t = 0; t < NV; ++t) {
    if constexpr (GPW > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        sums[(grp * 2 + 0) * L * E + l * E + e] = ag[t][e];
        sums[(grp * 2 + 1) * L * E + l * E + e] = ab[t][e];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < 2 * L * E; i += NT) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < GPW; ++k) s += sums[k * 2 * L * E + i];
        const int c = L * E * t + i % (L * E);
        if (c < a.cols) {
          if (i < L * E)
            pg[c] = s;
          else if (pb)
            pb[c] = s;
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int c = (l + L * t) * E + e;
        if (c < a.cols) {
          pg[c] = ag[t][e];
          if (pb) pb[c] = ab[t][e];
        }
      }
    }
  }
}

// dgain / dbias = sums over the P workgroups' rows of part [P][2][cols]; 64 columns per
// workgroup, wave w takes rows w, w + 16, ..., the waves' sums are added in order
__global__ void __launch_bounds__(1024) norm_colsum_kernel(const float* __restrict__ part, int P, int cols,
                                                           float* __restrict__ dgain, float* __restrict__ dbias) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  float* const out = blockIdx.y ? dbias : dgain;
  const float* p = part + (long long)blockIdx.y * cols;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int i = w; i < P; i += 16) s += p[(long long)i * 2 * cols + c];
  }
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < cols && out) {
#pragma unroll
    for (int k = 1; k < 16; ++k) s += red[k][lane];
    out[c] = s;
  }
}

__global__ void __launch_bounds__(256) norm_zero_kernel(float* a, float* b, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) {
    a[i] = 0.f;
    if (b) b[i] = 0.f;
  }
}

// Lanes per row and vectors per lane: the smallest group that holds the row. (The backward of bf16
// rows of 4097 to 8192 columns takes 1024 lanes with one vector: with four a lane its sums leave
// the registers.)
template <typename T, bool BWD, typename F>
hipError_t norm_dispatch(int cols, F f) {
  const int v = (cols + NormVec<T>::E - 1) / NormVec<T>::E;   // vectors of a row
  if (v <= 16) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
  if (v <= 32) return f(std::integral_constant<int, 16>{}, std::integral_constant<int, 2>{});
  if (v <= 64) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  if (v <= 128) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
  if (v <= 256) return f(std::integral_constant<int, 64>{}, std::integral_constant<int, 4>{});
  if (v <= 512) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 2>{});
  if constexpr (BWD && sizeof(T) == 2) {
    if (v <= 1024) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 1>{});
  } else {
    if (v <= 1024) return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 4>{});
  }
  if (v <= 2048) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 2>{});
  if constexpr (sizeof(T) == 4) {   // bf16 rows end at 4096 vectors
    if (v > 4096) return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 8>{});
  }
  return f(std::integral_constant<int, 1024>{}, std::integral_constant<int, 4>{});
}

// Workgroups of the backward: one for up to four steps of its groups (about 1 us each, where the
// second launch that joins several workgroups' sums costs 5 us), else up to one per CU.
template <typename T>
int norm_bwd_groups(const NormArgs& a) {
  int wgs = 0;
  (void)norm_dispatch<T, true>(a.cols, [&](auto L, auto) {
    constexpr int GPW = 1024 / decltype(L)::value;
    wgs = a.rows <= 4 * GPW ? 1 : (int)std::min<long long>((a.rows + GPW - 1) / GPW, 256);
    return hipSuccess;
  });
  return wgs;
}

template <typename T>
hipError_t norm_fwd(const NormArgs& a, const void* x, const float* gain, const float* bias, void* y, float* mean,
                    float* rstd, hipStream_t st) {
  return norm_dispatch<T, false>(a.cols, [&](auto L, auto NV) {
    constexpr int l = decltype(L)::value, nv = decltype(NV)::value, nt = l > 256 ? l : 256;
    const long long wgs = std::min<long long>((a.rows + nt / l - 1) / (nt / l), 256 * (2048 / nt));
    layernorm_fwd_kernel<T, l, nv, nt><<<(unsigned)wgs, nt, 0, st>>>((const T*)x, gain, bias, a, (T*)y, mean, rstd);
    return hipGetLastError();
  });
}

template <typename T>
hipError_t norm_bwd(const NormArgs& a, const void* x, const float* gain, const float* mean, const float* rstd,
                    const void* dy, void* dx, float* dgain, float* dbias, float* part, hipStream_t st) {
  const int wgs = norm_bwd_groups<T>(a);
  hipError_t e = norm_dispatch<T, true>(a.cols, [&](auto L, auto NV) {
    constexpr int l = decltype(L)::value, nv = decltype(NV)::value;
    if (wgs == 1)
      layernorm_bwd_kernel<T, l, nv, 1024><<<1, 1024, 0, st>>>((const T*)x, gain, mean, rstd, (const T*)dy, a, (T*)dx,
                                                               dgain, dbias, 0);
    else
      layernorm_bwd_kernel<T, l, nv, 1024><<<wgs, 1024, 0, st>>>((const T*)x, gain, mean, rstd, (const T*)dy, a,
                                                                 (T*)dx, part, part + a.cols, 2LL * a.cols);
    return hipGetLastError();
  });
  if (e != hipSuccess || wgs == 1) return e;
  norm_colsum_kernel<<<dim3((a.cols + 63) / 64, dbias ? 2 : 1), 1024, 0, st>>>(part, wgs, a.cols, dgain, dbias);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_layernorm_fwd(const NormArgs& a, const void* x, const float* gain, const float* bias, void* y,
                                float* mean, float* rstd, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  return a.bf16 ? norm_fwd<bf16_t>(a, x, gain, bias, y, mean, rstd, st)
                : norm_fwd<float>(a, x, gain, bias, y, mean, rstd, st);
}

size_t layernorm_bwd_ws_bytes(const NormArgs& a) {
  const int wgs = a.bf16 ? norm_bwd_groups<bf16_t>(a) : norm_bwd_groups<float>(a);
  return wgs > 1 ? sizeof(float) * 2 * (size_t)wgs * a.cols : 0;
}

hipError_t launch_layernorm_bwd(const NormArgs& a, const void* x, const float* gain, const float* mean,
                                const float* rstd, const void* dy, void* dx, float* dgain, float* dbias, void* ws,
                                hipStream_t st) {
  if (a.rows == 0) {   // empty sums
    norm_zero_kernel<<<(a.cols + 255) / 256, 256, 0, st>>>(dgain, dbias, a.cols);
    return hipGetLastError();
  }
  return a.bf16 ? norm_bwd<bf16_t>(a, x, gain, mean, rstd, dy, dx, dgain, dbias, (float*)ws, st)
                : norm_bwd<float>(a, x, gain, mean, rstd, dy, dx, dgain, dbias, (float*)ws, st);
}

}  // namespace bsa
