// Rotary positions of queries and keys, with the norm of each head in the same pass:
//   n = x rstd gain, rstd = 1 / sqrt(mean(x^2) + eps)   (without a gain: n = x),
//   y_a = m (n_a cos t - n_b sin t), y_b = m (n_a sin t + n_b cos t), t = position * freq,
// for the pairs (a, b) of the first `rot` values of a head; the rest of n passes. Backward:
//   dn = the pairs turned back, times m; dgain = sum dn x rstd, dx = rstd (dn gain - x rstd mean(dn gain x rstd)).
//
// A lane holds two pieces of 16 bytes of a head that rotate with each other (or two of its rest), so a pair
// never leaves its lane; a power of two of lanes holds a head and joins its norm's sum. Pieces that end
// inside a part of the head are loaded by element. A workgroup takes R rows of the tensors, forms the
// angles of a row once for all heads and keeps their cosines and sines in LDS.
#include <algorithm>

#include "common.hpp"
#include "dense.hpp"
#include "dense_common.hpp"

namespace bsa {
namespace {

// cos t and sin t of an angle in 64 bits: t - k pi / 2 in two steps (pi / 2 as the sum of two doubles; off by
// 2^-53 |t|), then the Taylor polynomials on [-pi / 4, pi / 4], whose next terms are 2e-9. Angles of a far
// position need the 64 bits: at 2^20 radians a float32 angle is off by 0.06. From 2^52 radians on (a position
// that is no position) the remainder means nothing and is taken as 0; infinities and NaN give NaN.
__device__ __forceinline__ void cos_sin(double t, float& c, float& s) {
  const double k = __builtin_rint(t * 0.63661977236758134);
  double r = __builtin_fma(-k, 1.5707963267948966, t);
  r = __builtin_fma(-k, 6.123233995736766e-17, r);
  float x = (float)r;
  x = fabsf(x) > 0.8f ? 0.f : x;
  const float q = x * x;
  float a = fmaf(q, 2.7557319e-6f, -1.9841270e-4f);
  a = fmaf(q, a, 8.3333333e-3f);
  a = fmaf(q, a, -1.6666667e-1f);
  a = fmaf(x * q, a, x);
  float b = fmaf(q, -2.7557319e-7f, 2.4801587e-5f);
  b = fmaf(q, b, -1.3888889e-3f);
  b = fmaf(q, b, 4.1666667e-2f);
  b = fmaf(q, b, -0.5f);
  b = fmaf(q, b, 1.f);
  // k mod 4, from its own bits (k is a whole number)
  const int quad = (int)(k - 4.0 * __builtin_floor(k * 0.25));
  const float u = quad & 1 ? a : b, v = quad & 1 ? b : a;
  c = quad == 1 || quad == 2 ? -u : u;
  s = quad & 2 ? -v : v;
}

struct RotParts {          // of queries and of keys
  const void* x;           // NULL: not needed (backward without a norm)
  const void* dy;
  void* out;
  const float* gain;       // NULL: no norm
  long long x_row, x_head, dy_row, dy_head, out_row, out_head;
  int heads;
};

struct RotP {
  RotParts part[2];
  const void* pos;
  const double* freq;
  long long rows;
  int hd, rot, half, axes, per_axis;   // half = rot / 2 pairs, per_axis of them for each axis
  int R, G, lrot;                      // rows of a workgroup's step; lanes of a head; lanes that rotate
  int pitch;                           // floats between the LDS rows of cosines
  bool fpos;
  float eps, mag;
  float* sums;                         // [workgroups][2][hd] partial gain gradients, or NULL
};

constexpr int kRotLds = 4096;          // cosines, and sines, that a workgroup holds

// The elements of a head that lane l of its lanes holds: [a, a + na) and [b, b + nb). INTER: neighbours
// rotate with each other.
struct LaneAt {
  int a, na, b, nb;
  bool turns;
};
template <int E, bool INTER>
__device__ __forceinline__ LaneAt lane_at(const RotP& p, int l) {
  LaneAt t;
  t.turns = l < p.lrot;
  if (t.turns) {
    t.a = INTER ? 2 * E * l : E * l;
    t.na = INTER ? p.rot - t.a : p.half - t.a;
    t.b = INTER ? t.a + E : p.half + t.a;
    t.nb = INTER ? p.rot - t.b : t.na;
  } else {
    t.a = p.rot + 2 * E * (l - p.lrot);
    t.na = p.hd - t.a;
    t.b = t.a + E;
    t.nb = p.hd - t.b;
  }
  t.na = max(0, min(t.na, E));
  t.nb = max(0, min(t.nb, E));
  return t;
}

template <typename T>
__device__ __forceinline__ void load_n(const T* p, int n, float* v) {
  constexpr int E = 16 / (int)sizeof(T);
  unpack16<T>(n == E ? load16u(p) : n > 0 ? load_partial(p, n) : make_uint4(0, 0, 0, 0), v);
}
template <typename T>
__device__ __forceinline__ void store_n(T* p, int n, const float* v) {
  constexpr int E = 16 / (int)sizeof(T);
  if (n == E)
    store16u(p, pack16<T>(v));
  else if (n > 0)
    store_partial(p, pack16<T>(v), n);
}

// Turns the lane's pairs by its E angles (sign -1: back).
template <int E, bool INTER>
__device__ __forceinline__ void turn(float (&a)[E], float (&b)[E], const float* c, const float* s, float sign) {
  auto pair = [&](float& u, float& v, int i) {
    const float si = sign * s[i], t = u * c[i] - v * si;
    v = u * si + v * c[i];
    u = t;
  };
  if constexpr (INTER) {
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      pair(a[e], a[e + 1], e / 2);
      pair(b[e], b[e + 1], E / 2 + e / 2);
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) pair(a[e], b[e], e);
  }
}

// The sum over the G lanes of a head.
__device__ __forceinline__ float head_sum(float x, int G) {
  for (int o = G >> 1; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

template <typename T, bool INTER, bool BWD>
__global__ void __launch_bounds__(256) rotary_kernel(RotP p) {
  constexpr int E = 16 / (int)sizeof(T);
  __shared__ __attribute__((aligned(16))) float cs[kRotLds], sn[kRotLds];
  const int l = threadIdx.x & (p.G - 1), slot = threadIdx.x / p.G, slots = 256 / p.G;
  const LaneAt at = lane_at<E, INTER>(p, l);
  float sum[2][2][E];
  if constexpr (BWD) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < E; ++e) sum[h][0][e] = sum[h][1][e] = 0.f;
  }
  for (long long r0 = (long long)blockIdx.x * p.R; r0 < p.rows; r0 += (long long)gridDim.x * p.R) {
    const int R = (int)min((long long)p.R, p.rows - r0);
    __syncthreads();      // the previous step's angles have been read
    for (int i = threadIdx.x; i < R * p.pitch; i += 256) {
      const int r = i / p.pitch, k = i - r * p.pitch;
      if (k >= p.half) {      // zeros behind a row: what a lane turns there stays 0
        cs[i] = sn[i] = 0.f;
        continue;
      }
      const long long w = (r0 + r) * p.axes + (p.axes == 1 ? 0 : k / p.per_axis);
      const double x = p.fpos ? (double)((const float*)p.pos)[w] : (double)((const int*)p.pos)[w];
      float c, s;
      cos_sin(x * p.freq[k], c, s);
      cs[i] = p.mag * c;
      sn[i] = p.mag * s;
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const RotParts& t = p.part[h];
      const bool norm = t.gain;
      float ga[E], gb[E];
      if (norm) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          ga[e] = e < at.na ? t.gain[at.a + e] : 0.f;
          gb[e] = e < at.nb ? t.gain[at.b + e] : 0.f;
        }
      }
      // the lanes of a head leave the loop together
      for (int i = slot; i < R * t.heads; i += slots) {
        const int r = i / t.heads, head = i - r * t.heads;
        const long long row = r0 + r;
        float c[E], s[E];
        if (at.turns) {
#pragma unroll
          for (int e = 0; e < E; e += 4) {
            *reinterpret_cast<f32x4*>(c + e) = *reinterpret_cast<const f32x4*>(&cs[r * p.pitch + E * l + e]);
            *reinterpret_cast<f32x4*>(s + e) = *reinterpret_cast<const f32x4*>(&sn[r * p.pitch + E * l + e]);
          }
        }
        const T* const x = (const T*)t.x + row * t.x_row + head * t.x_head;
        T* const out = (T*)t.out + row * t.out_row + head * t.out_head;
        float a[E], b[E];
        if constexpr (!BWD) {
          load_n(x + at.a, at.na, a);
          load_n(x + at.b, at.nb, b);
          if (norm) {
            float q = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) q = fmaf(a[e], a[e], fmaf(b[e], b[e], q));
            const float rstd = 1.0f / sqrtf(head_sum(q, p.G) / p.hd + p.eps);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              a[e] *= rstd * ga[e];
              b[e] *= rstd * gb[e];
            }
          }
          if (at.turns) turn<E, INTER>(a, b, c, s, 1.f);
        } else {
          const T* const dy = (const T*)t.dy + row * t.dy_row + head * t.dy_head;
          load_n(dy + at.a, at.na, a);
          load_n(dy + at.b, at.nb, b);
          float xa[E], xb[E];
          if (norm) {
            load_n(x + at.a, at.na, xa);
            load_n(x + at.b, at.nb, xb);
          }
          if (at.turns) turn<E, INTER>(a, b, c, s, -1.f);
          if (norm) {
            float q = 0.f, m = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
              q = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], q));
              m = fmaf(a[e] * ga[e], xa[e], fmaf(b[e] * gb[e], xb[e], m));
            }
            const float rstd = 1.0f / sqrtf(head_sum(q, p.G) / p.hd + p.eps);
            m = head_sum(m, p.G) / p.hd * rstd;       // mean(dn gain xhat)
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float ua = xa[e] * rstd, ub = xb[e] * rstd;
              sum[h][0][e] = fmaf(a[e], ua, sum[h][0][e]);
              sum[h][1][e] = fmaf(b[e], ub, sum[h][1][e]);
              a[e] = rstd * (a[e] * ga[e] - ua * m);
              b[e] = rstd * (b[e] * gb[e] - ub * m);
            }
          }
        }
        store_n(out + at.a, at.na, a);
        store_n(out + at.b, at.nb, b);
      }
    }
  }
  if constexpr (BWD) {
    if (!p.sums) return;
    // the sums of the workgroup's heads, in order
    __shared__ float red[256][2 * E + 1];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        red[threadIdx.x][e] = sum[h][0][e];
        red[threadIdx.x][E + e] = sum[h][1][e];
      }
      __syncthreads();
      for (int i = threadIdx.x; i < p.G * 2 * E; i += 256) {
        const int lane = i / (2 * E), e = i % (2 * E);
        const LaneAt w = lane_at<E, INTER>(p, lane);
        float v = 0.f;
        for (int s = 0; s < slots; ++s) v += red[s * p.G + lane][e];
        float* const to = p.sums + ((long long)blockIdx.x * 2 + h) * p.hd;
        if (e < E && e < w.na) to[w.a + e] = v;
        if (e >= E && e - E < w.nb) to[w.b + e - E] = v;
      }
    }
  }
}

// dgain = sum of the workgroups' partial sums, wave w takes every 16th in turn; columns [0, hd) of the queries,
// then of the keys.
__global__ void __launch_bounds__(1024) rotary_gain_kernel(const float* __restrict__ part, int P, int hd, float* dgq, float* dgk) {
  __shared__ float red[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < 2 * hd) {
#pragma unroll 8
    for (int i = w; i < P; i += 16) s += part[(long long)i * 2 * hd + c];
  }
  red[w][lane] = s;
  __syncthreads();
  if (w == 0 && c < 2 * hd) {
#pragma unroll
    for (int k = 1; k < 16; ++k) s += red[k][lane];
    float* const to = c < hd ? dgq : dgk;
    if (to) to[c < hd ? c : c - hd] = s;
  }
}

// ---- host ----

struct RotPlan {
  int E, R, G, lrot, pitch;
  unsigned grid;
};
// Workgroups of the backward with a norm at most: each leaves a row of partial sums.
constexpr int kRotSums = 1024;

RotPlan rot_plan(const RotaryArgs& a, bool sums) {
  RotPlan p;
  p.E = a.bf16 ? 8 : 4;
  const int half = a.rot / 2;
  p.lrot = (half + p.E - 1) / p.E;
  const int lanes = p.lrot + (a.hd - a.rot + 2 * p.E - 1) / (2 * p.E);
  p.G = 1;
  while (p.G < lanes) p.G *= 2;
  p.pitch = p.lrot * p.E;
  // four heads or more for every lane, while that leaves 512 workgroups
  const int slots = 256 / p.G, heads = a.heads + a.kv_heads;
  long long R = std::max(1, std::min((4 * slots + heads - 1) / heads, kRotLds / p.pitch));
  R = std::max<long long>(std::min(R, a.rows / 512), 1);
  p.R = (int)R;
  p.grid = (unsigned)std::min<long long>((a.rows + R - 1) / R, sums ? kRotSums : 1 << 20);
  return p;
}

template <bool BWD>
hipError_t run(const RotaryArgs& a, RotP& p, const RotPlan& l, hipStream_t st) {
  if (a.bf16)
    a.interleaved ? rotary_kernel<bf16_t, true, BWD><<<l.grid, 256, 0, st>>>(p) : rotary_kernel<bf16_t, false, BWD><<<l.grid, 256, 0, st>>>(p);
  else
    a.interleaved ? rotary_kernel<float, true, BWD><<<l.grid, 256, 0, st>>>(p) : rotary_kernel<float, false, BWD><<<l.grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

RotP params(const RotaryArgs& a, const RotPlan& l, const void* pos, const double* freq) {
  RotP p{};
  p.pos = pos;
  p.freq = freq;
  p.rows = a.rows;
  p.hd = a.hd;
  p.rot = a.rot;
  p.half = a.rot / 2;
  p.axes = a.axes;
  p.per_axis = p.half / a.axes;
  p.R = l.R;
  p.G = l.G;
  p.lrot = l.lrot;
  p.pitch = l.pitch;
  p.fpos = a.fpos;
  p.eps = a.eps;
  p.mag = a.mag;
  return p;
}

}  // namespace

hipError_t launch_rotary_fwd(const RotaryArgs& a, const void* q, const void* k, const void* pos, const double* freq,
                             const float* gain_q, const float* gain_k, void* out_q, void* out_k, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const RotPlan l = rot_plan(a, false);
  RotP p = params(a, l, pos, freq);
  p.part[0] = RotParts{q, nullptr, out_q, gain_q, a.q_row, a.q_head, 0, 0, a.oq_row, a.oq_head, a.heads};
  p.part[1] = RotParts{k, nullptr, out_k, gain_k, a.k_row, a.k_head, 0, 0, a.ok_row, a.ok_head, a.kv_heads};
  return run<false>(a, p, l, st);
}

size_t rotary_bwd_ws_bytes(const RotaryArgs& a) { return sizeof(float) * 2 * a.hd * (size_t)rot_plan(a, true).grid; }

hipError_t launch_rotary_bwd(const RotaryArgs& a, const void* q, const void* k, const void* pos, const double* freq,
                             const float* gain_q, const float* gain_k, const void* dy_q, const void* dy_k, void* dq, void* dk,
                             float* dgain_q, float* dgain_k, void* ws, hipStream_t st) {
  const bool sums = gain_q || gain_k;
  const RotPlan l = rot_plan(a, sums);
  if (a.rows > 0) {
    RotP p = params(a, l, pos, freq);
    p.part[0] = RotParts{q, dy_q, dq, gain_q, a.q_row, a.q_head, a.dq_row, a.dq_head, a.oq_row, a.oq_head, a.heads};
    p.part[1] = RotParts{k, dy_k, dk, gain_k, a.k_row, a.k_head, a.dk_row, a.dk_head, a.ok_row, a.ok_head, a.kv_heads};
    p.sums = sums ? (float*)ws : nullptr;
    const hipError_t e = run<true>(a, p, l, st);
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;
  rotary_gain_kernel<<<(2 * a.hd + 63) / 64, 1024, 0, st>>>((const float*)ws, a.rows > 0 ? (int)l.grid : 0, a.hd, dgain_q, dgain_k);
  return hipGetLastError();
}

}  // namespace bsa
