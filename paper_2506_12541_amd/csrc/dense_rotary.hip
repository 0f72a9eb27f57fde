// Rotary positions of queries and keys, with the norm of each head in the same pass:
//   n = x rstd gain, rstd = 1 / sqrt(mean(x^2) + eps)   (without a gain: n = x),
//   y_a = m (n_a cos t - n_b sin t), y_b = m (n_a sin t + n_b cos t), t = position * freq,
// for the pairs (a, b) of the first `rot` values of a head; the rest of n passes. Backward:
//   dn = the pairs turned back, times m; dgain = sum dn x rstd, dx = rstd (dn gain - x rstd mean(dn gain x rstd)).
//
// A lane holds two pieces of 16 bytes of a head that rotate with each other (or two of its rest), so a pair
// never leaves its lane; a power of two of lanes holds a head and joins its norm's sum. Pieces that end
// inside a part of the head are loaded by element. A wave takes R rows of the tensors (or some of the heads of
// few rows), forms the angles of a row once for all its heads, while its first pieces are on their way, and keeps their
// cosines and sines in LDS; waves share nothing, so no barrier holds them together.
// Bound by the bytes: 65536 rows of 8 + 8 heads of 64 (48 of them turn), bf16 with norms, the forward (268 MB) takes
// 56 us, the backward (403 MB) 86 and 5 to join the gains' gradients; a copy would take 52 and 78. 16384 rows of 32 + 8
// heads of 128 out of a fused projection (336 MB): 66 us, a copy 65.
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
  uint32_t magic;          // of a division by heads (Div)
};

struct RotP {
  RotParts part[2];
  const void* pos;
  const double* freq;
  long long rows;
  int hd, rot, half, axes, per_axis;   // half = rot / 2 pairs, per_axis of them for each axis
  int R, G, lrot;                      // rows of a wave's step; lanes of a head; lanes that rotate
  int pitch;                           // floats between the LDS rows of cosines
  uint32_t pitch_magic, axis_magic;    // of divisions by it and by per_axis (Div)
  bool fpos;
  float eps, mag, inv_hd;
  float* sums;                         // [workgroups][2][hd] partial gain gradients, or NULL
};

constexpr int kRotLds = 256;           // cosines, and sines, that a wave holds

// floor(x / d) for x < 2^16 and d < 2^16: by a multiplication, exact for these.
struct Div {
  int d;
  uint32_t magic;    // floor(2^32 / d) + 1 (d = 1: not used)
  __device__ __forceinline__ int div(int x) const { return d == 1 ? x : (int)__umulhi((uint32_t)x, magic); }
};

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

// WHOLE: pieces are whole or none.
template <typename T, bool WHOLE>
__device__ __forceinline__ uint4 load_n(const T* p, int n) {
  constexpr int E = 16 / (int)sizeof(T);
  if constexpr (WHOLE) return n > 0 ? load16u(p) : make_uint4(0, 0, 0, 0);
  return n == E ? load16u(p) : n > 0 ? load_partial(p, n) : make_uint4(0, 0, 0, 0);
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void store_n(T* p, int n, const float* v) {
  constexpr int E = 16 / (int)sizeof(T);
  if (WHOLE ? n > 0 : n == E)
    store16u(p, pack16<T>(v));
  else if (!WHOLE && n > 0)
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

// 1 / sqrt(x) to 2^-23, x > 0 (of a denormal number: as of the smallest normal one; NaN stays).
__device__ __forceinline__ float inverse_root(float x) {
  constexpr float least = 1.17549435e-38f;
  return __builtin_amdgcn_rsqf(x < least ? least : x);
}

// grid: x steps of R rows, four to a workgroup; y waves that share the heads of a step; z queries and keys.
template <typename T, bool INTER, bool BWD, bool WHOLE>
__global__ void __launch_bounds__(256, (BWD ? 4 : 1)) rotary_kernel(RotP p) {
  constexpr int E = 16 / (int)sizeof(T), RED = 2 * E + 1, ANGLES = 2 * 4 * kRotLds;
  __shared__ __attribute__((aligned(16))) float lds[BWD && 256 * RED > ANGLES ? 256 * RED : ANGLES];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float *const cs = lds + wid * 2 * kRotLds, *const sn = cs + kRotLds;
  const int l = lane & (p.G - 1), slot = lane / p.G, slots = 64 / p.G;
  const LaneAt at = lane_at<E, INTER>(p, l);
  const RotParts& t = p.part[blockIdx.z];
  const bool norm = t.gain;
  float ga[E], gb[E];
#pragma unroll
  for (int e = 0; e < E; ++e) ga[e] = gb[e] = 0.f;
  if (WHOLE && norm) {
    if (at.na > 0) __builtin_memcpy(ga, t.gain + at.a, sizeof(ga));
    if (at.nb > 0) __builtin_memcpy(gb, t.gain + at.b, sizeof(gb));
  } else if (norm) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (e < at.na) ga[e] = t.gain[at.a + e];
      if (e < at.nb) gb[e] = t.gain[at.b + e];
    }
  }
  float sum[2][E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[0][e] = sum[1][e] = 0.f;
  // a head's pieces on their way: x, and in the backward dy
  struct Item {
    int r, head;
    uint4 xa, xb, ya, yb;
  };
  const Div by_heads{t.heads, t.magic}, by_pitch{p.pitch, p.pitch_magic}, by_axis{p.per_axis, p.axis_magic};
  for (long long r0 = ((long long)blockIdx.x * 4 + wid) * p.R; r0 < p.rows; r0 += 4LL * gridDim.x * p.R) {
    const int R = (int)min((long long)p.R, p.rows - r0);
    const T* const xs = (const T*)t.x + r0 * t.x_row;
    const T* const ys = (const T*)t.dy + r0 * t.dy_row;
    T* const outs = (T*)t.out + r0 * t.out_row;
    auto load = [&](int i) {
      Item w;
      w.r = by_heads.div(i);
      w.head = i - w.r * t.heads;
      if (!BWD || norm) {
        const T* const x = xs + w.r * t.x_row + w.head * t.x_head;
        w.xa = load_n<T, WHOLE>(x + at.a, at.na);
        w.xb = load_n<T, WHOLE>(x + at.b, at.nb);
      }
      if constexpr (BWD) {
        const T* const dy = ys + w.r * t.dy_row + w.head * t.dy_head;
        w.ya = load_n<T, WHOLE>(dy + at.a, at.na);
        w.yb = load_n<T, WHOLE>(dy + at.b, at.nb);
      }
      return w;
    };
    auto finish = [&](const Item& w) {
      float c[E], s[E];
      if (at.turns) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          *reinterpret_cast<f32x4*>(c + e) = *reinterpret_cast<const f32x4*>(&cs[w.r * p.pitch + E * l + e]);
          *reinterpret_cast<f32x4*>(s + e) = *reinterpret_cast<const f32x4*>(&sn[w.r * p.pitch + E * l + e]);
        }
      }
      float a[E], b[E];
      if constexpr (!BWD) {
        unpack16<T>(w.xa, a);
        unpack16<T>(w.xb, b);
        if (norm) {
          float q = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) q = fmaf(a[e], a[e], fmaf(b[e], b[e], q));
          const float rstd = inverse_root(head_sum(q, p.G) * p.inv_hd + p.eps);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            a[e] *= rstd * ga[e];
            b[e] *= rstd * gb[e];
          }
        }
        if (at.turns) turn<E, INTER>(a, b, c, s, 1.f);
      } else {
        unpack16<T>(w.ya, a);
        unpack16<T>(w.yb, b);
        if (at.turns) turn<E, INTER>(a, b, c, s, -1.f);
        if (norm) {
          float xa[E], xb[E];
          unpack16<T>(w.xa, xa);
          unpack16<T>(w.xb, xb);
          float q = 0.f, m = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            q = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], q));
            m = fmaf(a[e] * ga[e], xa[e], fmaf(b[e] * gb[e], xb[e], m));
          }
          const float rstd = inverse_root(head_sum(q, p.G) * p.inv_hd + p.eps);
          m = head_sum(m, p.G) * p.inv_hd * rstd;       // mean(dn gain xhat)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float ua = xa[e] * rstd, ub = xb[e] * rstd;
            sum[0][e] = fmaf(a[e], ua, sum[0][e]);
            sum[1][e] = fmaf(b[e], ub, sum[1][e]);
            a[e] = rstd * (a[e] * ga[e] - ua * m);
            b[e] = rstd * (b[e] * gb[e] - ub * m);
          }
        }
      }
      T* const out = outs + w.r * t.out_row + w.head * t.out_head;
      store_n<T, WHOLE>(out + at.a, at.na, a);
      store_n<T, WHOLE>(out + at.b, at.nb, b);
    };
    // two heads of a lane in flight; the lanes of a head leave the loop together
    const int n = R * t.heads, by = slots * gridDim.y, first = blockIdx.y * slots + slot;
    Item w0 = load(min(first, n - 1)), w1 = load(min(first + by, n - 1));
    wave_sync();      // the previous step's angles have been read
    for (int i = lane; i < R * p.pitch; i += 64) {
      const int r = by_pitch.div(i), k = i - r * p.pitch;
      float c = 0.f, s = 0.f;      // behind a row: what a lane turns there stays 0
      if (k < p.half) {
        const long long w = p.axes == 1 ? r0 + r : (r0 + r) * p.axes + by_axis.div(k);
        const double x = p.fpos ? (double)((const float*)p.pos)[w] : (double)((const int*)p.pos)[w];
        cos_sin(x * p.freq[k], c, s);
      }
      cs[i] = p.mag * c;
      sn[i] = p.mag * s;
    }
    wave_sync();
    for (int i = first; i < n; i += 2 * by) {
      finish(w0);
      if (i + by < n) finish(w1);
      if (i + 2 * by < n) {
        w0 = load(i + 2 * by);
        w1 = load(min(i + 3 * by, n - 1));
      }
    }
  }
  if constexpr (BWD) {
    if (!p.sums) return;
    // the sums of the workgroup's heads, in order
    __syncthreads();
    float* const mine = lds + threadIdx.x * RED;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      mine[e] = sum[0][e];
      mine[E + e] = sum[1][e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.G * 2 * E; i += 256) {
      const int x = i / (2 * E), e = i % (2 * E);
      const LaneAt w = lane_at<E, INTER>(p, x);
      float v = 0.f;
      for (int s = 0; s < 4 * slots; ++s) v += lds[(s * p.G + x) * RED + e];
      float* const to = p.sums + (((long long)blockIdx.y * gridDim.x + blockIdx.x) * 2 + blockIdx.z) * p.hd;
      if (e < E && e < w.na) to[w.a + e] = v;
      if (e >= E && e - E < w.nb) to[w.b + e - E] = v;
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
  int R, G, lrot, pitch;
  bool whole;        // no piece ends inside a part of the head
  dim3 grid;
  int sums() const { return (int)(grid.x * grid.y); }
};
// Workgroups of the backward with a norm at most, for queries and for keys: each leaves a row of partial sums.
constexpr int kRotSums = 512;

RotPlan rot_plan(const RotaryArgs& a, bool sums) {
  RotPlan p;
  const int E = a.bf16 ? 8 : 4, half = a.rot / 2, rest = a.hd - a.rot;
  p.lrot = (half + E - 1) / E;
  const int lanes = p.lrot + (rest + 2 * E - 1) / (2 * E);
  p.G = 1;
  while (p.G < lanes) p.G *= 2;
  p.pitch = p.lrot * E;
  p.whole = (a.interleaved ? a.rot : half) % E == 0 && rest % E == 0;
  // four heads for every lane, while that leaves 2048 waves: an angle serves more of them, and the start of a step is
  // paid less often (65536 rows, 8 + 8 heads of 64: 8 rows 148 us, 2 rows 158; 16384 rows, 32 + 8 heads of 128: 1 row 67.7,
  // 2 rows 71.3)
  const int per_row = a.heads * p.G;
  p.R = (int)std::max<long long>(1, std::min<long long>(std::min((256 + per_row - 1) / per_row, kRotLds / p.pitch), a.rows / 2048));
  p.R = std::min(p.R, 65535 / std::max(a.heads, a.kv_heads));    // a step's heads, of queries and of keys, are counted by Div
  const long long groups = ((a.rows + p.R - 1) / p.R + 3) / 4;
  // few rows: waves share a row's heads, two for each lane
  const long long parts = std::max<long long>(1, std::min<long long>(256 / std::max<long long>(groups, 1), a.heads * p.G / 128));
  p.grid = dim3((unsigned)std::min<long long>(groups, sums ? kRotSums : 4096), (unsigned)parts, a.kv_heads ? 2 : 1);
  return p;
}

template <typename T, bool BWD>
void run(const RotaryArgs& a, const RotP& p, const RotPlan& l, hipStream_t st) {
  if (a.interleaved)
    l.whole ? rotary_kernel<T, true, BWD, true><<<l.grid, 256, 0, st>>>(p) : rotary_kernel<T, true, BWD, false><<<l.grid, 256, 0, st>>>(p);
  else
    l.whole ? rotary_kernel<T, false, BWD, true><<<l.grid, 256, 0, st>>>(p) : rotary_kernel<T, false, BWD, false><<<l.grid, 256, 0, st>>>(p);
}
template <bool BWD>
hipError_t run(const RotaryArgs& a, const RotP& p, const RotPlan& l, hipStream_t st) {
  a.bf16 ? run<bf16_t, BWD>(a, p, l, st) : run<float, BWD>(a, p, l, st);
  return hipGetLastError();
}

uint32_t magic(int d) { return d > 1 ? (uint32_t)((1ull << 32) / d + 1) : 0; }

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
  p.pitch_magic = magic(l.pitch);
  p.axis_magic = magic(p.per_axis);
  p.fpos = a.fpos;
  p.eps = a.eps;
  p.mag = a.mag;
  p.inv_hd = 1.0f / a.hd;
  return p;
}

}  // namespace

hipError_t launch_rotary_fwd(const RotaryArgs& a, const void* q, const void* k, const void* pos, const double* freq,
                             const float* gain_q, const float* gain_k, void* out_q, void* out_k, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const RotPlan l = rot_plan(a, false);
  RotP p = params(a, l, pos, freq);
  p.part[0] = RotParts{q, nullptr, out_q, gain_q, a.q_row, a.q_head, 0, 0, a.oq_row, a.oq_head, a.heads, magic(a.heads)};
  p.part[1] = RotParts{k, nullptr, out_k, gain_k, a.k_row, a.k_head, 0, 0, a.ok_row, a.ok_head, a.kv_heads, magic(a.kv_heads)};
  return run<false>(a, p, l, st);
}

size_t rotary_bwd_ws_bytes(const RotaryArgs& a) { return sizeof(float) * 2 * a.hd * (size_t)rot_plan(a, true).sums(); }

hipError_t launch_rotary_bwd(const RotaryArgs& a, const void* q, const void* k, const void* pos, const double* freq,
                             const float* gain_q, const float* gain_k, const void* dy_q, const void* dy_k, void* dq, void* dk,
                             float* dgain_q, float* dgain_k, void* ws, hipStream_t st) {
  const bool sums = gain_q || gain_k;
  const RotPlan l = rot_plan(a, sums);
  if (a.rows > 0) {
    RotP p = params(a, l, pos, freq);
    p.part[0] = RotParts{q, dy_q, dq, gain_q, a.q_row, a.q_head, a.dq_row, a.dq_head, a.oq_row, a.oq_head, a.heads, magic(a.heads)};
    p.part[1] = RotParts{k, dy_k, dk, gain_k, a.k_row, a.k_head, a.dk_row, a.dk_head, a.ok_row, a.ok_head, a.kv_heads, magic(a.kv_heads)};
    p.sums = sums ? (float*)ws : nullptr;
    const hipError_t e = run<true>(a, p, l, st);
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;
  rotary_gain_kernel<<<(2 * a.hd + 63) / 64, 1024, 0, st>>>((const float*)ws, a.rows > 0 ? l.sums() : 0, a.hd, dgain_q, dgain_k);
  return hipGetLastError();
}

}  // namespace bsa
