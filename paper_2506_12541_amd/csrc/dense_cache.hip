// Cache of 8 bits for packed attention: rows of keys and values are quantised as they are written, read back,
// and read by the attention (the layout of sequences and the masks are dense_attn.hip's).
//
// A row of a head is stored as e4m3 values and one power of two: e is the smallest exponent in [-64, 63] with
// max |x| 2^-e <= 448. e4m3 keeps 4 bits wherever it has a normal number, so a finer scale would gain nothing but the
// last places of subnormals, and a power of two makes the e4m3 rounding the only one: what a byte stands for is
// exact in bf16, and products with the scale are exact.
#include "dense_packed.hpp"

namespace bsa {
namespace {

constexpr int kExpLow = -64, kExpHigh = 63, kExpBias = 127;

// ---- quantising and reading back ----

// The cache row of row t of the new rows, -1 if it has none. Per lane; every lane of the wave is here. Up to 64
// sequences are found in registers (a lane holds one).
__device__ __forceinline__ int cache_row(const SeqArgs& a, long long t) {
  int lo = 0, n = a.S;      // the last sequence that starts at t or before lies in [lo, lo + n)
  if (a.S <= 64) {
    const int mine = a.cu_q[min((int)(threadIdx.x & 63), a.S - 1)];
#pragma unroll
    for (int step = 32; step > 0; step >>= 1) {
      const int at = __shfl(mine, min(lo + step, 63), 64);
      if (lo + step < a.S && at <= t) lo += step;
    }
  } else {
    while (n > 1) {
      const int half = n / 2;
      const bool right = a.cu_q[lo + half] <= t;
      lo += right ? half : 0;
      n = right ? n - half : half;
    }
  }
  const Seq q = seq_at(a, lo);
  const long long i = t - q.q0, at = (long long)q.lk - q.lq + i;
  return i >= 0 && i < q.lq && at >= 0 ? (int)(q.k0 + at) : -1;
}

struct CacheP {
  CacheArgs a;
  SeqArgs seq;
  const void *k, *v;             // rows outside the cache (written by the read kernel)
  uint8_t *ck, *cv, *ek, *ev;
};

__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// 16 elements of a row.
__device__ __forceinline__ void load16e(const float* p, float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack16<float>(*reinterpret_cast<const uint4*>(p + 4 * i), v + 4 * i);
}
__device__ __forceinline__ void load16e(const bf16_t* p, float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) unpack16<bf16_t>(*reinterpret_cast<const uint4*>(p + 8 * i), v + 8 * i);
}
__device__ __forceinline__ void store16e(float* p, const float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(p + 4 * i) = pack16<float>(v + 4 * i);
}
__device__ __forceinline__ void store16e(bf16_t* p, const float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) *reinterpret_cast<uint4*>(p + 8 * i) = pack16<bf16_t>(v + 8 * i);
}

// Two e4m3 values (the half `hi` of w) times 2^e as bf16: exact.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
}

// A lane holds 16 values of a head of a key row and of a value row, HD / 16 lanes the head.
template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_write_kernel(CacheP p) {
  constexpr int LPH = HD / 16;
  const CacheArgs& a = p.a;
  const long long total = a.rows * a.kv_heads;
  const int l = threadIdx.x % LPH;
  for (long long b = (long long)blockIdx.x * (256 / LPH); b < total; b += (long long)gridDim.x * (256 / LPH)) {
    const long long hr = b + threadIdx.x / LPH, t = min(hr, total - 1) / a.kv_heads;
    const int h = (int)(min(hr, total - 1) - t * a.kv_heads);
    const int row = cache_row(p.seq, t);
    float v[2][16];
    load16e((const T*)p.k + t * a.k_row + h * a.k_head + 16 * l, v[0]);
    load16e((const T*)p.v + t * a.v_row + h * a.v_head + 16 * l, v[1]);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      float top = 0.f;      // of the finite values
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x = fabsf(v[w][i]);
        top = fmaxf(top, x < __builtin_huge_valf() ? x : 0.f);
      }
#pragma unroll
      for (int o = LPH / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      const uint32_t bits = __float_as_uint(top);
      // 448 = 1.75 2^8
      const int e = max(kExpLow, min(kExpHigh, (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0)));
      const float inv = two_to(-e);
      int q[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float x = v[w][4 * i + c];
          y[c] = fabsf(x) < __builtin_huge_valf() ? __builtin_amdgcn_fmed3f(x * inv, -448.f, 448.f) : __builtin_nanf("");
        }
        q[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        q[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], q[i], true);
      }
      if (hr < total && row >= 0) {
        uint8_t* const to = w == 0 ? p.ck + row * a.ck_row + h * a.ck_head : p.cv + row * a.cv_row + h * a.cv_head;
        *reinterpret_cast<uint4*>(to + 16 * l) = make_uint4(q[0], q[1], q[2], q[3]);
        if (l == 0) (w == 0 ? p.ek : p.ev)[h * a.total_k + row] = (uint8_t)(e + kExpBias);
      }
    }
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_read_kernel(CacheP p) {
  constexpr int LPH = HD / 16;
  const CacheArgs& a = p.a;
  const long long total = a.rows * a.kv_heads;
  const int l = threadIdx.x % LPH;
  for (long long b = (long long)blockIdx.x * (256 / LPH); b < total; b += (long long)gridDim.x * (256 / LPH)) {
    const long long hr = b + threadIdx.x / LPH, t = min(hr, total - 1) / a.kv_heads;
    const int h = (int)(min(hr, total - 1) - t * a.kv_heads);
    const int row = cache_row(p.seq, t);
    uint4 q[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    float s[2] = {1.f, 1.f};
    if (row >= 0) {
      q[0] = *reinterpret_cast<const uint4*>(p.ck + row * a.ck_row + h * a.ck_head + 16 * l);
      q[1] = *reinterpret_cast<const uint4*>(p.cv + row * a.cv_row + h * a.cv_head + 16 * l);
      s[0] = two_to(p.ek[h * a.total_k + row] - kExpBias);
      s[1] = two_to(p.ev[h * a.total_k + row] - kExpBias);
    }
    if (hr >= total) continue;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const uint32_t word[4] = {q[w].x, q[w].y, q[w].z, q[w].w};
      float v[16];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = e4m3_pair<false>(word[i], s[w]), hi = e4m3_pair<true>(word[i], s[w]);
        v[4 * i] = __uint_as_float(lo << 16);
        v[4 * i + 1] = __uint_as_float(lo & 0xffff0000u);
        v[4 * i + 2] = __uint_as_float(hi << 16);
        v[4 * i + 3] = __uint_as_float(hi & 0xffff0000u);
      }
      T* const to = w == 0 ? (T*)p.k + t * a.k_row + h * a.k_head : (T*)p.v + t * a.v_row + h * a.v_head;
      store16e(to + 16 * l, v);
    }
  }
}

// ---- attention ----

struct CacheFwdP {
  FwdP f;                        // k and v: the cache's bytes
  const uint8_t *ek, *ev;
};

// A tile of ROWS x HD bytes on its way into LDS as bf16, by NW waves: loaded into registers, and stored
// once the tile before it is in use.
template <int HD, int ROWS, int NW>
struct ByteTile {
  static constexpr int PER = ROWS * HD / (64 * NW), B = PER >= 16 ? 16 : 8, CPR = HD / B, NU = PER / B;
  static_assert(B * NU == PER, "tile / wave split");
  uint2 w[NU][B / 8];
  uint8_t e[NU];
  __device__ __forceinline__ void load(const uint8_t* g, long long ld, const uint8_t* exps, int r0, int nrows, int wid, int lane) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int i = (wid * NU + u) * 64 + lane, r = min(r0 + i / CPR, nrows - 1);
      __builtin_memcpy(w[u], g + r * ld + B * (i % CPR), B);
      e[u] = exps[r];
    }
  }
  __device__ __forceinline__ void store(bf16_t* t, int wid, int lane) const {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const int i = (wid * NU + u) * 64 + lane, row = i / CPR, c = (i % CPR) * (B / 8);
      const float s = two_to((int)e[u] - kExpBias);
#pragma unroll
      for (int h = 0; h < B / 8; ++h)
        *reinterpret_cast<uint4*>(t + row * HD + 8 * ((c + h) ^ tswz<bf16_t, HD>(row))) =
            make_uint4(e4m3_pair<false>(w[u][h].x, s), e4m3_pair<true>(w[u][h].x, s), e4m3_pair<false>(w[u][h].y, s),
                       e4m3_pair<true>(w[u][h].y, s));
    }
  }
};

// float32 values as three bf16 parts: x1 = bf16(x), x2 = bf16(x - x1), x3 = bf16(x - x1 - x2). bf16: one.
template <typename T, int P>
__device__ __forceinline__ void to_parts(const float* v, bf16x8 (&out)[P]) {
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = v[i];
#pragma unroll
  for (int k = 0; k < P; ++k) {
    out[k] = make_chunk<bf16_t>(x);
    if (k + 1 < P) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] -= (float)out[k][i];
    }
  }
}

// As packed_fwd_kernel of dense_attn.hip, with keys and values from the cache.
template <typename T, int HD, int QB, bool SPLIT>
__global__ void __launch_bounds__((64 * kWaves)) cache_fwd_kernel(CacheFwdP cp) {
  static_assert(!SPLIT || QB == 1, "one block of rows");
  constexpr int NW = kWaves, KT = SPLIT ? 32 : 64, ST = SPLIT ? NW * KT : KT, ELEMS = (SPLIT ? NW : 1) * KT * HD;
  constexpr int KB = KT / 16, NCH = HD / 32, DB = HD / 16, R = 16 * QB * (SPLIT ? 1 : NW), P = sizeof(T) == 4 ? 3 : 1;
  __shared__ __attribute__((aligned(1024))) bf16_t ks0a[ELEMS], vs0a[ELEMS], ks1a[ELEMS], vs1a[ELEMS];
  const FwdP& p = cp.f;
  const AttnArgs& a = p.a;
  const Group G = p.G;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, j = lane >> 4;
  int slot, hk;
  xcd_slot(slot, hk);
  const Seq sq = find_seq<false>(slot, p.seq, G.G, R, a.zero_rest);
  const int rows = sq.lq * G.G, ext = sq.eq * G.G;
  const int nt = (rows + R - 1) / R;
  const long long tile = sq.tile < nt ? nt - 1 - sq.tile : sq.tile;
  if (tile < 0 || tile * R >= ext) return;
  const int p0 = (int)tile * R;
  if (p0 >= ext || (p0 >= rows && (!a.zero_rest || p.nsplit > 1))) return;
  T* const out = (T*)p.o;

  int pr[QB];
  int lim[QB];        // the last key that this lane's query sees
  bf16x8 qf[QB][NCH][P];
  f32x4 o[QB][DB];
  float mx[QB], ls[QB];
  const int off = sq.lk - sq.lq;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    pr[qb] = p0 + ((SPLIT ? 0 : wid * QB) + qb) * 16 + r;
    const bool on = pr[qb] < rows;
    const RowAt at = packed_row(sq, hk, G, on ? pr[qb] : 0);
    lim[qb] = !on ? -1 : a.causal ? min((int)(at.t - sq.q0) + off, sq.lk - 1) : sq.lk - 1;
    const T* qp = (const T*)p.q + at.t * a.q_row + at.h * a.q_head;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      typedef typename Chunk<T>::type CT;
      const CT x = on ? load_chunk(qp + 32 * c + 8 * j) : zero_chunk(CT{});
      if constexpr (P == 1) {
        qf[qb][c][0] = x;
      } else {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = x[e];
        to_parts<T, P>(v, qf[qb][c]);
      }
    }
    mx[qb] = kNegInf;
    ls[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[qb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // the workgroup's keys: its split's, cut behind the last key that its last query sees
  int k_lo, k_hi;
  split_range(sq.lk, p.nsplit, blockIdx.z, KT, k_lo, k_hi);
  const int plast = min(p0 + R, rows) - 1;
  if (p0 >= rows)
    k_hi = k_lo;
  else if (a.causal)
    k_hi = max(min(k_hi, G.div(plast) + off + 1), k_lo);
  // keys up to here are seen by every query of the workgroup: tiles below need no mask
  const int all = min(a.causal ? max(G.div(min(p0, rows)) + off + 1, 0) : sq.lk, k_hi);

  const uint8_t* const kh = (const uint8_t*)p.k + sq.k0 * a.k_row + hk * a.k_head;
  const uint8_t* const vh = (const uint8_t*)p.v + sq.k0 * a.v_row + hk * a.v_head;
  const uint8_t *const ek = cp.ek + hk * a.total_k + sq.k0, *const ev = cp.ev + hk * a.total_k + sq.k0;
  const int lw = SPLIT ? 0 : wid, own = SPLIT ? wid * KT * HD : 0;
  bf16_t *const ks0 = ks0a + own, *const vs0 = vs0a + own, *const ks1 = ks1a + own, *const vs1 = vs1a + own;
  ByteTile<HD, KT, SPLIT ? 1 : NW> kt, vt;
  auto load = [&](int t0) __attribute__((always_inline)) {
    kt.load(kh, a.k_row, ek, t0, sq.lk, lw, lane);
    vt.load(vh, a.v_row, ev, t0, sq.lk, lw, lane);
  };
  auto visible = [&]() __attribute__((always_inline)) {
    if constexpr (SPLIT)
      wave_sync();
    else
      __syncthreads();
  };
  int odd_key = INT32_MAX;   // the first key with a v that is not finite, from the diagonal's tiles
  auto step = [&](auto mask, int t0, bf16_t* kc, bf16_t* vc, bf16_t* kn, bf16_t* vn) __attribute__((always_inline)) {
    visible();
    if constexpr (decltype(mask)::value) {
      if (a.causal) {
        const int x = clear_tile<bf16_t, HD, KT, SPLIT>(vc);
        odd_key = x < KT ? min(odd_key, t0 + x) : odd_key;
      }
    }
    const bool more = t0 + ST < k_hi;
    if (more) load(t0 + ST);
    f32x4 s[QB][KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const bf16x8 kf = row_frag<HD>(kc, kb * 16 + r, 4 * c + j);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int x = P - 1; x >= 0; --x)      // the small parts first
            s[qb][kb] = mma(kf, qf[qb][c][x], c == 0 && x == P - 1 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[qb][kb]);
      }
    bf16x8 pf[QB][KB / 2][P];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      float tmax = kNegInf;
      if constexpr (decltype(mask)::value) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            s[qb][kb][i] = t0 + kb * 16 + 4 * j + i <= lim[qb] ? s[qb][kb][i] : kNegInf;
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) tmax = fmaxf(tmax, s[qb][kb][i]);
      // the reference maximum moves only when a score exceeds it by 2^kRescale
      if (__builtin_amdgcn_ballot_w64(tmax * p.sl2 > mx[qb] + kRescale)) {
        tmax = col_max(tmax) * p.sl2;
        const bool raise = tmax > mx[qb] + kRescale;
        const float mnew = raise ? tmax : mx[qb];
        const float alpha = raise ? fast_exp2(mx[qb] - mnew) : 1.0f;
        mx[qb] = mnew;
        ls[qb] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[qb][db] *= alpha;
      }
      const float mref = mx[qb] == kNegInf ? 0.f : mx[qb];
#pragma unroll
      for (int kp = 0; kp < KB / 2; ++kp) {
        float v8[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v8[i] = fast_exp2(__builtin_fmaf(s[qb][2 * kp][i], p.sl2, -mref));
          v8[4 + i] = fast_exp2(__builtin_fmaf(s[qb][2 * kp + 1][i], p.sl2, -mref));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) ls[qb] += v8[i];
        to_parts<T, P>(v8, pf[qb][kp]);
      }
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int kp = 0; kp < KB / 2; ++kp) {
        const bf16x8 vf = col_frag<HD>(vc, 32 * kp, 16 * db, lane);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
#pragma unroll
          for (int x = P - 1; x >= 0; --x) o[qb][db] = mma(vf, pf[qb][kp][x], o[qb][db]);
      }
    if (more) {     // the tile before this one has been read by every wave (visible)
      kt.store(kn, lw, lane);
      vt.store(vn, lw, lane);
    }
  };
  const int k_first = k_lo + (SPLIT ? wid * KT : 0);
  if (k_first < k_hi) {
    load(k_first);
    kt.store(ks0, lw, lane);
    vt.store(vs0, lw, lane);
    int t0 = k_first;
    for (; t0 + ST + KT <= all; t0 += 2 * ST) {
      step(std::false_type{}, t0, ks0, vs0, ks1, vs1);
      step(std::false_type{}, t0 + ST, ks1, vs1, ks0, vs0);
    }
    for (; t0 < k_hi; t0 += 2 * ST) {
      step(std::true_type{}, t0, ks0, vs0, ks1, vs1);
      if (t0 + ST < k_hi) step(std::true_type{}, t0 + ST, ks1, vs1, ks0, vs0);
    }
  }
  if (odd_key != INT32_MAX) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (odd_key <= lim[qb]) o[qb][db] *= __builtin_nanf("");
  }
  // four columns of a finished row (first: the thread that also writes the row's statistics)
  auto store = [&](int row, int c, f32x4 v, float m, float l, bool first) {
    if (row >= ext) return;
    const RowAt at = packed_row(sq, hk, G, row);
    if (p.nsplit > 1) {
      if (row >= rows) return;
      const long long pos = ((long long)blockIdx.z * a.total_q + at.t) * a.heads + at.h;
      if (k_lo < k_hi) store4(p.part + pos * HD + c, v, 1.f);   // else l = 0: not read
      if (first) p.ml[pos] = make_float2(m, l);
    } else {
      if (row >= rows && !a.zero_rest) return;
      const bool any = row < rows && !(l == 0.f);   // a sum of NaN stays one
      store4(out + at.t * a.o_row + at.h * a.o_head + c, any ? v : f32x4{0.f, 0.f, 0.f, 0.f}, any ? 1.0f / l : 0.f);
      if (first) p.lse[at.h * a.total_q + at.t] = any ? (m + log2f(l)) * kLn2 : kNegInf;
    }
  };
  if constexpr (!SPLIT) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const float l = col_sum(ls[qb]);
#pragma unroll
      for (int db = 0; db < DB; ++db) store(pr[qb], 16 * db + 4 * j, o[qb][db], mx[qb], l, db == 0 && j == 0);
    }
  } else {
    __shared__ float2 mls[NW][16];
    const float l = col_sum(ls[0]);
    __syncthreads();   // every wave has read its last tile
    static_assert(NW * 16 * HD * 4 <= ELEMS * 2, "the waves' results in a staged tensor's place");
    float* const mine = reinterpret_cast<float*>(ks0a) + wid * 16 * HD;
#pragma unroll
    for (int db = 0; db < DB; ++db) *join_at<HD>(mine, r, 4 * db + j) = o[0][db];
    if (j == 0) mls[wid][r] = make_float2(mx[0], l);
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * (HD / 4); i += 64 * NW) {
      const int row = i / (HD / 4), c4 = i % (HD / 4);
      float m = kNegInf, sum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) m = fmaxf(m, mls[w][row].x);
      const float mref = m == kNegInf ? 0.f : m;
      f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float f = fast_exp2(mls[w][row].x - mref);
        sum += f * mls[w][row].y;
        v += f * *join_at<HD>(reinterpret_cast<float*>(ks0a) + w * 16 * HD, row, c4);
      }
      store(p0 + row, 4 * c4, v, m, sum, c4 == 0);
    }
  }
}

// ---- host ----

// float32 rows take three parts of registers: 16 rows a wave.
constexpr int cache_qb(bool bf16) { return bf16 ? 2 : 1; }

FwdPlan cache_plan(const AttnArgs& a) {
  const long long rows = a.total_q * a.group();
  const long long avg_k = a.total_k / a.seqs;
  const int R = 16 * cache_qb(a.bf16) * kWaves;
  auto wgs = [&](int r) { return std::max<long long>((rows + r - 1) / r, a.seqs) * a.kv_heads; };
  FwdPlan f;
  f.split = rows <= 32LL * a.seqs || wgs(R) < 128;
  const long long n = 512 / wgs(f.split ? 16 : R);
  f.nsplit = (int)std::max<long long>(std::min<long long>(std::min<long long>(n, avg_k / 256), 64), 1);
  return f;
}

template <typename T, int HD>
hipError_t cache_attn(const CacheFwdP& p, bool split, hipStream_t st) {
  const AttnArgs& a = p.f.a;
  constexpr int QB = cache_qb(sizeof(T) == 2);
  auto grid = [&](int R) { return dim3(tile_slots(a.total_q, a.group(), R, a.seqs), a.kv_heads, p.f.nsplit); };
  if (split)
    cache_fwd_kernel<T, HD, 1, true><<<grid(16), 64 * kWaves, 0, st>>>(p);
  else
    cache_fwd_kernel<T, HD, QB, false><<<grid(16 * QB * kWaves), 64 * kWaves, 0, st>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.f.nsplit == 1) return e;
  const long long n = a.total_q * a.heads, per = 256 / (HD / 4);
  packed_join_kernel<T, HD><<<(unsigned)((n + per - 1) / per), 256, 0, st>>>(p.f);
  return hipGetLastError();
}

template <typename T, int HD>
hipError_t cache_move(const CacheP& p, bool write, hipStream_t st) {
  const long long per = 256 / (HD / 16), n = (p.a.rows * p.a.kv_heads + per - 1) / per;
  const unsigned grid = (unsigned)std::min<long long>(n, 1 << 20);
  if (write)
    cache_write_kernel<T, HD><<<grid, 256, 0, st>>>(p);
  else
    cache_read_kernel<T, HD><<<grid, 256, 0, st>>>(p);
  return hipGetLastError();
}

#define BSA_CACHE_DISPATCH(FN, a, ...)                                                                      \
  ((a).bf16 ? ((a).hd == 128  ? FN<bf16_t, 128>(__VA_ARGS__)                                                \
               : (a).hd == 64 ? FN<bf16_t, 64>(__VA_ARGS__)                                                 \
                              : FN<bf16_t, 32>(__VA_ARGS__))                                                \
            : ((a).hd == 128  ? FN<float, 128>(__VA_ARGS__)                                                 \
               : (a).hd == 64 ? FN<float, 64>(__VA_ARGS__)                                                  \
                              : FN<float, 32>(__VA_ARGS__)))

}  // namespace

hipError_t launch_cache_write(const CacheArgs& a, const void* k, const void* v, const int* cu_q, const int* cu_k,
                              const int* used_k, void* ck, void* cv, unsigned char* ek, unsigned char* ev, hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const CacheP p{a, SeqArgs{cu_q, cu_k, used_k, a.seqs, a.rows, a.total_k}, k, v, (uint8_t*)ck, (uint8_t*)cv, ek, ev};
  return BSA_CACHE_DISPATCH(cache_move, a, p, true, st);
}

hipError_t launch_cache_read(const CacheArgs& a, const void* ck, const void* cv, const unsigned char* ek,
                             const unsigned char* ev, const int* cu_q, const int* cu_k, const int* used_k, void* k, void* v,
                             hipStream_t st) {
  if (a.rows == 0) return hipSuccess;
  const CacheP p{a, SeqArgs{cu_q, cu_k, used_k, a.seqs, a.rows, a.total_k}, k, v, (uint8_t*)ck, (uint8_t*)cv, (uint8_t*)ek, (uint8_t*)ev};
  return BSA_CACHE_DISPATCH(cache_move, a, p, false, st);
}

bool cache_attention_fits(const AttnArgs& a) {
  return tile_slots(a.total_q, a.group(), cache_plan(a).split ? 16 : 16 * cache_qb(a.bf16) * kWaves, a.seqs) < 1u << 24;
}

size_t cache_attention_ws_bytes(const AttnArgs& a) {
  const int s = cache_plan(a).nsplit;
  if (s == 1) return 0;
  const size_t rows = (size_t)s * a.total_q * a.heads;
  return align256(rows * a.hd * sizeof(float)) + align256(rows * sizeof(float2));
}

hipError_t launch_cache_attention(const AttnArgs& a, const void* q, const void* ck, const void* cv, const unsigned char* ek,
                                  const unsigned char* ev, const int* cu_q, const int* cu_k, const int* used_k, void* o,
                                  float* lse, void* ws, hipStream_t st) {
  if (a.total_q == 0) return hipSuccess;
  const FwdPlan f = cache_plan(a);
  CacheFwdP p{FwdP{a, q, ck, cv, SeqArgs{cu_q, cu_k, used_k, a.seqs, a.total_q, a.total_k}, group_of(a), o, lse,
                   a.scale * kLog2e, f.nsplit, nullptr, nullptr},
              ek, ev};
  if (f.nsplit > 1) {
    p.f.part = (float*)ws;
    p.f.ml = (float2*)((char*)ws + align256((size_t)f.nsplit * a.total_q * a.heads * a.hd * sizeof(float)));
  }
  return BSA_CACHE_DISPATCH(cache_attn, a, p, f.split, st);
}

}  // namespace bsa
