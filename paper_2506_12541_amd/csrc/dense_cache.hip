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
  int chunk;                     // keys of a split
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
template <typename T> constexpr int parts_of() { return sizeof(T) == 4 ? 3 : 1; }
// Of a probability in calls of few rows (cache_step_kernel). Beside a bf16 query two, within 2^-16 of it: the matrix cores wait for
// memory there, so a second product costs 0 to 1.5 % (32 tokens against 64 to 8192 rows: 69.8 us, so 70.0; 16 x 1 to 4
// rows, 4 key heads: 36.8 and 37.2), and outputs are off by their own rounding alone: 0.0017 of the norm, with one part 0.0023 to
// 0.0026.
template <typename T> constexpr int probability_parts() { return sizeof(T) == 4 ? 3 : 2; }
template <int P>
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

// Four columns c.. of a finished packed row, or of its split's part (any: the split has keys; else l = 0 and its
// part is not read). first: the thread that also writes the row's statistics.
template <typename T, int HD>
__device__ __forceinline__ void store_row(const FwdP& p, const Seq& sq, int hk, int split, int row, int c, f32x4 v, float m, float l,
                                          bool any, bool first) {
  const AttnArgs& a = p.a;
  const int rows = sq.lq * p.G.G;
  if (row >= sq.eq * p.G.G) return;
  const RowAt at = packed_row(sq, hk, p.G, row);
  if (p.nsplit > 1) {
    if (row >= rows) return;
    const long long pos = ((long long)split * a.total_q + at.t) * a.heads + at.h;
    if (any) store4(p.part + pos * HD + c, v, 1.f);
    if (first) p.ml[pos] = make_float2(m, l);
  } else {
    if (row >= rows && !a.zero_rest) return;
    const bool saw = row < rows && !(l == 0.f);   // a sum of NaN stays one
    store4((T*)p.o + at.t * a.o_row + at.h * a.o_head + c, saw ? v : f32x4{0.f, 0.f, 0.f, 0.f}, saw ? 1.0f / l : 0.f);
    if (first) p.lse[at.h * a.total_q + at.t] = saw ? (m + log2f(l)) * kLn2 : kNegInf;
  }
}

// The keys of this workgroup's split, cut behind the last key that its last query sees: [lo, hi). Every query of
// the workgroup (packed rows [p0, p0 + R)) sees the keys below `all`.
struct Keys {
  int lo, hi, all;
};
__device__ __forceinline__ Keys keys_of(const FwdP& p, const Seq& sq, int split, int nsplit, int p0, int R, int KT) {
  Keys k;
  const int rows = sq.lq * p.G.G, off = sq.lk - sq.lq;
  split_range(sq.lk, nsplit, split, KT, k.lo, k.hi);
  if (p0 >= rows)
    k.hi = k.lo;
  else if (p.a.causal)
    k.hi = max(min(k.hi, p.G.div(min(p0 + R, rows) - 1) + off + 1), k.lo);
  k.all = min(p.a.causal ? max(p.G.div(min(p0, rows)) + off + 1, 0) : sq.lk, k.hi);
  return k;
}

// The workgroup's first packed row (tiles in descending order: with a causal mask the longest rows come first),
// -1: it has none.
__device__ __forceinline__ int first_row(const FwdP& p, const Seq& sq, int R) {
  const int rows = sq.lq * p.G.G, ext = sq.eq * p.G.G, nt = (rows + R - 1) / R;
  const long long tile = sq.tile < nt ? nt - 1 - sq.tile : sq.tile;
  if (tile < 0 || tile * R >= ext) return -1;
  const int p0 = (int)tile * R;
  return p0 >= rows && (!p.a.zero_rest || p.nsplit > 1) ? -1 : p0;
}

// Eight values of a query as its parts.
template <typename T, int P>
__device__ __forceinline__ void query_parts(const T* q, bool on, bf16x8 (&out)[P]) {
  typedef typename Chunk<T>::type CT;
  const CT x = on ? load_chunk(q) : zero_chunk(CT{});
  if constexpr (P == 1) {
    out[0] = x;
  } else {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e];
    to_parts<P>(v, out);
  }
}

// Eight e4m3 values times a power of two as bf16.
__device__ __forceinline__ bf16x8 e4m3_chunk(uint2 w, float scale) {
  return __builtin_bit_cast(bf16x8, make_uint4(e4m3_pair<false>(w.x, scale), e4m3_pair<true>(w.x, scale),
                                               e4m3_pair<false>(w.y, scale), e4m3_pair<true>(w.y, scale)));
}

// A lane's part of 32 keys: of key r of each 16 its bytes [64 i + 16 j, + 16) and the code of its scale, and the
// codes of the values of the keys 16 b + 4 j + [0, 4), whose scores the lane will hold.
template <int HD>
struct StepTile {
  static constexpr int NP = HD == 32 ? 1 : HD / 64, W = HD == 32 ? 2 : 4;     // pieces, words of a piece
  uint32_t w[2][NP][W];
  uint8_t ek[2];
  uint32_t ev[2];
  // the head's first value in chunk c (8 values) of lane group j
  __device__ __forceinline__ static int first(int c, int j) { return HD == 32 ? 8 * j : 64 * (c / 2) + 16 * j + 8 * (c % 2); }
  __device__ __forceinline__ uint2 chunk(int kb, int c) const {
    return HD == 32 ? make_uint2(w[kb][0][0], w[kb][0][1]) : make_uint2(w[kb][c / 2][2 * (c % 2) % W], w[kb][c / 2][(2 * (c % 2) + 1) % W]);
  }
  // keys at or past nkeys repeat the last one
  __device__ __forceinline__ void load(const uint8_t* k, long long ld, const uint8_t* ck, const uint8_t* cv, int t0, int nkeys,
                                       int r, int j) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const int row = min(t0 + 16 * kb + r, nkeys - 1);
#pragma unroll
      for (int i = 0; i < NP; ++i) __builtin_memcpy(w[kb][i], k + row * ld + 64 * i + 4 * W * j, 4 * W);
      ek[kb] = ck[row];
    }
    if (t0 + 32 <= nkeys) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) __builtin_memcpy(&ev[kb], cv + t0 + 16 * kb + 4 * j, 4);
    } else {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        ev[kb] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) ev[kb] |= (uint32_t)cv[min(t0 + 16 * kb + 4 * j + i, nkeys - 1)] << (8 * i);
      }
    }
  }
};

// A value tile of 32 rows x HD bytes in LDS, pieces of 16 bytes; the swizzle puts the 8 rows that a lane group reads
// at a time (byte_cols) on distinct banks.
template <int HD>
__device__ __forceinline__ int byte_swz(int row) {
  const int far = row >> 4 & 1;
  return HD == 128 ? (row >> 1 & 1) | far << 1 | (row >> 2 & 1) << 2 : HD == 64 ? far | (row >> 2 & 1) << 1 : far;
}
template <int HD>
__device__ __forceinline__ void byte_tile_issue(uint8_t* lds, const uint8_t* g, long long ld, int r0, int nrows, int lane) {
  constexpr int CPR = HD / 16;
#pragma unroll
  for (int u = 0; u < 32 * CPR / 64; ++u) {
    const int i = u * 64 + lane, row = i / CPR;
    load_lds16(g + min(r0 + row, nrows - 1) * ld + 16 * ((i % CPR) ^ byte_swz<HD>(row)), lds + 1024 * u);
  }
}
// Column 16 db + r of the rows 4 j + [0, 4) and 16 + 4 j + [0, 4): the transposing read hands lane r of a 16-lane
// group byte r of the eight 16-byte rows that the lanes 2 i and 2 i + 1 address.
template <int HD>
__device__ __forceinline__ uint2 byte_cols(const uint8_t* t, int db, int r, int j) {
  typedef int v2i __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) v2i lds_v2i;
  const int i = r >> 1, row = (i & 3) + 4 * j + 16 * (i >> 2);
  const uint8_t* at = t + row * HD + 16 * (db ^ byte_swz<HD>(row)) + 8 * (r & 1);
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2i*)at));
}
// Clears the 16-byte pieces of a wave's landed tile that hold a NaN byte; returns the first row with one (32: none).
template <int HD>
__device__ __forceinline__ int clear_bytes(uint8_t* t, int lane) {
  constexpr int CPR = HD / 16;
  uint4* const piece = reinterpret_cast<uint4*>(t);
  int first = 32;
#pragma unroll
  for (int u = 32 * CPR / 64 - 1; u >= 0; --u) {
    const uint4 v = piece[u * 64 + lane];
    constexpr uint32_t ones = 0x7f7f7f7fu, one = 0x01010101u;      // 0x7f and 0xff are NaN
    const uint32_t any = ((v.x & ones) + one) | ((v.y & ones) + one) | ((v.z & ones) + one) | ((v.w & ones) + one);
    if (any & 0x80808080u) {
      piece[u * 64 + lane] = make_uint4(0, 0, 0, 0);
      first = (u * 64 + lane) / CPR;
    }
  }
  if (!__builtin_amdgcn_ballot_w64(first < 32)) return 32;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o, 64));
  wave_sync();
  return __builtin_amdgcn_readfirstlane(first);
}

// Many rows: as packed_fwd_kernel of dense_attn.hip, the tiles of keys and values converted to bf16 as they are
// stored in LDS, once for the workgroup. Bound by the matrix cores and the exponentials beside them: two waves share a
// SIMD (one register more than 256 leaves one: chunks of 200 to 1024 rows against 1024 to 8192, 252 us, so 173), and the one
// that multiplies goes first (166). 4 x 1024 rows against 8192, 32 heads of 128, causal: 497 us, 1.04 PFLOP/s; packed_fwd_kernel on
// bf16 caches 492. A quarter of its LDS cycles are bank conflicts, which tiles loaded directly do not have. float32 queries: 1150 us, 1.34
// PFLOP/s of their three products. bf16: probabilities enter their product as one bf16 part each, as in packed_fwd_kernel, where a
// second would add half of the products again; the output carries 0.0023 of the norm, its own rounding alone is 0.0017.
template <typename T, int HD, int QB>
__global__ void __launch_bounds__((64 * kWaves), 2) cache_fwd_kernel(CacheFwdP cp) {
  constexpr int NW = kWaves, KT = 64, KB = KT / 16, NCH = HD / 32, DB = HD / 16, R = 16 * QB * NW, P = parts_of<T>();
  __shared__ __attribute__((aligned(1024))) bf16_t ks0[KT * HD], vs0[KT * HD], ks1[KT * HD], vs1[KT * HD];
  const FwdP& p = cp.f;
  const AttnArgs& a = p.a;
  const Group G = p.G;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, j = lane >> 4;
  int slot, hk;
  xcd_slot(slot, hk);
  const Seq sq = find_seq<false>(slot, p.seq, G.G, R, a.zero_rest);
  const int rows = sq.lq * G.G, p0 = first_row(p, sq, R);
  if (p0 < 0) return;

  int pr[QB];
  int lim[QB];        // the last key that this lane's query sees
  bf16x8 qf[QB][NCH][P];
  f32x4 o[QB][DB];
  float mx[QB], ls[QB];
  const int off = sq.lk - sq.lq;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    pr[qb] = p0 + (wid * QB + qb) * 16 + r;
    const bool on = pr[qb] < rows;
    const RowAt at = packed_row(sq, hk, G, on ? pr[qb] : 0);
    lim[qb] = !on ? -1 : a.causal ? min((int)(at.t - sq.q0) + off, sq.lk - 1) : sq.lk - 1;
    const T* qp = (const T*)p.q + at.t * a.q_row + at.h * a.q_head;
#pragma unroll
    for (int c = 0; c < NCH; ++c) query_parts<T, P>(qp + 32 * c + 8 * j, on, qf[qb][c]);
    mx[qb] = kNegInf;
    ls[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[qb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const auto [k_lo, k_hi, all] = keys_of(p, sq, blockIdx.z, p.nsplit, p0, R, KT);
  const uint8_t* const kh = (const uint8_t*)p.k + sq.k0 * a.k_row + hk * a.k_head;
  const uint8_t* const vh = (const uint8_t*)p.v + sq.k0 * a.v_row + hk * a.v_head;
  const uint8_t *const ek = cp.ek + hk * a.total_k + sq.k0, *const ev = cp.ev + hk * a.total_k + sq.k0;
  ByteTile<HD, KT, NW> kt, vt;
  auto load = [&](int t0) __attribute__((always_inline)) {
    kt.load(kh, a.k_row, ek, t0, sq.lk, wid, lane);
    vt.load(vh, a.v_row, ev, t0, sq.lk, wid, lane);
  };
  int odd_key = INT32_MAX;   // the first key with a v that is not finite, from the diagonal's tiles
  auto step = [&](auto mask, int t0, bf16_t* kc, bf16_t* vc, bf16_t* kn, bf16_t* vn) __attribute__((always_inline)) {
    __syncthreads();
    if constexpr (decltype(mask)::value) {
      if (a.causal) {
        const int x = clear_tile<bf16_t, HD, KT, false>(vc);
        odd_key = x < KT ? min(odd_key, t0 + x) : odd_key;
      }
    }
    const bool more = t0 + KT < k_hi;
    if (more) load(t0 + KT);
    f32x4 s[QB][KB];
    __builtin_amdgcn_s_setprio(1);
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
    __builtin_amdgcn_s_setprio(0);
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
        to_parts<P>(v8, pf[qb][kp]);
      }
    }
    __builtin_amdgcn_s_setprio(1);
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
    __builtin_amdgcn_s_setprio(0);
    if (more) {     // the tile before this one has been read by every wave (the barrier)
      kt.store(kn, wid, lane);
      vt.store(vn, wid, lane);
    }
  };
  if (k_lo < k_hi) {
    load(k_lo);
    kt.store(ks0, wid, lane);
    vt.store(vs0, wid, lane);
    int t0 = k_lo;
    for (; t0 + 2 * KT <= all; t0 += 2 * KT) {
      step(std::false_type{}, t0, ks0, vs0, ks1, vs1);
      step(std::false_type{}, t0 + KT, ks1, vs1, ks0, vs0);
    }
    for (; t0 < k_hi; t0 += 2 * KT) {
      step(std::true_type{}, t0, ks0, vs0, ks1, vs1);
      if (t0 + KT < k_hi) step(std::true_type{}, t0 + KT, ks1, vs1, ks0, vs0);
    }
  }
  if (odd_key != INT32_MAX) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (odd_key <= lim[qb]) o[qb][db] *= __builtin_nanf("");
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float l = col_sum(ls[qb]);
#pragma unroll
    for (int db = 0; db < DB; ++db)
      store_row<T, HD>(p, sq, hk, blockIdx.z, pr[qb], 16 * db + 4 * j, o[qb][db], mx[qb], l, k_lo < k_hi, db == 0 && j == 0);
  }
}

// The work of a workgroup of cache_step_kernel: 16 packed rows of a sequence, a run of its keys, HW key heads.
struct StepAt {
  Seq sq;          // tile < 0: none
  int hk, split, nsplit;
};
// The grid (x tile slots, a multiple of 8; y groups of key heads; z splits) renumbered. Workgroups are dealt to the 8
// XCDs round-robin by linear id: the heads of a tile and split run on one XCD, one behind another, since a row of
// a packed cache holds them side by side. Up to 64 sequences: a sequence takes as many splits as its keys fill, of
// `chunk` keys each, and work lies without gaps (found from every lane holding one sequence), so that workgroups
// are of one size and spread over the CUs (1 stream of 131072 keys, 8 key heads of 128, where 7 of 8 workgroups of
// the grid are empty: 166 us with the gaps, 75 without). More: every sequence is cut into the same number.
__device__ __forceinline__ StepAt step_at(const CacheFwdP& cp) {
  const FwdP& p = cp.f;
  const int lane = threadIdx.x & 63;
  const unsigned ny = gridDim.y, nz = gridDim.z, lin = blockIdx.x + gridDim.x * (blockIdx.y + ny * blockIdx.z);
  const unsigned i = lin / 8, pair = i / ny * 8 + lin % 8;
  StepAt w;
  w.hk = i % ny;
  if (p.seq.S > 64) {
    w.nsplit = nz;
    w.split = pair % nz;
    w.sq = find_seq<false>(pair / nz, p.seq, p.G.G, 16, p.a.zero_rest);
    return w;
  }
  const Seq me = seq_at(p.seq, min(lane, p.seq.S - 1));
  const int tiles = ((p.a.zero_rest ? me.eq : me.lq) * p.G.G + 15) / 16;
  const int splits = max(1, min((me.lk + cp.chunk - 1) / cp.chunk, (int)nz));
  const int n = lane < p.seq.S ? tiles * splits : 0;
  int end = n;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int up = __shfl_up(end, o, 64);
    end += lane >= o ? up : 0;
  }
  const uint64_t hit = __builtin_amdgcn_ballot_w64((int)pair >= end - n && (int)pair < end);
  const int s = hit ? __builtin_ctzll(hit) : 0;
  w.sq = seq_at(p.seq, s);
  w.nsplit = __builtin_amdgcn_readlane(splits, s);
  const int at = (int)pair - __builtin_amdgcn_readlane(end - n, s);
  w.split = at % w.nsplit;
  w.sq.tile = hit ? at / w.nsplit : -1;
  return w;
}

// Few rows against long caches: the waves of a workgroup own the same 16 packed rows of HW key heads, and each
// walks its head's keys (with HW < 4 in turn with others) in tiles of 32 by itself. Keys go from memory into the registers of the matrix instructions' operand: which 8 of a
// head's values a lane multiplies at a time is free as long as queries do alike, so a lane takes 16 bytes of a key, two
// operands' worth. Values need the other index order and go through LDS as bytes (direct loads, transposing reads).
// A key's scale enters as its bytes become bf16, a value's by its probability (a power of two: no rounding more).
// Heads side by side read a packed cache's rows in long runs: 32 x 8192 keys, 8 heads of 128, 106 us (5.1 TB/s), of one
// head a workgroup 127, as fast as in a head-major cache. Bound by the bytes of the caches: 32 tokens against 64 to 8192 rows
// (324 MB) 64 us and 6 to join them, 2 against 65536 to 131072 (371 MB) 72 and 8; a copy would take 62 and 72.
template <typename T, int HD, int HW>
__global__ void __launch_bounds__(256, 2) cache_step_kernel(CacheFwdP cp) {
  constexpr int NW = kWaves, NK = NW / HW, KT = 32, ST = NK * KT, KB = 2, DB = HD / 16, NCH = HD / 32, P = parts_of<T>(), PP = probability_parts<T>();
  typedef StepTile<HD> Tile;
  constexpr int VB = KT * HD;      // bytes of a wave's value tile
  __shared__ __attribute__((aligned(1024))) uint8_t vs[2 * NW * VB];
  const FwdP& p = cp.f;
  const AttnArgs& a = p.a;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, j = lane >> 4;
  const StepAt w = step_at(cp);
  const Seq& sq = w.sq;
  const int hk = w.hk * HW + wid % HW, split = w.split;
  const int rows = sq.lq * p.G.G, p0 = first_row(p, sq, 16);
  if (p0 < 0) return;
  const bool on = p0 + r < rows;
  const RowAt at = packed_row(sq, hk, p.G, on ? p0 + r : 0);
  // the last key that this lane's query sees
  const int lim = !on ? -1 : a.causal ? min((int)(at.t - sq.q0) + sq.lk - sq.lq, sq.lk - 1) : sq.lk - 1;
  bf16x8 qf[NCH][P];
#pragma unroll
  for (int c = 0; c < NCH; ++c) query_parts<T, P>((const T*)p.q + at.t * a.q_row + at.h * a.q_head + Tile::first(c, j), on, qf[c]);
  f32x4 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
  float mx = kNegInf, ls = 0.f;
  const auto [k_lo, k_hi, all] = keys_of(p, sq, split, w.nsplit, p0, 16, KT);

  const uint8_t* const kh = (const uint8_t*)p.k + sq.k0 * a.k_row + hk * a.k_head;
  const uint8_t* const vh = (const uint8_t*)p.v + sq.k0 * a.v_row + hk * a.v_head;
  const uint8_t *const ek = cp.ek + hk * a.total_k + sq.k0, *const ev = cp.ev + hk * a.total_k + sq.k0;
  uint8_t *const v0 = vs + wid * VB, *const v1 = vs + (NW + wid) * VB;
  Tile k0, k1;
  auto issue = [&](int t0, Tile& kt, uint8_t* vt) __attribute__((always_inline)) {
    byte_tile_issue<HD>(vt, vh, a.v_row, t0, sq.lk, lane);
    kt.load(kh, a.k_row, ek, ev, t0, sq.lk, r, j);
  };
  int odd_key = INT32_MAX;   // the first key with a v that is NaN, from the diagonal's tiles
  auto step = [&](auto mask, int t0, const Tile& kc, uint8_t* vc, Tile& kn, uint8_t* vn) __attribute__((always_inline)) {
    vm_drain();
    wave_sync();
    if constexpr (decltype(mask)::value) {
      if (a.causal) {
        const int x = clear_bytes<HD>(vc, lane);
        odd_key = x < KT ? min(odd_key, t0 + x) : odd_key;
      }
    }
    if (t0 + ST < k_hi) issue(t0 + ST, kn, vn);
    f32x4 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const float sc = __uint_as_float((uint32_t)kc.ek[kb] << 23);
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const bf16x8 kf = e4m3_chunk(kc.chunk(kb, c), sc);
#pragma unroll
        for (int x = P - 1; x >= 0; --x)      // the small parts first
          s[kb] = mma(kf, qf[c][x], c == 0 && x == P - 1 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[kb]);
      }
    }
    float tmax = kNegInf;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (decltype(mask)::value) s[kb][i] = t0 + kb * 16 + 4 * j + i <= lim ? s[kb][i] : kNegInf;
        tmax = fmaxf(tmax, s[kb][i]);
      }
    // the reference maximum moves only when a score exceeds it by 2^kRescale
    if (__builtin_amdgcn_ballot_w64(tmax * p.sl2 > mx + kRescale)) {
      tmax = col_max(tmax) * p.sl2;
      const bool raise = tmax > mx + kRescale;
      const float mnew = raise ? tmax : mx;
      const float alpha = raise ? fast_exp2(mx - mnew) : 1.0f;
      mx = mnew;
      ls *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
    }
    const float mref = mx == kNegInf ? 0.f : mx;
    float v8[8];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = fast_exp2(__builtin_fmaf(s[kb][i], p.sl2, -mref));
        ls += e;
        v8[4 * kb + i] = e * __uint_as_float((kc.ev[kb] >> (8 * i) & 0xff) << 23);
      }
    bf16x8 pf[PP];
    to_parts<PP>(v8, pf);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const bf16x8 vf = e4m3_chunk(byte_cols<HD>(vc, db, r, j), 1.f);
#pragma unroll
      for (int x = PP - 1; x >= 0; --x) o[db] = mma(vf, pf[x], o[db]);
    }
  };
  const int k_first = k_lo + wid / HW * KT;
  if (k_first < k_hi) {
    issue(k_first, k0, v0);
    int t0 = k_first;
    for (; t0 + ST + KT <= all; t0 += 2 * ST) {
      step(std::false_type{}, t0, k0, v0, k1, v1);
      step(std::false_type{}, t0 + ST, k1, v1, k0, v0);
    }
    for (; t0 < k_hi; t0 += 2 * ST) {
      step(std::true_type{}, t0, k0, v0, k1, v1);
      if (t0 + ST < k_hi) step(std::true_type{}, t0 + ST, k1, v1, k0, v0);
    }
  }
  if (odd_key <= lim) {
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] *= __builtin_nanf("");
  }
  // the results of a head's waves are joined in the place of the value tiles
  __shared__ float2 mls[NW][16];
  const float l = col_sum(ls);
  __syncthreads();   // every wave has read its last tile
  static_assert(NW * 16 * HD * 4 <= sizeof(vs), "the waves' results in the value tiles' place");
  float* const all_o = reinterpret_cast<float*>(vs);
#pragma unroll
  for (int db = 0; db < DB; ++db) *join_at<HD>(all_o + wid * 16 * HD, r, 4 * db + j) = o[db];
  if (j == 0) mls[wid][r] = make_float2(mx, l);
  __syncthreads();
  for (int i = wid / HW * 64 + lane; i < 16 * (HD / 4); i += 64 * NK) {
    const int row = i / (HD / 4), c4 = i % (HD / 4);
    float m = kNegInf, sum = 0.f;
#pragma unroll
    for (int x = 0; x < NK; ++x) m = fmaxf(m, mls[x * HW + wid % HW][row].x);
    const float mref = m == kNegInf ? 0.f : m;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = wid % HW; x < NW; x += HW) {
      const float f = fast_exp2(mls[x][row].x - mref);
      sum += f * mls[x][row].y;
      v += f * *join_at<HD>(all_o + x * 16 * HD, row, c4);
    }
    store_row<T, HD>(p, sq, hk, split, p0 + row, 4 * c4, v, m, sum, k_lo < k_hi, c4 == 0);
    // the splits that the sequence does not have
    if (split == 0 && c4 == 0 && p0 + row < rows) {
      const RowAt at = packed_row(sq, hk, p.G, p0 + row);
      for (int z = w.nsplit; z < p.nsplit; ++z) p.ml[((long long)z * a.total_q + at.t) * a.heads + at.h] = make_float2(kNegInf, 0.f);
    }
  }
}

// Joins the splits of a row: o = sum_z 2^(m_z - m) o_z / sum_z 2^(m_z - m) l_z. 256 threads to a (query row, head):
// HD / 4 columns by groups of splits, each taking every NG-th, joined in LDS in order.
template <typename T, int HD>
__global__ void __launch_bounds__(256) cache_join_kernel(FwdP p) {
  constexpr int TPR = HD / 4, NG = 256 / TPR;
  __shared__ __attribute__((aligned(16))) float acc_s[NG][HD];
  __shared__ float2 ml_s[NG];
  const AttnArgs& a = p.a;
  const long long row = blockIdx.x;
  const int c = 4 * (threadIdx.x % TPR), g = threadIdx.x / TPR;
  const long long t = row / a.heads;
  const int h = (int)(row - t * a.heads);
  const bool in = t < p.seq.cu_q[a.seqs];
  if (!in && !a.zero_rest) return;      // the whole workgroup
  float m = kNegInf, l = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  if (in) {
    const long long per = a.total_q * a.heads;
    constexpr int U = 8;     // splits in flight
    for (int z0 = g; z0 < p.nsplit; z0 += U * NG) {
      float2 ml[U];
      f32x4 part[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long at = min(z0 + u * NG, p.nsplit - 1) * per + row;
        ml[u] = p.ml[at];
        part[u] = *reinterpret_cast<const f32x4*>(p.part + at * HD + c);
      }
      float mn = m;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (z0 + u * NG >= p.nsplit || ml[u].y == 0.f) ml[u] = make_float2(kNegInf, 0.f);
        mn = fmaxf(mn, ml[u].x);
      }
      const float mref = mn == kNegInf ? 0.f : mn, w0 = fast_exp2(m - mref);
      m = mn;
      l *= w0;
      acc *= w0;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w1 = fast_exp2(ml[u].x - mref);
        l += w1 * ml[u].y;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += ml[u].y == 0.f ? 0.f : w1 * part[u][e];   // saw nothing: not written
      }
    }
  }
  *reinterpret_cast<f32x4*>(&acc_s[g][c]) = acc;
  if (c == 0) ml_s[g] = make_float2(m, l);
  __syncthreads();
  if (g != 0) return;
#pragma unroll
  for (int x = 0; x < NG; ++x) m = fmaxf(m, ml_s[x].x);
  const float mref = m == kNegInf ? 0.f : m;
  f32x4 v{0.f, 0.f, 0.f, 0.f};
  l = 0.f;
#pragma unroll
  for (int x = 0; x < NG; ++x) {
    const float w = fast_exp2(ml_s[x].x - mref);
    l += w * ml_s[x].y;
    const f32x4 u = *reinterpret_cast<const f32x4*>(&acc_s[x][c]);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += w * u[e];
  }
  const bool any = !(l == 0.f);
  store4((T*)p.o + t * a.o_row + h * a.o_head + c, any ? v : f32x4{0.f, 0.f, 0.f, 0.f}, any ? 1.0f / l : 0.f);
  if (c == 0) p.lse[h * a.total_q + t] = any ? (m + log2f(l)) * kLn2 : kNegInf;
}

// ---- host ----

// float32 rows take three parts of registers: 16 rows a wave.
constexpr int cache_qb(bool bf16) { return bf16 ? 2 : 1; }

// Key heads that a workgroup of cache_step_kernel takes side by side.
int step_heads(const AttnArgs& a) { return a.kv_heads % 4 == 0 ? 4 : a.kv_heads % 2 == 0 ? 2 : 1; }

// How the attention runs: cache_step_kernel (split) where a sequence has 32 packed rows or fewer on average, or the
// tiles of cache_fwd_kernel would leave half of the CUs idle; and splits of the key axis, with at least 256 keys of
// an average sequence each. The lengths are on the device: a cache counts with its capacity.
// cache_step_kernel: as many workgroups as are resident (three to a CU): 32 tokens against caches of 64 to 8192 rows,
// 8 key heads of 128, 512 workgroups: 78 us, 768: 69.5, 1024: 73.8, 2048: 76; with caches of 8192 filled to 1000: 44, 30, 28, 22.
// At most 256 splits: 2 tokens against 65536 to 131072 rows, 128: 84 us, 256: 79.
FwdPlan cache_plan(const AttnArgs& a) {
  const long long rows = a.total_q * a.group();
  const long long avg_k = a.total_k / a.seqs;
  const int R = 16 * cache_qb(a.bf16) * kWaves;
  auto wgs = [&](int r) { return std::max<long long>((rows + r - 1) / r, a.seqs) * a.kv_heads; };
  FwdPlan f;
  f.split = rows <= 32LL * a.seqs || wgs(R) < 128;
  const long long n = f.split ? 768LL * step_heads(a) / wgs(16) : 512 / wgs(R);
  f.nsplit = (int)std::max<long long>(std::min<long long>(std::min<long long>(n, avg_k / 256), f.split ? 256 : 64), 1);
  return f;
}

template <typename T, int HD>
hipError_t cache_attn(const CacheFwdP& p, bool split, hipStream_t st) {
  const AttnArgs& a = p.f.a;
  constexpr int QB = cache_qb(sizeof(T) == 2);
  auto grid = [&](int R) { return dim3(tile_slots(a.total_q, a.group(), R, a.seqs), a.kv_heads, p.f.nsplit); };
  if (split) {
    dim3 g = grid(16);
    const int hw = step_heads(a);
    g.y /= hw;
    if (hw == 4)
      cache_step_kernel<T, HD, 4><<<g, 64 * kWaves, 0, st>>>(p);
    else if (hw == 2)
      cache_step_kernel<T, HD, 2><<<g, 64 * kWaves, 0, st>>>(p);
    else
      cache_step_kernel<T, HD, 1><<<g, 64 * kWaves, 0, st>>>(p);
  } else {
    cache_fwd_kernel<T, HD, QB><<<grid(16 * QB * kWaves), 64 * kWaves, 0, st>>>(p);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.f.nsplit == 1) return e;
  cache_join_kernel<T, HD><<<(unsigned)(a.total_q * a.heads), 256, 0, st>>>(p.f);
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

// A grid's x times its 256 threads, and its workgroups (numbered in 32 bits), stay below 2^32.
bool cache_attention_fits(const AttnArgs& a) {
  const FwdPlan f = cache_plan(a);
  const unsigned long long x = tile_slots(a.total_q, a.group(), f.split ? 16 : 16 * cache_qb(a.bf16) * kWaves, a.seqs);
  return x < 1u << 24 && x * (a.kv_heads / (f.split ? step_heads(a) : 1)) * f.nsplit < 1ull << 32;
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
              ek, ev, std::max((int)((a.total_k / a.seqs + f.nsplit - 1) / f.nsplit + 63) / 64 * 64, 64)};
  if (f.nsplit > 1) {
    p.f.part = (float*)ws;
    p.f.ml = (float2*)((char*)ws + align256((size_t)f.nsplit * a.total_q * a.heads * a.hd * sizeof(float)));
  }
  return BSA_CACHE_DISPATCH(cache_attn, a, p, f.split, st);
}

}  // namespace bsa
