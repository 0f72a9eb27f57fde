// Packed attention: sequences of different lengths one behind another, grouped heads, causal or
// not. Sequence s has the query rows [cu_q[s], cu_q[s + 1]) and the key rows [cu_k[s],
// cu_k[s] + len_k); with S = scale q k^T over the keys a query may see, P = softmax(S):
//   o = P v, lse = log sum exp S;   D = rowsum(dO o), dS = P (dO v^T - D),
//   dq = scale dS k, dk = scale dS^T q, dv = P^T dO, dk and dv summed over a key head's group.
// A row that sees no key has o = 0, lse = -inf and no gradient.
//
// The G = heads / kv_heads query heads of a key head share its tiles: a sequence has len_q G
// packed rows (row p = query p / G, head p % G of the group), so grouped heads, single tokens
// and the sum over the group need no separate code, and one read of a key tile serves them all.
// A query-major pass forms o (and dq), a key-major pass dk and dv; no atomics, every sum in a
// fixed order.
//
// The scores are formed transposed (S^T = K Q^T on 16 x 16 tiles, a lane owns a query column),
// so that probabilities are already laid out as the operand of the next product.
//
// Lengths live on the device, so the grid covers the most tiles there can be: sequence s takes
// tile slots floor(cu[s] G / rows) + s and on, which is monotone and never less than it needs; a
// workgroup finds its sequence by a 64-way search and leaves when its tile is empty.
#include "dense_packed.hpp"

namespace bsa {
namespace {

// As TileLoad, for packed rows r0 + [0, ROWS) (rows of them, > 0).
template <typename T, int HD, int ROWS, int NW>
struct PackedLoad {
  static constexpr int E = 16 / (int)sizeof(T), CPR = HD / E, NI = ROWS * CPR / 64;
  static_assert(NI % NW == 0, "tile / wave split");
  __device__ __forceinline__ static void issue(T* lds, const T* g, long long row_ld, long long head_ld, const Seq& sq,
                                               int hk, const Group& G, int r0, int rows, int wid, int lane) {
#pragma unroll
    for (int u = 0; u < NI / NW; ++u) {
      const int blk = wid * (NI / NW) + u, idx = blk * 64 + lane;
      const int row = idx / CPR, c = (idx % CPR) ^ tswz<T, HD>(row);
      const RowAt at = packed_row(sq, hk, G, min(r0 + row, rows - 1));
      load_lds16(g + at.t * row_ld + at.h * head_ld + E * c, lds + blk * 64 * E);
    }
  }
};

// ---- forward ----

template <typename T, int HD, int QB, bool SPLIT>
__global__ void __launch_bounds__((64 * Share<T, HD, SPLIT>::NW)) packed_fwd_kernel(FwdP p) {
  typedef Share<T, HD, SPLIT> SH;
  static_assert(!SPLIT || QB == 1, "one block of rows");
  constexpr int KT = SH::tile, KB = KT / 16, NCH = HD / 32, DB = HD / 16, R = 16 * QB * (SPLIT ? 1 : SH::NW), ST = SH::step;
  typedef typename Chunk<T>::type CT;
  __shared__ __attribute__((aligned(1024))) T ks0a[SH::elems], vs0a[SH::elems], ks1a[SH::elems], vs1a[SH::elems];
  const AttnArgs& a = p.a;
  const Group G = p.G;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, j = lane >> 4;
  int slot, hk;
  xcd_slot(slot, hk);
  const Seq sq = find_seq<false>(slot, p.seq, G.G, R, a.zero_rest);
  const int rows = sq.lq * G.G, ext = sq.eq * G.G;
  // tiles in descending order: with a causal mask the longest rows come first
  const int nt = (rows + R - 1) / R;
  const long long tile = sq.tile < nt ? nt - 1 - sq.tile : sq.tile;
  if (tile < 0 || tile * R >= ext) return;
  const int p0 = (int)tile * R;
  if (p0 >= ext || (p0 >= rows && (!a.zero_rest || p.nsplit > 1))) return;
  T* const out = (T*)p.o;

  int pr[QB];
  int lim[QB];        // the last key that this lane's query sees
  CT qf[QB][NCH];
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
    for (int c = 0; c < NCH; ++c) qf[qb][c] = on ? load_chunk(qp + 32 * c + 8 * j) : zero_chunk(CT{});
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

  const T* const kh = (const T*)p.k + sq.k0 * a.k_row + hk * a.k_head;
  const T* const vh = (const T*)p.v + sq.k0 * a.v_row + hk * a.v_head;
  const int lw = SPLIT ? 0 : wid, own = SPLIT ? wid * KT * HD : 0;
  T *const ks0 = ks0a + own, *const vs0 = vs0a + own, *const ks1 = ks1a + own, *const vs1 = vs1a + own;
  auto issue = [&](int t0, T* kd, T* vd) __attribute__((always_inline)) {
    TileLoad<T, HD, KT, SH::LW>::issue(kd, kh, a.k_row, t0, sq.lk, lw, lane);
    TileLoad<T, HD, KT, SH::LW>::issue(vd, vh, a.v_row, t0, sq.lk, lw, lane);
  };
  int odd_key = INT32_MAX;   // the first key with a v that is not finite, from the diagonal's tiles
  auto step = [&](auto mask, int t0, T* kc, T* vc, T* kn, T* vn) __attribute__((always_inline)) {
    tile_ready<SPLIT>();
    if constexpr (decltype(mask)::value) {
      if (a.causal) {
        const int x = clear_tile<T, HD, KT, SPLIT>(vc);
        odd_key = x < KT ? min(odd_key, t0 + x) : odd_key;
      }
    }
    if (t0 + ST < k_hi) issue(t0 + ST, kn, vn);
    f32x4 s[QB][KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        const CT kf = row_frag<HD>(kc, kb * 16 + r, 4 * c + j);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
          s[qb][kb] = mma(kf, qf[qb][c], c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[qb][kb]);
      }
    CT pf[QB][KB / 2];
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
        pf[qb][kp] = make_chunk<T>(v8);
      }
    }
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int kp = 0; kp < KB / 2; ++kp) {
        const CT vf = col_frag<HD>(vc, 32 * kp, 16 * db, lane);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) o[qb][db] = mma(vf, pf[qb][kp], o[qb][db]);
      }
  };
  const int k_first = k_lo + (SPLIT ? wid * KT : 0);
  if (k_first < k_hi) {
    issue(k_first, ks0, vs0);
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
    __shared__ float2 mls[SH::NW][16];
    const float l = col_sum(ls[0]);
    __syncthreads();   // every wave has read its last tile
    static_assert(SH::NW * 16 * HD * 4 <= SH::elems * sizeof(T), "the waves' results in a staged tensor's place");
    float* const mine = reinterpret_cast<float*>(ks0a) + wid * 16 * HD;
#pragma unroll
    for (int db = 0; db < DB; ++db) *join_at<HD>(mine, r, 4 * db + j) = o[0][db];
    if (j == 0) mls[wid][r] = make_float2(mx[0], l);
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * (HD / 4); i += 64 * SH::NW) {
      const int row = i / (HD / 4), c4 = i % (HD / 4);
      float m = kNegInf, sum = 0.f;
#pragma unroll
      for (int w = 0; w < SH::NW; ++w) m = fmaxf(m, mls[w][row].x);
      const float mref = m == kNegInf ? 0.f : m;
      f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < SH::NW; ++w) {
        const float f = fast_exp2(mls[w][row].x - mref);
        sum += f * mls[w][row].y;
        v += f * *join_at<HD>(reinterpret_cast<float*>(ks0a) + w * 16 * HD, row, c4);
      }
      store(p0 + row, 4 * c4, v, m, sum, c4 == 0);
    }
  }
}

// ---- backward ----

struct BwdP {
  AttnArgs a;
  const void *q, *k, *v, *o, *d_o;
  const float* lse;
  SeqArgs seq;
  Group G;
  void *dq, *dk, *dv;
  float2* terms;     // [kv_heads][total_q G] packed rows: lse in log2 units (+inf: sees nothing), D
  float sl2;
};

// dq, and each row's terms for the key-major pass. D comes from the output as it was rounded to
// bf16, and an error e of D is common to a row's keys: where few keys carry a row dP - D cancels,
// and e dominates (scores with a deviation of 9: dq and dk were off by 0.005 of their norm, three
// times the rounding of the result). But sum P (dP - D) = -e is summed beside, in float32: with M =
// sum P k, which takes one product more, dq = scale (sum P (dP - D) k - sum P (dP - D) M), and the
// key-major pass gets D + sum P (dP - D).
template <typename T, int HD, int QB, bool SPLIT>
__global__ void __launch_bounds__((64 * Share<T, HD, SPLIT>::NW), (!SPLIT && HD == 128 ? 2 : 1)) packed_dq_kernel(BwdP p) {
  typedef Share<T, HD, SPLIT> SH;
  static_assert(!SPLIT || QB == 1, "one block of rows");
  constexpr int KT = SH::tile, NCH = HD / 32, DB = HD / 16, R = 16 * QB * (SPLIT ? 1 : SH::NW), ST = SH::step;
  typedef typename Chunk<T>::type CT;
  __shared__ __attribute__((aligned(1024))) T ks0a[SH::elems], vs0a[SH::elems], ks1a[SH::elems], vs1a[SH::elems];
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
  if (p0 >= ext || (p0 >= rows && !a.zero_rest)) return;

  int pr[QB];
  int lim[QB];
  CT qf[QB][NCH], df[QB][NCH];
  constexpr bool FIX = sizeof(T) == 2;   // float32 outputs are exact enough
  f32x4 acc[QB][DB], mean[FIX ? QB : 1][DB];
  float l2[QB], dd[QB], e[QB];
  const int off = sq.lk - sq.lq;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    pr[qb] = p0 + ((SPLIT ? 0 : wid * QB) + qb) * 16 + r;
    const bool on = pr[qb] < rows;
    const RowAt at = packed_row(sq, hk, G, on ? pr[qb] : 0);
    lim[qb] = !on ? -1 : a.causal ? min((int)(at.t - sq.q0) + off, sq.lk - 1) : sq.lk - 1;
    const T* qp = (const T*)p.q + at.t * a.q_row + at.h * a.q_head;
    const T* dp = (const T*)p.d_o + at.t * a.do_row + at.h * a.do_head;
    const T* op = (const T*)p.o + at.t * a.o_row + at.h * a.o_head;
    float d = 0.f;
    bool odd = false;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      qf[qb][c] = zero_chunk(CT{});
      df[qb][c] = zero_chunk(CT{});
      if (on && lim[qb] >= 0) {
        qf[qb][c] = load_chunk(qp + 32 * c + 8 * j);
        df[qb][c] = load_chunk(dp + 32 * c + 8 * j);
        const CT of = load_chunk(op + 32 * c + 8 * j);
        odd |= odd_chunk(qf[qb][c]) || odd_chunk(df[qb][c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) d = fmaf((float)df[qb][c][e], (float)of[e], d);
      }
    }
    dd[qb] = col_sum(d);
    l2[qb] = on && lim[qb] >= 0 ? p.lse[at.h * a.total_q + at.t] * kLog2e : __builtin_huge_valf();
    // a row whose q or dO is not finite: the key-major pass, which clears it, gets its NaN from here
    if (col_max(odd ? 1.f : 0.f) != 0.f) l2[qb] = __builtin_nanf("");
    e[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      acc[qb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (FIX) mean[qb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  const int plast = min(p0 + R, rows) - 1;
  const int k_hi = p0 >= rows ? 0 : a.causal ? max(min(sq.lk, G.div(plast) + off + 1), 0) : sq.lk;
  const int all = min(a.causal ? max(G.div(min(p0, rows)) + off + 1, 0) : sq.lk, k_hi);

  const T* const kh = (const T*)p.k + sq.k0 * a.k_row + hk * a.k_head;
  const T* const vh = (const T*)p.v + sq.k0 * a.v_row + hk * a.v_head;
  const int lw = SPLIT ? 0 : wid, own = SPLIT ? wid * KT * HD : 0;
  T *const ks0 = ks0a + own, *const vs0 = vs0a + own, *const ks1 = ks1a + own, *const vs1 = vs1a + own;
  auto issue = [&](int t0, T* kd, T* vd) __attribute__((always_inline)) {
    TileLoad<T, HD, KT, SH::LW>::issue(kd, kh, a.k_row, t0, sq.lk, lw, lane);
    TileLoad<T, HD, KT, SH::LW>::issue(vd, vh, a.v_row, t0, sq.lk, lw, lane);
  };
  int odd_key = INT32_MAX;   // the first key with a k that is not finite, from the diagonal's tiles
  auto step = [&](auto mask, int t0, T* kc, T* vc, T* kn, T* vn) __attribute__((always_inline)) {
    tile_ready<SPLIT>();
    if constexpr (decltype(mask)::value) {
      if (a.causal) {
        const int x = clear_tile<T, HD, KT, SPLIT>(kc);
        odd_key = x < KT ? min(odd_key, t0 + x) : odd_key;
      }
    }
    if (t0 + ST < k_hi) issue(t0 + ST, kn, vn);
#pragma unroll
    for (int kp = 0; kp < KT / 32; ++kp) {
      f32x4 s[QB][2], g[QB][2];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
          const CT kf = row_frag<HD>(kc, kp * 32 + kb * 16 + r, 4 * c + j);
          const CT vf = row_frag<HD>(vc, kp * 32 + kb * 16 + r, 4 * c + j);
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) {
            s[qb][kb] = mma(kf, qf[qb][c], c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[qb][kb]);
            g[qb][kb] = mma(vf, df[qb][c], c == 0 ? f32x4{-dd[qb], -dd[qb], -dd[qb], -dd[qb]} : g[qb][kb]);
          }
        }
      CT ds[QB], pf[QB];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float v8[8], p8[8];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float pv = fast_exp2(__builtin_fmaf(s[qb][kb][i], p.sl2, -l2[qb]));
            const float x = pv * g[qb][kb][i];
            const bool see = !decltype(mask)::value || t0 + kp * 32 + kb * 16 + 4 * j + i <= lim[qb];
            v8[4 * kb + i] = see ? x : 0.f;
            p8[4 * kb + i] = see ? pv : 0.f;
            if constexpr (FIX) e[qb] += v8[4 * kb + i];
          }
        ds[qb] = make_chunk<T>(v8);
        if constexpr (FIX) pf[qb] = make_chunk<T>(p8);
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const CT kt = col_frag<HD>(kc, 32 * kp, 16 * db, lane);
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          acc[qb][db] = mma(kt, ds[qb], acc[qb][db]);
          if constexpr (FIX) mean[qb][db] = mma(kt, pf[qb], mean[qb][db]);
        }
      }
    }
  };
  const int k_first = SPLIT ? wid * KT : 0;
  if (k_first < k_hi) {
    issue(k_first, ks0, vs0);
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
  if constexpr (FIX) {
    // (here: with a NaN put into acc, as for float32, the loop above was scheduled worse, 360 -> 460 us at d = 64)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) e[qb] = odd_key <= lim[qb] ? __builtin_nanf("") : e[qb];
    if constexpr (SPLIT) {   // the sum over the waves, in each of them
      __shared__ float es[SH::NW][16];
      e[0] = col_sum(e[0]);
      if (j == 0) es[wid][r] = e[0];
      __syncthreads();
      e[0] = es[0][r];
#pragma unroll
      for (int w = 1; w < SH::NW; ++w) e[0] += es[w][r];
    } else {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) e[qb] = col_sum(e[qb]);
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int db = 0; db < DB; ++db) acc[qb][db] -= e[qb] * mean[qb][db];
  }
  if constexpr (!FIX) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        if (odd_key <= lim[qb]) acc[qb][db] *= __builtin_nanf("");
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
    if (pr[qb] < rows && j == 0 && (!SPLIT || wid == 0))
      p.terms[((long long)hk * a.total_q + sq.q0) * G.G + pr[qb]] = make_float2(l2[qb], dd[qb] + e[qb]);
  auto store = [&](int row, int c, f32x4 v) {
    if (row >= ext || (row >= rows && !a.zero_rest)) return;
    const RowAt at = packed_row(sq, hk, G, row);
    // (a row of no sequence summed products of its zeros: NaN beside a key that is not finite)
    store4((T*)p.dq + (at.t * a.heads + at.h) * HD + c, row < rows ? v : f32x4{0.f, 0.f, 0.f, 0.f}, a.scale);
  };
  if constexpr (!SPLIT) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int db = 0; db < DB; ++db) store(pr[qb], 16 * db + 4 * j, acc[qb][db]);
  } else {
    join_sum<HD, SH::NW>(reinterpret_cast<float*>(ks0a), acc[0], [&](int row, int c, f32x4 v) { store(p0 + row, c, v); });
  }
}

// dk and dv of 16 KW keys per wave (a lane owns a key column, S = Q K^T), over the packed query
// rows that see them, in tiles of KT rows.
template <typename T, int HD, int KW, bool SPLIT>
__global__ void __launch_bounds__((64 * Share<T, HD, SPLIT>::NW)) packed_dkv_kernel(BwdP p) {
  typedef Share<T, HD, SPLIT> SH;
  static_assert(!SPLIT || KW == 1, "one block of keys");
  constexpr int QT = SH::tile, NCH = HD / 32, DB = HD / 16, R = 16 * KW * (SPLIT ? 1 : SH::NW), ST = SH::step;
  constexpr int TM = (SPLIT ? SH::NW : 1) * 2 * QT;
  typedef typename Chunk<T>::type CT;
  __shared__ __attribute__((aligned(1024))) T qs0a[SH::elems], ds0a[SH::elems], qs1a[SH::elems], ds1a[SH::elems];
  __shared__ __attribute__((aligned(16))) float tm0a[TM], tm1a[TM];   // lse, then -D, of a tile's rows
  const AttnArgs& a = p.a;
  const Group G = p.G;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, j = lane >> 4;
  int slot, hk;
  xcd_slot(slot, hk);
  const Seq sq = find_seq<true>(slot, p.seq, 1, R, a.zero_rest);
  const long long k0 = sq.tile * R;
  if (k0 < 0 || k0 >= sq.ek || (k0 >= sq.lk && !a.zero_rest)) return;
  const int rows = sq.lq * G.G;
  const int off = sq.lk - sq.lq;

  int key[KW];
  int first[KW];           // the first packed row that sees this lane's key
  CT kf[KW][NCH], vf[KW][NCH];
  f32x4 dk[KW][DB], dv[KW][DB];
#pragma unroll
  for (int w = 0; w < KW; ++w) {
    key[w] = (int)k0 + ((SPLIT ? 0 : wid * KW) + w) * 16 + r;
    const bool on = key[w] < sq.lk;
    first[w] = !on ? rows : a.causal ? max(key[w] - off, 0) * G.G : 0;
    const long long row = sq.k0 + (on ? key[w] : 0);
    const T* kp = (const T*)p.k + row * a.k_row + hk * a.k_head;
    const T* vp = (const T*)p.v + row * a.v_row + hk * a.v_head;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      kf[w][c] = on ? load_chunk(kp + 32 * c + 8 * j) : zero_chunk(CT{});
      vf[w][c] = on ? load_chunk(vp + 32 * c + 8 * j) : zero_chunk(CT{});
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      dk[w][db] = f32x4{0.f, 0.f, 0.f, 0.f};
      dv[w][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  // Rows from here on see every key of the workgroup. Only the causal diagonal is masked: rows
  // behind the sequence's last repeat it with an lse of +inf (P = 0), and what keys behind its end
  // sum up is not stored.
  const int all = a.causal ? max((int)min(k0 + R, (long long)sq.lk) - 1 - off, 0) * G.G : 0;
  const int p_lo = k0 >= sq.lk ? rows : a.causal ? max((int)k0 - off, 0) * G.G / QT * QT : 0;

  const int lw = SPLIT ? 0 : wid, own = SPLIT ? wid * QT * HD : 0, tid = SPLIT ? lane : threadIdx.x;
  T *const qs0 = qs0a + own, *const ds0 = ds0a + own, *const qs1 = qs1a + own, *const ds1 = ds1a + own;
  float *const tm0 = tm0a + (SPLIT ? wid * 2 * QT : 0), *const tm1 = tm1a + (SPLIT ? wid * 2 * QT : 0);
  // tile rows are packed rows: query and head vary by row
  auto issue = [&](int t0, T* qd, T* dd, float* td) __attribute__((always_inline)) {
    PackedLoad<T, HD, QT, SH::LW>::issue(qd, (const T*)p.q, a.q_row, a.q_head, sq, hk, G, t0, rows, lw, lane);
    PackedLoad<T, HD, QT, SH::LW>::issue(dd, (const T*)p.d_o, a.do_row, a.do_head, sq, hk, G, t0, rows, lw, lane);
    if (tid < QT) {
      const float2 t = t0 + tid < rows ? p.terms[((long long)hk * a.total_q + sq.q0) * G.G + t0 + tid]
                                       : make_float2(__builtin_huge_valf(), 0.f);
      td[tid] = t.x;
      td[QT + tid] = -t.y;
    }
  };
  auto step = [&](auto mask, int t0, T* qc, T* dc, const float* tc, T* qn, T* dn, float* tn) __attribute__((always_inline)) {
    tile_ready<SPLIT>();
    if constexpr (decltype(mask)::value) {   // masked tiles are the causal diagonal's
      clear_tile<T, HD, QT, SPLIT>(qc);      // keys that such a row sees get NaN from its lse
      clear_tile<T, HD, QT, SPLIT>(dc);
    }
    if (t0 + ST < rows) issue(t0 + ST, qn, dn, tn);
    f32x4 s[KW][2], g[KW][2];
    CT pf[KW], sf[KW];
    auto scores = [&](int qp) __attribute__((always_inline)) {
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) {
        const f32x4 nd = *reinterpret_cast<const f32x4*>(tc + QT + qp * 32 + qb * 16 + 4 * j);
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
          const CT qf = row_frag<HD>(qc, qp * 32 + qb * 16 + r, 4 * c + j);
          const CT df = row_frag<HD>(dc, qp * 32 + qb * 16 + r, 4 * c + j);
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            s[w][qb] = mma(qf, kf[w][c], c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[w][qb]);
            g[w][qb] = mma(df, vf[w][c], c == 0 ? nd : g[w][qb]);
          }
        }
      }
    };
    auto probs = [&](int qp) __attribute__((always_inline)) {
      f32x4 l2[2];
#pragma unroll
      for (int qb = 0; qb < 2; ++qb) l2[qb] = *reinterpret_cast<const f32x4*>(tc + qp * 32 + qb * 16 + 4 * j);
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        float p8[8], s8[8];
#pragma unroll
        for (int qb = 0; qb < 2; ++qb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float pv = fast_exp2(__builtin_fmaf(s[w][qb][i], p.sl2, -l2[qb][i]));
            float x = pv * g[w][qb][i];
            if constexpr (decltype(mask)::value) {
              const int row = t0 + qp * 32 + qb * 16 + 4 * j + i;
              const bool see = row >= first[w];
              pv = see ? pv : 0.f;
              x = see ? x : 0.f;
            }
            p8[4 * qb + i] = pv;
            s8[4 * qb + i] = x;
          }
        pf[w] = make_chunk<T>(p8);
        sf[w] = make_chunk<T>(s8);
      }
    };
    auto grads = [&](int qp) __attribute__((always_inline)) {
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const CT dt = col_frag<HD>(dc, 32 * qp, 16 * db, lane);
        const CT qt = col_frag<HD>(qc, 32 * qp, 16 * db, lane);
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          dv[w][db] = mma(dt, pf[w], dv[w][db]);
          dk[w][db] = mma(qt, sf[w], dk[w][db]);
        }
      }
    };
#pragma unroll
    for (int qp = 0; qp < QT / 32; ++qp) {
      scores(qp);
      probs(qp);
      grads(qp);
    }
  };
  const int p_first = p_lo + (SPLIT ? wid * QT : 0);
  if (p_first < rows) {
    issue(p_first, qs0, ds0, tm0);
    int t0 = p_first;
    for (; t0 < min(all, rows); t0 += 2 * ST) {
      step(std::true_type{}, t0, qs0, ds0, tm0, qs1, ds1, tm1);
      if (t0 + ST < rows) step(std::true_type{}, t0 + ST, qs1, ds1, tm1, qs0, ds0, tm0);
    }
    for (; t0 < rows; t0 += 2 * ST) {
      step(std::false_type{}, t0, qs0, ds0, tm0, qs1, ds1, tm1);
      if (t0 + ST < rows) step(std::false_type{}, t0 + ST, qs1, ds1, tm1, qs0, ds0, tm0);
    }
  }
  auto store = [&](T* out, int k, int c, f32x4 v, float sc) {
    if (k >= sq.ek || (k >= sq.lk && !a.zero_rest)) return;
    store4(out + ((sq.k0 + k) * a.kv_heads + hk) * HD + c, k < sq.lk ? v : f32x4{0.f, 0.f, 0.f, 0.f}, sc);
  };
  if constexpr (!SPLIT) {
#pragma unroll
    for (int w = 0; w < KW; ++w)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        store((T*)p.dk, key[w], 16 * db + 4 * j, dk[w][db], a.scale);
        store((T*)p.dv, key[w], 16 * db + 4 * j, dv[w][db], 1.f);
      }
  } else {
    join_sum<HD, SH::NW>(reinterpret_cast<float*>(qs0a), dk[0],
                         [&](int row, int c, f32x4 v) { store((T*)p.dk, (int)k0 + row, c, v, a.scale); });
    join_sum<HD, SH::NW>(reinterpret_cast<float*>(ds0a), dv[0],
                         [&](int row, int c, f32x4 v) { store((T*)p.dv, (int)k0 + row, c, v, 1.f); });
  }
}

// ---- host ----

template <typename T, int HD>
hipError_t attn_fwd(FwdP p, bool split, hipStream_t st) {
  const AttnArgs& a = p.a;
  auto grid = [&](int R) { return dim3(tile_slots(a.total_q, a.group(), R, a.seqs), a.kv_heads, p.nsplit); };
  if (split)
    packed_fwd_kernel<T, HD, 1, true><<<grid(16), 64 * Share<T, HD, true>::NW, 0, st>>>(p);
  else
    packed_fwd_kernel<T, HD, kFwdQB, false><<<grid(16 * kFwdQB * kWaves), 64 * kWaves, 0, st>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.nsplit == 1) return e;
  const long long n = a.total_q * a.heads, per = 256 / (HD / 4);
  packed_join_kernel<T, HD><<<(unsigned)((n + per - 1) / per), 256, 0, st>>>(p);
  return hipGetLastError();
}

// 16-row blocks of queries, and of keys, that a wave of the backward owns.
constexpr int dq_blocks(int hd) { return hd == 128 ? 1 : 2; }
constexpr int dkv_blocks(int hd, bool bf16) { return hd == 128 || !bf16 ? 1 : 2; }

// The backward's passes SPLIT where their usual tiles would not give three workgroups to every
// four CUs.
bool dq_split(const AttnArgs& a) {
  const int R = 16 * dq_blocks(a.hd) * kWaves;
  return (a.total_q * a.group() + R - 1) / R * a.kv_heads < 192;
}
bool dkv_split(const AttnArgs& a) {
  const int R = 16 * dkv_blocks(a.hd, a.bf16) * kWaves;
  return (a.total_k + R - 1) / R * a.kv_heads < 192;
}

template <typename T, int HD>
hipError_t attn_bwd(BwdP p, hipStream_t st) {
  constexpr int QB = dq_blocks(HD), KW = dkv_blocks(HD, sizeof(T) == 2);
  constexpr int RQ = 16 * QB * kWaves, RK = 16 * KW * kWaves;
  const AttnArgs& a = p.a;
  if (a.total_q > 0) {
    auto grid = [&](int R) { return dim3(tile_slots(a.total_q, a.group(), R, a.seqs), a.kv_heads); };
    if (dq_split(a))
      packed_dq_kernel<T, HD, 1, true><<<grid(16), 64 * Share<T, HD, true>::NW, 0, st>>>(p);
    else
      packed_dq_kernel<T, HD, QB, false><<<grid(RQ), 64 * kWaves, 0, st>>>(p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.total_k > 0) {
    auto grid = [&](int R) { return dim3(tile_slots(a.total_k, 1, R, a.seqs), a.kv_heads); };
    if (dkv_split(a))
      packed_dkv_kernel<T, HD, 1, true><<<grid(16), 64 * Share<T, HD, true>::NW, 0, st>>>(p);
    else
      packed_dkv_kernel<T, HD, KW, false><<<grid(RK), 64 * kWaves, 0, st>>>(p);
    return hipGetLastError();
  }
  return hipSuccess;
}

#define BSA_ATTN_DISPATCH(FN, a, ...)                                                                       \
  ((a).bf16 ? ((a).hd == 128  ? FN<bf16_t, 128>(__VA_ARGS__)                                                \
               : (a).hd == 64 ? FN<bf16_t, 64>(__VA_ARGS__)                                                 \
                              : FN<bf16_t, 32>(__VA_ARGS__))                                                \
            : ((a).hd == 128  ? FN<float, 128>(__VA_ARGS__)                                                 \
               : (a).hd == 64 ? FN<float, 64>(__VA_ARGS__)                                                  \
                              : FN<float, 32>(__VA_ARGS__)))

}  // namespace

// The grids in x times their 256 threads (64 Share::NW at most) stay below 2^32, where a launch's limit lies.
bool attention_fwd_fits(const AttnArgs& a) {
  return tile_slots(a.total_q, a.group(), fwd_plan(a).split ? 16 : 16 * kFwdQB * kWaves, a.seqs) < 1u << 24;
}
bool attention_bwd_fits(const AttnArgs& a) {
  return tile_slots(a.total_q, a.group(), dq_split(a) ? 16 : 16 * dq_blocks(a.hd) * kWaves, a.seqs) < 1u << 24 &&
         tile_slots(a.total_k, 1, dkv_split(a) ? 16 : 16 * dkv_blocks(a.hd, a.bf16) * kWaves, a.seqs) < 1u << 24;
}

size_t attention_fwd_ws_bytes(const AttnArgs& a) {
  const int s = fwd_plan(a).nsplit;
  if (s == 1) return 0;
  const size_t rows = (size_t)s * a.total_q * a.heads;
  return align256(rows * a.hd * sizeof(float)) + align256(rows * sizeof(float2));
}

hipError_t launch_attention_fwd(const AttnArgs& a, const void* q, const void* k, const void* v, const int* cu_q,
                                const int* cu_k, const int* used_k, void* o, float* lse, void* ws, hipStream_t st) {
  if (a.total_q == 0) return hipSuccess;
  const FwdPlan f = fwd_plan(a);
  FwdP p{a, q, k, v, SeqArgs{cu_q, cu_k, used_k, a.seqs, a.total_q, a.total_k}, group_of(a), o, lse, a.scale * kLog2e,
         f.nsplit, nullptr, nullptr};
  if (p.nsplit > 1) {
    p.part = (float*)ws;
    p.ml = (float2*)((char*)ws + align256((size_t)p.nsplit * a.total_q * a.heads * a.hd * sizeof(float)));
  }
  return BSA_ATTN_DISPATCH(attn_fwd, a, p, f.split, st);
}

size_t attention_bwd_ws_bytes(const AttnArgs& a) { return align256(sizeof(float2) * (size_t)a.total_q * a.heads); }

hipError_t launch_attention_bwd(const AttnArgs& a, const void* q, const void* k, const void* v, const void* o,
                                const float* lse, const void* d_o, const int* cu_q, const int* cu_k, const int* used_k,
                                void* dq, void* dk, void* dv, void* ws, hipStream_t st) {
  BwdP p{a, q, k, v, o, d_o, lse, SeqArgs{cu_q, cu_k, used_k, a.seqs, a.total_q, a.total_k}, group_of(a), dq, dk, dv, (float2*)ws, a.scale * kLog2e};
  return BSA_ATTN_DISPATCH(attn_bwd, a, p, st);
}

}  // namespace bsa
