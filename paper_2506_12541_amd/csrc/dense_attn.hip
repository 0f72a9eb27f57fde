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
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.hpp"
#include "attn_common.hpp"
#include "dense.hpp"
#include "dense_common.hpp"

namespace bsa {
namespace {

constexpr int kWaves = 4;

struct Seq {
  int s;
  long long q0, k0;      // first query and key row
  int lq, lk;            // query and key rows
  int eq, ek;            // rows up to the next sequence's first (eq >= lq, ek >= lk)
  long long tile;        // this workgroup's tile within the sequence
};

__device__ __forceinline__ long long clampll(long long x, long long lo, long long hi) {
  return x < lo ? lo : x > hi ? hi : x;
}

struct SeqArgs {
  const int *cu_q, *cu_k, *used_k;
  int S;
  long long total_q, total_k;
};

// Offsets outside the tensors are pulled inside: no read or write leaves them.
__device__ __forceinline__ Seq seq_at(const SeqArgs& a, int s) {
  Seq q;
  q.s = s;
  q.q0 = clampll(a.cu_q[s], 0, a.total_q);
  q.k0 = clampll(a.cu_k[s], 0, a.total_k);
  q.lq = (int)(clampll(a.cu_q[s + 1], q.q0, a.total_q) - q.q0);
  q.ek = (int)(clampll(a.cu_k[s + 1], q.k0, a.total_k) - q.k0);
  q.lk = a.used_k ? (int)clampll(a.used_k[s], 0, q.ek) : q.ek;
  q.eq = q.lq;
  if (s + 1 == a.S) {
    q.eq = (int)(a.total_q - q.q0);
    q.ek = (int)(a.total_k - q.k0);
  }
  q.tile = 0;
  return q;
}

// The sequence and tile that `slot` stands for, in tiles of R packed query rows (KEYS: of R key
// rows); mult packed rows for each row of cu; rest: rows behind the sequence's are covered too.
//
// Up to 64 sequences: those with the most work a tile come first (a tile's work is the other
// side's length), found from every lane holding one sequence, so that the last workgroups to
// finish are short ones (16 clouds of 1800 to 3586 rows in rising order, 8 heads of 64: the
// key-major pass took 716 us in that order, 641 so, with the XCD numbering below). More: in their
// order, sequence s from slot floor(cu[s] mult / R) + s on, by a 64-way search.
template <bool KEYS>
__device__ __forceinline__ Seq find_seq(long long slot, const SeqArgs& a, int mult, int R, bool rest) {
  const int lane = threadIdx.x & 63;
  Seq q;
  if (a.S <= 64) {
    const Seq me = seq_at(a, min(lane, a.S - 1));
    const long long mine = KEYS ? (rest ? me.ek : me.lk) : (long long)(rest ? me.eq : me.lq) * mult;
    const int n = lane < a.S ? (int)((mine + R - 1) / R) : 0, weight = KEYS ? me.lq : me.lk;
    int before = 0;     // tiles of the sequences that come first
    for (int i = 0; i < a.S; ++i) {
      const int w = __builtin_amdgcn_readlane(weight, i), m = __builtin_amdgcn_readlane(n, i);
      before += w > weight || (w == weight && i < lane) ? m : 0;
    }
    const uint64_t hit = __builtin_amdgcn_ballot_w64(slot >= before && slot < before + n);
    if (hit == 0) {
      q = seq_at(a, 0);
      q.tile = -1;
      return q;
    }
    const int s = __builtin_ctzll(hit);
    q = seq_at(a, s);
    q.tile = slot - __builtin_amdgcn_readlane(before, s);
    return q;
  }
  const int* cu = KEYS ? a.cu_k : a.cu_q;
  int lo = 0, n = a.S;
  while (n > 1) {
    const int step = (n + 63) / 64;
    const int i = lane * step;
    const bool le = i < n && (i == 0 || (long long)cu[lo + i] * mult / R + lo + i <= slot);
    const int c = __builtin_popcountll(__builtin_amdgcn_ballot_w64(le)) - 1;
    lo += c * step;
    n = min(step, n - c * step);
  }
  q = seq_at(a, __builtin_amdgcn_readfirstlane(lo));
  q.tile = slot - ((long long)cu[q.s] * mult / R + q.s);
  return q;
}

// Workgroups are dealt to the 8 XCDs round-robin by linear id, and each XCD has its own L2: the
// grid (x tile slots, a multiple of 8; y key heads) is renumbered so that the workgroups of a key
// head run on as few XCDs as possible. A bijection for 8 k key heads or a divisor of 8; else
// the grid is kept.
__device__ __forceinline__ void xcd_slot(int& slot, int& hk) {
  const unsigned nx = gridDim.x, ny = gridDim.y, lin = blockIdx.x + nx * blockIdx.y, c = lin % 8, i = lin / 8;
  slot = blockIdx.x;
  hk = blockIdx.y;
  if (ny % 8 == 0) {
    hk = c + 8 * (i / nx);
    slot = i % nx;
  } else if (8 % ny == 0) {
    hk = c % ny;
    slot = i * (8 / ny) + c / ny;
  }
}

// How a workgroup shares its work. Usually its waves own different rows (of queries, or of keys)
// and walk tiles of the other side together. Where that leaves CUs idle or rows unused (single
// tokens against a cache, short sequences: SPLIT), its waves own the same 16 rows and each walks
// every NW-th tile of 32, staged for itself alone without a barrier; their results are joined in LDS.
template <typename T, int HD, bool SPLIT> struct Share {
  // two staged tiles of two tensors and every wave within 128 KB
  static constexpr int NW = SPLIT && sizeof(T) * HD > 256 ? 2 : kWaves;
  static constexpr int tile = SPLIT || sizeof(T) == 4 ? 32 : 64;   // rows of a staged tile
  static constexpr int LW = SPLIT ? 1 : NW;                        // waves that load a tile
  static constexpr int elems = (SPLIT ? NW : 1) * tile * HD;       // of one staged tensor
  static constexpr int step = SPLIT ? NW * tile : tile;            // rows from a wave's tile to its next
};

// The next tile may be read: every wave's part of it has landed.
template <bool SPLIT>
__device__ __forceinline__ void tile_ready() {
  vm_drain();
  if constexpr (SPLIT)
    wave_sync();
  else
    __syncthreads();
}

// 16 x HD float32 results of one wave in transposed accumulators (lane: row lane % 16, columns 16 db +
// 4 (lane / 16) + i), row-major in LDS; columns are swizzled by row against bank conflicts.
template <int HD>
__device__ __forceinline__ f32x4* join_at(float* m, int row, int c4) {
  return reinterpret_cast<f32x4*>(m + row * HD + 4 * (c4 ^ (row & (HD / 4 - 1))));
}

// The sum of the NW waves' results (at m, NW x 16 x HD floats), in order, four columns at a time.
template <int HD, int NW, typename F>
__device__ __forceinline__ void join_sum(float* m, const f32x4 (&acc)[HD / 16], F store) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  __syncthreads();   // every wave has read its last tile
#pragma unroll
  for (int db = 0; db < HD / 16; ++db) *join_at<HD>(m + wid * 16 * HD, lane & 15, 4 * db + (lane >> 4)) = acc[db];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * (HD / 4); i += 64 * NW) {
    const int row = i / (HD / 4), c4 = i % (HD / 4);
    f32x4 v = *join_at<HD>(m, row, c4);
#pragma unroll
    for (int w = 1; w < NW; ++w) v += *join_at<HD>(m + w * 16 * HD, row, c4);
    store(row, 4 * c4, v);
  }
}

// ---- LDS tiles of ROWS x HD elements, filled by direct loads, 16-byte pieces swizzled ----

// 256-byte bf16 rows (each starts at bank 0) are read both as row fragments and by transposing reads;
// an even exclusive-or by the row's low bits keeps the pairs of pieces that a transposing read takes
// together and puts 8 rows on distinct banks. (swz<128> serves row fragments alone: with it a third of
// the forward's LDS cycles were conflicts, now none are; d = 128 passes over 4096 tokens -0 to -2 %.)
template <typename T, int HD>
__device__ __forceinline__ int tswz(int row) {
  return sizeof(T) == 2 && HD == 128 ? 2 * (row & 7) : swz<HD * (int)sizeof(T) / 2>(row);
}

// Rows r0 + [0, ROWS) of a matrix with row stride ld, by NW waves; rows at or past nrows repeat the
// last one (masked by the caller; nrows > 0).
template <typename T, int HD, int ROWS, int NW>
struct TileLoad {
  static constexpr int E = 16 / (int)sizeof(T), CPR = HD / E, NI = ROWS * CPR / 64;
  static_assert(NI % NW == 0, "tile / wave split");
  __device__ __forceinline__ static void issue(T* lds, const T* g, long long ld, int r0, int nrows, int wid, int lane) {
#pragma unroll
    for (int u = 0; u < NI / NW; ++u) {
      const int blk = wid * (NI / NW) + u, idx = blk * 64 + lane;
      const int row = idx / CPR, c = (idx % CPR) ^ tswz<T, HD>(row);
      const int r = min(r0 + row, nrows - 1);
      load_lds16(g + r * ld + E * c, lds + blk * 64 * E);
    }
  }
};

// 8 consecutive elements (chunk lc) of a tile row
template <int HD>
__device__ __forceinline__ bf16x8 row_frag(const bf16_t* t, int x, int lc) {
  return *reinterpret_cast<const bf16x8*>(t + x * HD + 8 * (lc ^ tswz<bf16_t, HD>(x)));
}
template <int HD>
__device__ __forceinline__ f32x8 row_frag(const float* t, int x, int lc) {
  const float* row = t + x * HD;
  const int s = tswz<float, HD>(x);
  const float4 a = *reinterpret_cast<const float4*>(row + 4 * ((2 * lc) ^ s));
  const float4 b = *reinterpret_cast<const float4*>(row + 4 * ((2 * lc + 1) ^ s));
  return f32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}
// column m0 + lane % 16 at rows k0 + 4j + i and k0 + 16 + 4j + i (j = lane / 16, i = 0..3)
template <int HD>
__device__ __forceinline__ bf16x8 col_frag(const bf16_t* t, int k0, int m0, int lane) {
  if constexpr (HD != 128) {
    return lds_tr_chunk<HD>(t, k0, m0, lane);
  } else {   // the same reads with this file's swizzle
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int p = lane & 15, x0 = k0 + 4 * (lane >> 4) + (p >> 2), x1 = x0 + 16, col = m0 + 4 * (p & 3);
    const bf16_t* a0 = t + x0 * HD + 8 * ((col >> 3) ^ tswz<bf16_t, HD>(x0)) + (col & 7);
    const bf16_t* a1 = t + x1 * HD + 8 * ((col >> 3) ^ tswz<bf16_t, HD>(x1)) + (col & 7);
    const uint2 v0 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a0));
    const uint2 v1 = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a1));
    return __builtin_bit_cast(bf16x8, make_uint4(v0.x, v0.y, v1.x, v1.y));
  }
}
template <int HD>
__device__ __forceinline__ f32x8 col_frag(const float* t, int k0, int m0, int lane) {
  const int c = m0 + (lane & 15), j = lane >> 4;
  f32x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int x = k0 + (e < 4 ? 0 : 16) + 4 * j + (e & 3);
    v[e] = t[x * HD + 4 * ((c >> 2) ^ tswz<float, HD>(x)) + (c & 3)];
  }
  return v;
}

// ---- values that are not finite, behind the causal mask ----
//
// A masked probability is 0, but 0 times an infinity or NaN of a masked row is NaN in a matrix product.
// So before a tile on the causal diagonal is used, its 16-byte pieces that hold such a value are zeroed, and the rows
// that see one get their NaN apart: o and dq from the first such key, the key-major pass from the row's lse. (Doing it within the products cost 10 to 40 % in registers on calls that hold no
// such value.)

// An exponent of all ones carries into its value's sign bit.
template <typename T>
__device__ __forceinline__ bool odd_piece(const uint4& u) {
  constexpr uint32_t ones = sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u, low = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
  const uint32_t any = ((u.x & ones) + low) | ((u.y & ones) + low) | ((u.z & ones) + low) | ((u.w & ones) + low);
  return any & (sizeof(T) == 2 ? 0x80008000u : 0x80000000u);
}

__device__ __forceinline__ bool odd_chunk(const bf16x8& x) { return odd_piece<bf16_t>(__builtin_bit_cast(uint4, x)); }
__device__ __forceinline__ bool odd_chunk(const f32x8& x) {
  uint32_t any = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) any |= (__float_as_uint(x[e]) & 0x7f800000u) + 0x00800000u;
  return any & 0x80000000u;
}

// Clears a landed tile of ROWS x HD; returns its first row that held such a value (ROWS: none). Every wave
// that shares the tile searches all of it, so that all of them take the same way.
template <typename T, int HD, int ROWS, bool SPLIT>
__device__ __forceinline__ int clear_tile(T* tile) {
  constexpr int CPR = HD * (int)sizeof(T) / 16;
  uint4* const piece = reinterpret_cast<uint4*>(tile);
  const int lane = threadIdx.x & 63;
  uint32_t odd = 0;      // one bit per piece of this lane
  static_assert(ROWS * CPR / 64 <= 32, "a bit each");
#pragma unroll 4
  for (int u = 0; u < ROWS * CPR / 64; ++u) odd |= (uint32_t)odd_piece<T>(piece[u * 64 + lane]) << u;
  if (!__builtin_amdgcn_ballot_w64(odd != 0)) return ROWS;
  int first = odd ? (__builtin_ctz(odd) * 64 + lane) / CPR : ROWS;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) first = min(first, __shfl_xor(first, o, 64));
  if constexpr (!SPLIT) __syncthreads();   // every wave has searched it
  for (; odd; odd &= odd - 1) piece[__builtin_ctz(odd) * 64 + lane] = make_uint4(0, 0, 0, 0);
  if constexpr (SPLIT)
    wave_sync();
  else
    __syncthreads();
  return __builtin_amdgcn_readfirstlane(first);
}

// Quotients by the group size: floor(x / G) by a multiplication, one too large at most (x < 2^31).
struct Group {
  int G;
  uint32_t magic;    // floor(2^32 / G) + 1
  __device__ __forceinline__ int div(int x) const {
    if (G == 1) return x;
    const int q = (int)__umulhi((uint32_t)x, magic);
    return q * G > x ? q - 1 : q;
  }
};

// Element offsets of a packed row: query row t = q0 + p / G, head hk G + p % G.
struct RowAt {
  long long t;
  int h;
};
__device__ __forceinline__ RowAt packed_row(const Seq& sq, int hk, const Group& g, int p) {
  const int q = g.div(p);
  return RowAt{sq.q0 + q, hk * g.G + p - q * g.G};
}

// The same for packed rows r0 + [0, ROWS) (rows of them, > 0).
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

struct FwdP {
  AttnArgs a;
  const void *q, *k, *v;
  SeqArgs seq;
  Group G;
  void* o;
  float* lse;
  float sl2;         // scale log2(e)
  int nsplit;        // splits of the key axis
  float* part;       // [nsplit][total_q][heads][hd] unnormalised outputs
  float2* ml;        // [nsplit][total_q][heads] reference maximum (log2 units) and sum
};

// Keys [lo, hi) of split z: equal runs of whole tiles.
__device__ __forceinline__ void split_range(int lk, int nsplit, int z, int KT, int& lo, int& hi) {
  const int tiles = (lk + KT - 1) / KT, per = (tiles + nsplit - 1) / nsplit;
  lo = min(z * per * KT, lk);
  hi = min(lo + per * KT, lk);
}

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

// Joins the splits of a row: o = sum_z 2^(m_z - m) o_z / sum_z 2^(m_z - m) l_z. HD / 4 threads
// per (query row, head); rows of no sequence are left, or zeroed.
template <typename T, int HD>
__global__ void __launch_bounds__(256) packed_join_kernel(FwdP p) {
  constexpr int TPR = HD / 4;
  const AttnArgs& a = p.a;
  const long long row = (long long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  const int c = 4 * (threadIdx.x % TPR);
  if (row >= a.total_q * a.heads) return;
  const long long t = row / a.heads;
  const int h = (int)(row - t * a.heads);
  const bool in = t < p.seq.cu_q[a.seqs];
  if (!in && !a.zero_rest) return;
  float m = kNegInf, l = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  if (in) {
    const long long per = a.total_q * a.heads;
#pragma unroll 8
    for (int z = 0; z < p.nsplit; ++z) m = fmaxf(m, p.ml[z * per + row].x);
    const float mref = m == kNegInf ? 0.f : m;
#pragma unroll 8
    for (int z = 0; z < p.nsplit; ++z) {
      const float2 ml = p.ml[z * per + row];
      const f32x4 part = *reinterpret_cast<const f32x4*>(p.part + (z * per + row) * HD + c);
      const float w = fast_exp2(ml.x - mref);
      l += w * ml.y;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] += ml.y == 0.f ? 0.f : w * part[e];   // saw nothing: not written
    }
  }
  const bool any = !(l == 0.f);
  store4((T*)p.o + t * a.o_row + h * a.o_head + c, any ? acc : f32x4{0.f, 0.f, 0.f, 0.f}, any ? 1.0f / l : 0.f);
  if (c == 0) p.lse[h * a.total_q + t] = any ? (m + log2f(l)) * kLn2 : kNegInf;
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

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// A multiple of 8 (xcd_slot).
unsigned tile_slots(long long total, int mult, int R, int S) { return (unsigned)((total * mult / R + S + 7) / 8 * 8); }

Group group_of(const AttnArgs& a) { return Group{a.group(), (uint32_t)((1ull << 32) / a.group() + 1)}; }

// How the forward runs: SPLIT (Share) where a sequence has 32 packed rows or fewer on average, or
// the 128-row tiles would leave half of the CUs idle; and the splits of the key axis, up to two
// workgroups per CU with at least 256 keys of an average sequence each (32 single tokens against
// caches of up to 8192 rows, 8 key heads of 128: 116 us with 2 splits, 120 with 4, 138 with 8: a
// workgroup's start costs about as much as 100 keys). The lengths are on the device: a cache
// counts with its capacity.
struct FwdPlan {
  bool split;
  int nsplit;
};
constexpr int kFwdQB = 2;
FwdPlan fwd_plan(const AttnArgs& a) {
  const long long rows = a.total_q * a.group();
  const long long avg_k = a.total_k / a.seqs;
  auto wgs = [&](int R) { return std::max<long long>((rows + R - 1) / R, a.seqs) * a.kv_heads; };
  FwdPlan f;
  f.split = rows <= 32LL * a.seqs || wgs(16 * kFwdQB * kWaves) < 128;
  const long long n = 512 / wgs(f.split ? 16 : 16 * kFwdQB * kWaves);
  f.nsplit = (int)std::max<long long>(std::min<long long>(std::min<long long>(n, avg_k / 256), 64), 1);
  return f;
}

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
