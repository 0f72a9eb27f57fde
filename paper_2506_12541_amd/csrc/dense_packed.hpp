// Pieces shared by the kernels of attention over packed sequences (queries and keys of one type, and
// queries against the 8-bit cache): sequences and their tiles, staged tiles in LDS, packed rows of grouped
// heads, splits of the key axis and their joining.
#pragma once
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

}  // namespace
}  // namespace bsa
