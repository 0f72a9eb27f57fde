// Moves shared by the dense operators' kernels: 16-byte pieces at element alignment (gfx950
// global memory accesses may be unaligned), pieces that end inside a row, and conversion of a
// piece to and from float32.
#pragma once
#include "common.hpp"

namespace bsa {
namespace {

template <typename T>
__device__ __forceinline__ uint4 load16u(const T* p) {
  uint4 v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
// The same of eight bf16 values by whole words: a load of 16 bytes that begins inside a 4-byte word takes more than twice
// as long. Such a load begins one value earlier, so the value in front of p has to be in bounds as well: it is in a
// matrix that begins with a word.
__device__ __forceinline__ uint4 load16_words(const bf16_t* p) {
  const bool odd = (uintptr_t)p & 2;
  uint4 v;
  __builtin_memcpy(&v, __builtin_assume_aligned(p - (odd ? 1 : 0), 4), 16);
  const uint32_t last = *reinterpret_cast<const uint16_t*>(p + 7);
  if (odd)
    v = make_uint4(__builtin_amdgcn_alignbit(v.y, v.x, 16), __builtin_amdgcn_alignbit(v.z, v.y, 16),
                   __builtin_amdgcn_alignbit(v.w, v.z, 16), last << 16 | v.w >> 16);
  return v;
}
template <typename T>
__device__ __forceinline__ void store16u(T* p, uint4 v) {
  __builtin_memcpy(p, &v, 16);
}

// The first n (0 < n < 16 / sizeof(T)) elements at p, zeros behind them.
__device__ __forceinline__ uint4 load_partial(const float* p, int n) {
  return make_uint4(__float_as_uint(p[0]), n > 1 ? __float_as_uint(p[1]) : 0u, n > 2 ? __float_as_uint(p[2]) : 0u, 0u);
}
__device__ __forceinline__ uint4 load_partial(const bf16_t* p, int n) {
  auto at = [&](int i) -> uint32_t { return i < n ? (uint32_t)p[i] : 0u; };
  return make_uint4(at(0) | (at(1) << 16), at(2) | (at(3) << 16), at(4) | (at(5) << 16), at(6));
}
__device__ __forceinline__ void store_partial(float* p, uint4 v, int n) {
  p[0] = __uint_as_float(v.x);
  if (n > 1) p[1] = __uint_as_float(v.y);
  if (n > 2) p[2] = __uint_as_float(v.z);
}
__device__ __forceinline__ void store_partial(bf16_t* p, uint4 v, int n) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) p[i] = (bf16_t)(w[i / 2] >> (16 * (i & 1)));
}

template <typename T> __device__ __forceinline__ void unpack16(uint4 u, float* v);
template <> __device__ __forceinline__ void unpack16<float>(uint4 u, float* v) {
  v[0] = __uint_as_float(u.x);
  v[1] = __uint_as_float(u.y);
  v[2] = __uint_as_float(u.z);
  v[3] = __uint_as_float(u.w);
}
template <> __device__ __forceinline__ void unpack16<bf16_t>(uint4 u, float* v) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
template <typename T> __device__ __forceinline__ uint4 pack16(const float* v);
template <> __device__ __forceinline__ uint4 pack16<float>(const float* v) {
  return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
template <> __device__ __forceinline__ uint4 pack16<bf16_t>(const float* v) {
  return __builtin_bit_cast(uint4, make_chunk<bf16_t>(v));
}

// Eight consecutive elements at element alignment; load_chunk_to: the first n of them (n <= 0:
// none), zeros behind.
__device__ __forceinline__ bf16x8 load_chunk_u(const bf16_t* p) { return __builtin_bit_cast(bf16x8, load16u(p)); }
__device__ __forceinline__ f32x8 load_chunk_u(const float* p) {
  f32x8 v;
  __builtin_memcpy(&v, p, 32);
  return v;
}
__device__ __forceinline__ bf16x8 load_chunk_to(const bf16_t* p, int n) {
  const uint4 v = n >= 8 ? load16u(p) : n > 0 ? load_partial(p, n) : make_uint4(0, 0, 0, 0);
  return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ f32x8 load_chunk_to(const float* p, int n) {
  f32x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.f;
  return v;
}

}  // namespace
}  // namespace bsa
