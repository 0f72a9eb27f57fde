// Internal declarations of the dense operators (layer norm, affine map, gated map, rotary positions,
// packed attention, 8-bit cache): argument records shared by their launchers and the C entry points (dense_api.cpp).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace bsa {

// dense_norm.hip: rows x cols, elements of type T (bf16 or f32) with row strides; gain and bias f32
struct NormArgs {
  long long rows;
  int cols;
  bool bf16;
  float eps;
  long long ldx, ldy, lddy, lddx;
};
constexpr int kNormMaxCols = 32768;
hipError_t launch_layernorm_fwd(const NormArgs& a, const void* x, const float* gain, const float* bias, void* y,
                                float* mean, float* rstd, hipStream_t st);
size_t layernorm_bwd_ws_bytes(const NormArgs& a);
hipError_t launch_layernorm_bwd(const NormArgs& a, const void* x, const float* gain, const float* mean,
                                const float* rstd, const void* dy, void* dx, float* dgain, float* dbias, void* ws,
                                hipStream_t st);

// dense_linear.hip: z = x w^T + bias, y = act(z) + res; x [m, k], w [n, k], y [m, n]
enum DenseAct { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };
struct LinearArgs {
  long long m;
  int k, n;
  bool bf16;
  int act;
  long long ldx, ldw, ldy, ldr, lddy;
  int readable_k = 0, readable_n = 0;   // backward: columns of x and w, and of dy, that may be read (0: k and n)
};
size_t linear_fwd_ws_bytes(const LinearArgs& a);
hipError_t launch_linear_fwd(const LinearArgs& a, const void* x, const void* w, const void* bias, const void* res,
                             void* y, void* pre, void* ws, hipStream_t st);
size_t linear_bwd_ws_bytes(const LinearArgs& a);
// dx, dw and db may be NULL (not formed)
hipError_t launch_linear_bwd(const LinearArgs& a, const void* x, const void* w, const void* pre, const void* dy,
                             void* dx, void* dw, void* db, void* ws, hipStream_t st);

// dense_gated.hip: [g | u] = x w^T + bias, y = act(g) u; x [m, k], w [2n, k], y [m, n]
struct GatedArgs {
  long long m;
  int k, n;
  bool bf16;
  int act;
  long long ldx, ldw, ldy, lddy;
};
size_t gated_fwd_ws_bytes(const GatedArgs& a);
hipError_t launch_gated_fwd(const GatedArgs& a, const void* x, const void* w, const void* bias, void* y, void* pre, void* ws,
                            hipStream_t st);
size_t gated_bwd_ws_bytes(const GatedArgs& a);
// dx, dw and db may be NULL (not formed)
hipError_t launch_gated_bwd(const GatedArgs& a, const void* x, const void* w, const void* pre, const void* dy, void* dx,
                            void* dw, void* db, void* ws, hipStream_t st);

// dense_rotary.hip: rotary positions and head norms of q [rows, heads, hd] and k [rows, kv_heads, hd];
// strides in elements. o*: y of the forward, dx of the backward; d*: dy.
struct RotaryArgs {
  long long rows;
  int heads, kv_heads, hd, rot, axes;
  bool fpos, interleaved, bf16;
  float eps, mag;
  long long q_row, q_head, k_row, k_head, oq_row, oq_head, ok_row, ok_head, dq_row, dq_head, dk_row, dk_head;
};
constexpr int kRotMaxDim = 256;
hipError_t launch_rotary_fwd(const RotaryArgs& a, const void* q, const void* k, const void* pos, const double* freq,
                             const float* gain_q, const float* gain_k, void* out_q, void* out_k, hipStream_t st);
size_t rotary_bwd_ws_bytes(const RotaryArgs& a);
hipError_t launch_rotary_bwd(const RotaryArgs& a, const void* q, const void* k, const void* pos, const double* freq,
                             const float* gain_q, const float* gain_k, const void* dy_q, const void* dy_k, void* dq, void* dk,
                             float* dgain_q, float* dgain_k, void* ws, hipStream_t st);

// dense_attn.hip: packed attention. Strides in elements of the storage type.
struct AttnArgs {
  int seqs, heads, kv_heads, hd;
  long long total_q, total_k;
  bool causal, bf16, zero_rest;
  float scale;
  long long q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, do_row, do_head;
  int group() const { return heads / kv_heads; }
};
bool attention_fwd_fits(const AttnArgs& a);   // the launches are within the limits of one
bool attention_bwd_fits(const AttnArgs& a);
size_t attention_fwd_ws_bytes(const AttnArgs& a);
hipError_t launch_attention_fwd(const AttnArgs& a, const void* q, const void* k, const void* v, const int* cu_q,
                                const int* cu_k, const int* used_k, void* o, float* lse, void* ws, hipStream_t st);
size_t attention_bwd_ws_bytes(const AttnArgs& a);
hipError_t launch_attention_bwd(const AttnArgs& a, const void* q, const void* k, const void* v, const void* o,
                                const float* lse, const void* d_o, const int* cu_q, const int* cu_k, const int* used_k,
                                void* dq, void* dk, void* dv, void* ws, hipStream_t st);

// dense_cache.hip: a cache of e4m3 rows [total_k, kv_heads, hd] with one exponent for each row and key head,
// exp [kv_heads, total_k]. New rows [rows, kv_heads, hd] of sequence s are the last cu_q[s + 1] - cu_q[s] of
// its used_k[s]. Strides in elements (cache: bytes).
struct CacheArgs {
  int seqs, kv_heads, hd;
  long long rows, total_k;
  bool bf16;
  long long k_row, k_head, v_row, v_head, ck_row, ck_head, cv_row, cv_head;
};
hipError_t launch_cache_write(const CacheArgs& a, const void* k, const void* v, const int* cu_q, const int* cu_k,
                              const int* used_k, void* ck, void* cv, unsigned char* ek, unsigned char* ev, hipStream_t st);
hipError_t launch_cache_read(const CacheArgs& a, const void* ck, const void* cv, const unsigned char* ek,
                             const unsigned char* ev, const int* cu_q, const int* cu_k, const int* used_k, void* k, void* v,
                             hipStream_t st);
// attention that reads it: strides of k and v in a are the cache's
bool cache_attention_fits(const AttnArgs& a);
size_t cache_attention_ws_bytes(const AttnArgs& a);
hipError_t launch_cache_attention(const AttnArgs& a, const void* q, const void* ck, const void* cv, const unsigned char* ek,
                                  const unsigned char* ev, const int* cu_q, const int* cu_k, const int* used_k, void* o,
                                  float* lse, void* ws, hipStream_t st);

}  // namespace bsa
