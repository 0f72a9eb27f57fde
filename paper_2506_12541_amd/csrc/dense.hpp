// Internal declarations of the dense operators (layer norm, affine map, packed attention):
// argument records shared by their launchers and the C entry points (dense_api.cpp).
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
};
size_t linear_fwd_ws_bytes(const LinearArgs& a);
hipError_t launch_linear_fwd(const LinearArgs& a, const void* x, const void* w, const void* bias, const void* res,
                             void* y, void* pre, void* ws, hipStream_t st);
size_t linear_bwd_ws_bytes(const LinearArgs& a);
// dx, dw and db may be NULL (not formed)
hipError_t launch_linear_bwd(const LinearArgs& a, const void* x, const void* w, const void* pre, const void* dy,
                             void* dx, void* dw, void* db, void* ws, hipStream_t st);

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

}  // namespace bsa
