// C entry points of the dense operators: argument checks and launches. Declarations and
// contracts: include/bsa.h.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <string>

#include "dense.hpp"
#include "kernels.hpp"
#include "status.hpp"

namespace {

using bsa::set_error;

bsa_status_t bad(const char* msg) { return set_error(BSA_ERR_INVALID_ARGUMENT, msg); }

// The body of an entry point: no C++ exception leaves it.
template <typename F>
bsa_status_t entry(F f) noexcept {
  try {
    bsa::clear_error();
    return f();
  } catch (...) {
    return BSA_ERR_HIP;
  }
}

bsa_status_t launched(hipError_t e, const char* where) {
  if (e == hipSuccess) return BSA_OK;
  return set_error(BSA_ERR_HIP, std::string(where) + ": " + hipGetErrorString(e));
}

bsa_status_t small_ws(const char* where, size_t need) {
  return set_error(BSA_ERR_WORKSPACE_TOO_SMALL, std::string(where) + " workspace needs " + std::to_string(need) + " bytes");
}

constexpr const char* kTooManyTiles = "too many tiles for one launch (2^32 threads or more)";

bool dtype_ok(int32_t d) { return d == BSA_F32 || d == BSA_BF16; }
bool ld_ok(int64_t ld, int64_t cols) { return ld == 0 || ld >= cols; }
long long ld_of(int64_t ld, int64_t cols) { return ld ? ld : cols; }
// An output that is formed starts where one of the inputs does (NULL: not formed, not read).
bool on_one(const void* out, std::initializer_list<const void*> inputs) {
  return out && std::find(inputs.begin(), inputs.end(), out) != inputs.end();
}
bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

bsa_status_t check(const bsa_layernorm_t* p, bsa::NormArgs* a) {
  if (!p) return bad("params is NULL");
  if (p->rows < 0 || p->rows > ((int64_t)1 << 40)) return bad("rows must be in [0, 2^40]");
  if (p->cols < 1) return bad("cols must be >= 1");
  if (p->cols > bsa::kNormMaxCols) return set_error(BSA_ERR_UNSUPPORTED, "cols must be <= 32768");
  if (!dtype_ok(p->dtype)) return bad("bad dtype");
  if (!(p->eps > 0.0f) || std::isinf(p->eps)) return bad("eps must be finite and > 0");
  if (!ld_ok(p->ld_x, p->cols) || !ld_ok(p->ld_y, p->cols) || !ld_ok(p->ld_dy, p->cols) || !ld_ok(p->ld_dx, p->cols))
    return bad("leading dimensions must be 0 or >= cols");
  *a = bsa::NormArgs{p->rows,          p->cols, p->dtype == BSA_BF16, p->eps, ld_of(p->ld_x, p->cols), ld_of(p->ld_y, p->cols),
                     ld_of(p->ld_dy, p->cols), ld_of(p->ld_dx, p->cols)};
  return BSA_OK;
}

bsa_status_t check(const bsa_linear_t* p, bsa::LinearArgs* a) {
  if (!p) return bad("params is NULL");
  if (p->m < 0 || p->m > INT32_MAX) return bad("m must be in [0, 2^31)");
  if (p->k < 1 || p->n < 1) return bad("k and n must be >= 1");
  if (p->k > (1 << 24) || p->n > (1 << 24)) return set_error(BSA_ERR_UNSUPPORTED, "k and n must be <= 2^24");
  // 256 x 256 tiles have 512 threads, 128 x 128 tiles 256 (64 x 64 tiles are used where there are few)
  const auto fits = [](int64_t M, int64_t N) {
    return (M + 255) / 256 * ((N + 255) / 256) < 1 << 23 && (M + 127) / 128 * ((N + 127) / 128) < 1 << 24;
  };
  if (!fits(p->m, std::max(p->n, p->k)) || !fits(p->n, p->k)) return set_error(BSA_ERR_UNSUPPORTED, kTooManyTiles);
  if (!dtype_ok(p->dtype)) return bad("bad dtype");
  if (p->act < BSA_ACT_NONE || p->act > BSA_ACT_SILU) return bad("bad act");
  if (!ld_ok(p->ld_x, p->k) || !ld_ok(p->ld_w, p->k) || !ld_ok(p->ld_y, p->n) || !ld_ok(p->ld_res, p->n) ||
      !ld_ok(p->ld_dy, p->n))
    return bad("leading dimensions must be 0 or at least the row's length");
  *a = bsa::LinearArgs{p->m, p->k, p->n, p->dtype == BSA_BF16, p->act, ld_of(p->ld_x, p->k), ld_of(p->ld_w, p->k),
                       ld_of(p->ld_y, p->n), ld_of(p->ld_res, p->n), ld_of(p->ld_dy, p->n)};
  return BSA_OK;
}

bsa_status_t check(const bsa_attention_t* p, bsa::AttnArgs* a) {
  if (!p) return bad("params is NULL");
  if (p->seqs < 1) return bad("seqs must be >= 1");
  if (p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads != 0) return bad("kv_heads must divide heads (both >= 1)");
  if (p->heads > 65535) return set_error(BSA_ERR_UNSUPPORTED, "heads must be <= 65535");
  if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128)
    return set_error(BSA_ERR_UNSUPPORTED, "head_dim must be 32, 64 or 128");
  if (p->total_q < 0 || p->total_q > INT32_MAX || p->total_k < 0 || p->total_k > INT32_MAX)
    return bad("total_q and total_k must be in [0, 2^31)");
  if (p->total_q * (p->heads / p->kv_heads) > ((int64_t)1 << 30) || p->total_k > ((int64_t)1 << 30) || p->seqs > (1 << 24))
    return set_error(BSA_ERR_UNSUPPORTED, "query rows times heads / kv_heads and key rows must be <= 2^30, seqs <= 2^24");
  if (p->causal != 0 && p->causal != 1) return bad("causal must be 0/1");
  if (p->zero_rest != 0 && p->zero_rest != 1) return bad("zero_rest must be 0/1");
  if (!dtype_ok(p->dtype)) return bad("bad dtype");
  if (!(p->softmax_scale >= 0.0f) || std::isinf(p->softmax_scale)) return bad("softmax_scale must be finite and >= 0");
  const int e = p->dtype == BSA_BF16 ? 8 : 4;   // elements of 16 bytes
  *a = bsa::AttnArgs{p->seqs, p->heads, p->kv_heads, p->head_dim, p->total_q, p->total_k, p->causal != 0,
                     p->dtype == BSA_BF16, p->zero_rest != 0,
                     p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / std::sqrt((float)p->head_dim),
                     p->q_row, p->q_head, p->k_row, p->k_head, p->v_row, p->v_head, p->o_row, p->o_head, p->do_row, p->do_head};
  const struct { long long *row, *head; int heads; } st[5] = {{&a->q_row, &a->q_head, p->heads},
                                                              {&a->k_row, &a->k_head, p->kv_heads},
                                                              {&a->v_row, &a->v_head, p->kv_heads},
                                                              {&a->o_row, &a->o_head, p->heads},
                                                              {&a->do_row, &a->do_head, p->heads}};
  for (const auto& s : st) {
    if (*s.row == 0 && *s.head == 0) {
      *s.head = p->head_dim;
      *s.row = (long long)s.heads * p->head_dim;
    }
    if (*s.row < 0 || *s.head < 0 || *s.row % e != 0 || *s.head % e != 0)
      return bad("strides must be >= 0 and multiples of 16 bytes");
  }
  return BSA_OK;
}

}  // namespace

extern "C" {

bsa_status_t bsa_layernorm_sizes(const bsa_layernorm_t* p, size_t* ws_bwd_bytes) {
  return entry([&] {
    bsa::NormArgs a;
    const bsa_status_t s = check(p, &a);
    if (s == BSA_OK && ws_bwd_bytes) *ws_bwd_bytes = bsa::layernorm_bwd_ws_bytes(a);
    return s;
  });
}

bsa_status_t bsa_layernorm_forward(const bsa_layernorm_t* p, const void* x, const float* gain, const float* bias, void* y,
                                   float* mean, float* rstd, void* stream) {
  return entry([&] {
    bsa::NormArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK || a.rows == 0) return s;
    if (!x || !gain || !y || !mean || !rstd) return bad("x, gain, y, mean and rstd must be non-NULL");
    if (x == y) return bad("y may not alias x");
    hipError_t e;
    BSA_PHASE("norm.fwd", (hipStream_t)stream,
              e = bsa::launch_layernorm_fwd(a, x, gain, bias, y, mean, rstd, (hipStream_t)stream));
    return launched(e, "bsa_layernorm_forward");
  });
}

bsa_status_t bsa_layernorm_backward(const bsa_layernorm_t* p, const void* x, const float* gain, const float* mean,
                                    const float* rstd, const void* dy, void* dx, float* dgain, float* dbias, void* ws,
                                    size_t ws_bytes, void* stream) {
  return entry([&] {
    bsa::NormArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK) return s;
    if (!gain || !dgain) return bad("gain and dgain must be non-NULL");
    if (a.rows > 0 && (!x || !mean || !rstd || !dy || !dx)) return bad("x, mean, rstd, dy and dx must be non-NULL");
    if ((dx == dy && a.lddx != a.lddy) || (dx == x && a.lddx != a.ldx))
      return bad("dx may be dy or x only with the same leading dimension");
    const size_t need = bsa::layernorm_bwd_ws_bytes(a);
    if (need && (!ws || ws_bytes < need)) return small_ws("layer norm backward", need);
    hipError_t e;
    BSA_PHASE("norm.bwd", (hipStream_t)stream,
              e = bsa::launch_layernorm_bwd(a, x, gain, mean, rstd, dy, dx, dgain, dbias, ws, (hipStream_t)stream));
    return launched(e, "bsa_layernorm_backward");
  });
}

bsa_status_t bsa_linear_sizes(const bsa_linear_t* p, size_t* ws_fwd_bytes, size_t* ws_bwd_bytes) {
  return entry([&] {
    bsa::LinearArgs a;
    const bsa_status_t s = check(p, &a);
    if (s != BSA_OK) return s;
    if (ws_fwd_bytes) *ws_fwd_bytes = bsa::linear_fwd_ws_bytes(a);
    if (ws_bwd_bytes) *ws_bwd_bytes = bsa::linear_bwd_ws_bytes(a);
    return s;
  });
}

bsa_status_t bsa_linear_forward(const bsa_linear_t* p, const void* x, const void* w, const void* bias, const void* res,
                                void* y, void* pre, void* ws, size_t ws_bytes, void* stream) {
  return entry([&] {
    bsa::LinearArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK || a.m == 0) return s;
    if (!x || !w || !y) return bad("x, w and y must be non-NULL");
    if (on_one(y, {x, w, bias, pre})) return bad("y may not alias x, w, bias or pre");
    if (on_one(pre, {x, w, bias, res})) return bad("pre may not alias an input");
    if (res == y && a.ldr != a.ldy) return bad("res may be y only with the same leading dimension");
    const size_t need = bsa::linear_fwd_ws_bytes(a);
    if (need && (!ws || ws_bytes < need)) return small_ws("affine map forward", need);
    hipError_t e;
    BSA_PHASE("linear.fwd", (hipStream_t)stream,
              e = bsa::launch_linear_fwd(a, x, w, bias, res, y, pre, ws, (hipStream_t)stream));
    return launched(e, "bsa_linear_forward");
  });
}

bsa_status_t bsa_linear_backward(const bsa_linear_t* p, const void* x, const void* w, const void* pre, const void* dy,
                                 void* dx, void* dw, void* db, void* ws, size_t ws_bytes, void* stream) {
  return entry([&] {
    bsa::LinearArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK) return s;
    if (!dx && !dw && !db) return BSA_OK;
    if (a.m > 0) {
      if (!dy) return bad("dy must be non-NULL");
      if (a.act != bsa::kActNone && !pre) return bad("pre must be non-NULL for a map with an activation");
      if (dx && !w) return bad("w must be non-NULL for dx");
      if (dw && !x) return bad("x must be non-NULL for dw");
    }
    for (const void* g : {dx, dw, db})
      if (on_one(g, {x, w, a.act == bsa::kActNone ? nullptr : pre, dy})) return bad("a gradient may not alias an input");
    const size_t need = bsa::linear_bwd_ws_bytes(a);
    if (need && (!ws || ws_bytes < need)) return small_ws("affine map backward", need);
    hipError_t e;
    BSA_PHASE("linear.bwd", (hipStream_t)stream,
              e = bsa::launch_linear_bwd(a, x, w, pre, dy, dx, dw, db, ws, (hipStream_t)stream));
    return launched(e, "bsa_linear_backward");
  });
}

bsa_status_t bsa_attention_sizes(const bsa_attention_t* p, size_t* ws_fwd_bytes, size_t* ws_bwd_bytes) {
  return entry([&] {
    bsa::AttnArgs a;
    const bsa_status_t s = check(p, &a);
    if (s != BSA_OK) return s;
    if (ws_fwd_bytes) *ws_fwd_bytes = bsa::attention_fwd_ws_bytes(a);
    if (ws_bwd_bytes) *ws_bwd_bytes = bsa::attention_bwd_ws_bytes(a);
    return s;
  });
}

bsa_status_t bsa_attention_forward(const bsa_attention_t* p, const void* q, const void* k, const void* v,
                                   const int32_t* cu_q, const int32_t* cu_k, const int32_t* used_k, void* o, float* lse,
                                   void* ws, size_t ws_bytes, void* stream) {
  return entry([&] {
    bsa::AttnArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK || a.total_q == 0) return s;
    if (!bsa::attention_fwd_fits(a)) return set_error(BSA_ERR_UNSUPPORTED, kTooManyTiles);
    if (!q || !cu_q || !cu_k || !o || !lse) return bad("q, cu_q, cu_k, o and lse must be non-NULL");
    if (a.total_k > 0 && (!k || !v)) return bad("k and v must be non-NULL");
    if (o == q || o == k || o == v) return bad("o may not alias an input");
    const long long d = a.hd, rows = (a.total_q - 1) * a.o_row + d, heads = (a.heads - 1) * a.o_head + d;
    if (!((a.heads == 1 || a.o_head >= d) && (a.total_q == 1 || a.o_row >= heads)) &&
        !((a.total_q == 1 || a.o_row >= d) && (a.heads == 1 || a.o_head >= rows)))
      return bad("o's rows and heads may not overlap");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16))
      return bad("q, k, v and o must be 16-byte aligned");
    const size_t need = bsa::attention_fwd_ws_bytes(a);
    if (need && (!ws || ws_bytes < need)) return small_ws("attention forward", need);
    if (need && !aligned(ws, 16)) return bad("ws must be 16-byte aligned");
    hipError_t e;
    BSA_PHASE("attn.fwd", (hipStream_t)stream,
              e = bsa::launch_attention_fwd(a, q, k, v, cu_q, cu_k, used_k, o, lse, ws, (hipStream_t)stream));
    return launched(e, "bsa_attention_forward");
  });
}

bsa_status_t bsa_attention_backward(const bsa_attention_t* p, const void* q, const void* k, const void* v, const void* o,
                                    const float* lse, const void* d_o, const int32_t* cu_q, const int32_t* cu_k,
                                    const int32_t* used_k, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes,
                                    void* stream) {
  return entry([&] {
    bsa::AttnArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK) return s;
    if (!bsa::attention_bwd_fits(a)) return set_error(BSA_ERR_UNSUPPORTED, kTooManyTiles);
    if (!cu_q || !cu_k) return bad("cu_q and cu_k must be non-NULL");
    if (a.total_q > 0 && (!q || !o || !lse || !d_o || !dq)) return bad("q, o, lse, d_o and dq must be non-NULL");
    if (a.total_k > 0 && (!k || !v || !dk || !dv)) return bad("k, v, dk and dv must be non-NULL");
    for (const void* t : {q, k, v, o, d_o, (const void*)dq, (const void*)dk, (const void*)dv})
      if (!aligned(t, 16)) return bad("q, k, v, o, d_o, dq, dk and dv must be 16-byte aligned");
    for (const void* g : {dq, dk, dv})
      if (on_one(g, {q, k, v, o, d_o})) return bad("a gradient may not alias an input");
    const size_t need = bsa::attention_bwd_ws_bytes(a);
    if (need && (!ws || ws_bytes < need)) return small_ws("attention backward", need);
    if (need && !aligned(ws, 16)) return bad("ws must be 16-byte aligned");
    hipError_t e;
    BSA_PHASE("attn.bwd", (hipStream_t)stream,
              e = bsa::launch_attention_bwd(a, q, k, v, o, lse, d_o, cu_q, cu_k, used_k, dq, dk, dv, ws, (hipStream_t)stream));
    return launched(e, "bsa_attention_backward");
  });
}

}  // extern "C"
