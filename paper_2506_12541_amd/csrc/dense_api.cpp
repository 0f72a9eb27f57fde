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
  // 256 x 256 tiles have 512 threads, 128 x 128 tiles 256 (smaller ones are used where they are fewer than 2^24)
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

bsa_status_t check(const bsa_gated_t* p, bsa::GatedArgs* a) {
  if (!p) return bad("params is NULL");
  if (p->n < 1) return bad("k and n must be >= 1");
  if (p->n > (1 << 23)) return set_error(BSA_ERR_UNSUPPORTED, "n must be <= 2^23");
  if (p->act < BSA_ACT_NONE || p->act > BSA_ACT_SILU) return bad("bad act");
  if (!ld_ok(p->ld_y, p->n) || !ld_ok(p->ld_dy, p->n)) return bad("leading dimensions must be 0 or at least the row's length");
  // its products are those of a map to 2 n channels
  const bsa_linear_t both{p->m, p->k, 2 * p->n, p->dtype, BSA_ACT_NONE, p->ld_x, p->ld_w, 0, 0, 0};
  bsa::LinearArgs l;
  const bsa_status_t s = check(&both, &l);
  if (s != BSA_OK) return s;
  *a = bsa::GatedArgs{p->m, p->k, p->n, l.bf16, p->act, l.ldx, l.ldw, ld_of(p->ld_y, p->n), ld_of(p->ld_dy, p->n)};
  return BSA_OK;
}

// Strides of a [rows, heads, cols] tensor: both 0 is packed; whole multiples of `unit`.
bool strides_ok(long long* row, long long* head, int heads, int cols, int unit) {
  if (*row == 0 && *head == 0) {
    *head = cols;
    *row = (long long)heads * cols;
  }
  return *row >= 0 && *head >= 0 && *row % unit == 0 && *head % unit == 0;
}
// An output's rows and heads do not overlap.
bool apart(long long rows, long long row, int heads, long long head, int cols) {
  const long long all_rows = (rows - 1) * row + cols, all_heads = (heads - 1) * head + cols;
  return ((heads == 1 || head >= cols) && (rows <= 1 || row >= all_heads)) ||
         ((rows <= 1 || row >= cols) && (heads == 1 || head >= all_rows));
}
// An output may be the input itself where their strides are one.
bool on_other_strides(const void* out, long long row, long long head, const void* in, long long in_row, long long in_head) {
  return out && out == in && (row != in_row || head != in_head);
}

bsa_status_t check(const bsa_rotary_t* p, bsa::RotaryArgs* a) {
  if (!p) return bad("params is NULL");
  if (p->rows < 0 || p->rows > ((int64_t)1 << 40)) return bad("rows must be in [0, 2^40]");
  if (p->heads < 1 || p->kv_heads < 0) return bad("heads must be >= 1 and kv_heads >= 0");
  if (p->heads > 65535 || p->kv_heads > 65535) return set_error(BSA_ERR_UNSUPPORTED, "heads must be <= 65535");
  if (p->head_dim < 2) return bad("head_dim must be >= 2");
  if (p->head_dim > bsa::kRotMaxDim) return set_error(BSA_ERR_UNSUPPORTED, "head_dim must be <= 256");
  if (p->rot < 2 || p->rot > p->head_dim || p->rot % 2 != 0) return bad("rot must be even and in [2, head_dim]");
  if (p->axes < 1 || p->axes > 4 || p->rot / 2 % p->axes != 0) return bad("axes must be in [1, 4] and divide rot / 2");
  if (p->pos_type != BSA_POS_I32 && p->pos_type != BSA_POS_F32) return bad("bad pos_type");
  if (p->interleaved != 0 && p->interleaved != 1) return bad("interleaved must be 0/1");
  if (!dtype_ok(p->dtype)) return bad("bad dtype");
  if (!(p->eps > 0.0f) || std::isinf(p->eps)) return bad("eps must be finite and > 0");
  if (!(p->magnitude > 0.0f) || std::isinf(p->magnitude)) return bad("magnitude must be finite and > 0");
  *a = bsa::RotaryArgs{p->rows, p->heads, p->kv_heads, p->head_dim, p->rot, p->axes, p->pos_type == BSA_POS_F32,
                       p->interleaved != 0, p->dtype == BSA_BF16, p->eps, p->magnitude,
                       p->q_row, p->q_head, p->k_row, p->k_head, p->oq_row, p->oq_head, p->ok_row, p->ok_head,
                       p->dq_row, p->dq_head, p->dk_row, p->dk_head};
  const struct { long long *row, *head; int heads; } st[6] = {{&a->q_row, &a->q_head, p->heads},   {&a->k_row, &a->k_head, p->kv_heads},
                                                              {&a->oq_row, &a->oq_head, p->heads}, {&a->ok_row, &a->ok_head, p->kv_heads},
                                                              {&a->dq_row, &a->dq_head, p->heads}, {&a->dk_row, &a->dk_head, p->kv_heads}};
  for (const auto& t : st)
    if (!strides_ok(t.row, t.head, t.heads, p->head_dim, 1)) return bad("strides must be >= 0");
  if (!apart(p->rows, a->oq_row, p->heads, a->oq_head, p->head_dim) ||
      (p->kv_heads && !apart(p->rows, a->ok_row, p->kv_heads, a->ok_head, p->head_dim)))
    return bad("an output's rows and heads may not overlap");
  return BSA_OK;
}

bsa_status_t check(const bsa_cache_t* p, bsa::CacheArgs* a) {
  if (!p) return bad("params is NULL");
  if (p->seqs < 1) return bad("seqs must be >= 1");
  if (p->kv_heads < 1) return bad("kv_heads must be >= 1");
  if (p->kv_heads > 65535 || p->seqs > (1 << 24)) return set_error(BSA_ERR_UNSUPPORTED, "kv_heads must be <= 65535, seqs <= 2^24");
  if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128)
    return set_error(BSA_ERR_UNSUPPORTED, "head_dim must be 32, 64 or 128");
  if (p->rows < 0 || p->total_k < 0) return bad("rows and total_k must be >= 0");
  if (p->rows > ((int64_t)1 << 30) || p->total_k > ((int64_t)1 << 30))
    return set_error(BSA_ERR_UNSUPPORTED, "rows and total_k must be <= 2^30");
  if (!dtype_ok(p->dtype)) return bad("bad dtype");
  *a = bsa::CacheArgs{p->seqs, p->kv_heads, p->head_dim, p->rows, p->total_k, p->dtype == BSA_BF16, p->k_row, p->k_head,
                      p->v_row, p->v_head, p->ck_row, p->ck_head, p->cv_row, p->cv_head};
  const int e = p->dtype == BSA_BF16 ? 8 : 4;   // elements of 16 bytes
  if (!strides_ok(&a->k_row, &a->k_head, p->kv_heads, p->head_dim, e) || !strides_ok(&a->v_row, &a->v_head, p->kv_heads, p->head_dim, e) ||
      !strides_ok(&a->ck_row, &a->ck_head, p->kv_heads, p->head_dim, 16) || !strides_ok(&a->cv_row, &a->cv_head, p->kv_heads, p->head_dim, 16))
    return bad("strides must be >= 0 and multiples of 16 bytes");
  if (!apart(p->total_k, a->ck_row, p->kv_heads, a->ck_head, p->head_dim) || !apart(p->total_k, a->cv_row, p->kv_heads, a->cv_head, p->head_dim))
    return bad("the cache's rows and heads may not overlap");
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
  for (const auto& s : st)
    if (!strides_ok(s.row, s.head, s.heads, p->head_dim, e)) return bad("strides must be >= 0 and multiples of 16 bytes");
  return BSA_OK;
}

// The strides of k and v are bytes of the cache.
bsa_status_t check_cache(const bsa_attention_t* p, bsa::AttnArgs* a) {
  const bsa_status_t s = check(p, a);
  if (s != BSA_OK) return s;
  a->k_row = p->k_row, a->k_head = p->k_head, a->v_row = p->v_row, a->v_head = p->v_head;
  if (!strides_ok(&a->k_row, &a->k_head, a->kv_heads, a->hd, 16) || !strides_ok(&a->v_row, &a->v_head, a->kv_heads, a->hd, 16))
    return bad("strides of the cache must be multiples of 16 bytes");
  return s;
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

bsa_status_t bsa_gated_sizes(const bsa_gated_t* p, size_t* ws_fwd_bytes, size_t* ws_bwd_bytes) {
  return entry([&] {
    bsa::GatedArgs a;
    const bsa_status_t s = check(p, &a);
    if (s != BSA_OK) return s;
    if (ws_fwd_bytes) *ws_fwd_bytes = bsa::gated_fwd_ws_bytes(a);
    if (ws_bwd_bytes) *ws_bwd_bytes = bsa::gated_bwd_ws_bytes(a);
    return s;
  });
}

bsa_status_t bsa_gated_forward(const bsa_gated_t* p, const void* x, const void* w, const void* bias, void* y, void* pre,
                               void* ws, size_t ws_bytes, void* stream) {
  return entry([&] {
    bsa::GatedArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK || a.m == 0) return s;
    if (!x || !w || !y) return bad("x, w and y must be non-NULL");
    if (on_one(y, {x, w, bias, pre})) return bad("y may not alias x, w, bias or pre");
    if (on_one(pre, {x, w, bias})) return bad("pre may not alias an input");
    const size_t need = bsa::gated_fwd_ws_bytes(a);
    if (need && (!ws || ws_bytes < need)) return small_ws("gated map forward", need);
    if (need && !aligned(ws, 16)) return bad("ws must be 16-byte aligned");
    hipError_t e;
    BSA_PHASE("gated.fwd", (hipStream_t)stream, e = bsa::launch_gated_fwd(a, x, w, bias, y, pre, ws, (hipStream_t)stream));
    return launched(e, "bsa_gated_forward");
  });
}

bsa_status_t bsa_gated_backward(const bsa_gated_t* p, const void* x, const void* w, const void* pre, const void* dy, void* dx,
                                void* dw, void* db, void* ws, size_t ws_bytes, void* stream) {
  return entry([&] {
    bsa::GatedArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK) return s;
    if (!dx && !dw && !db) return BSA_OK;
    if (a.m > 0) {
      if (!dy || !pre) return bad("dy and pre must be non-NULL");
      if (dx && !w) return bad("w must be non-NULL for dx");
      if (dw && !x) return bad("x must be non-NULL for dw");
    }
    for (const void* g : {dx, dw, db})
      if (on_one(g, {x, w, pre, dy})) return bad("a gradient may not alias an input");
    const size_t need = bsa::gated_bwd_ws_bytes(a);
    if (need && (!ws || ws_bytes < need)) return small_ws("gated map backward", need);
    if (need && !aligned(ws, 16)) return bad("ws must be 16-byte aligned");
    hipError_t e;
    BSA_PHASE("gated.bwd", (hipStream_t)stream,
              e = bsa::launch_gated_bwd(a, x, w, pre, dy, dx, dw, db, ws, (hipStream_t)stream));
    return launched(e, "bsa_gated_backward");
  });
}

bsa_status_t bsa_rotary_sizes(const bsa_rotary_t* p, size_t* ws_bwd_bytes) {
  return entry([&] {
    bsa::RotaryArgs a;
    const bsa_status_t s = check(p, &a);
    if (s == BSA_OK && ws_bwd_bytes) *ws_bwd_bytes = bsa::rotary_bwd_ws_bytes(a);
    return s;
  });
}

bsa_status_t bsa_rotary_forward(const bsa_rotary_t* p, const void* q, const void* k, const void* positions, const double* freq,
                                const float* gain_q, const float* gain_k, void* y_q, void* y_k, void* stream) {
  return entry([&] {
    bsa::RotaryArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK || a.rows == 0) return s;
    if (!q || !positions || !freq || !y_q) return bad("q, positions, freq and y_q must be non-NULL");
    if (a.kv_heads && (!k || !y_k)) return bad("k and y_k must be non-NULL with key heads");
    if (y_q == y_k || (a.kv_heads && (y_q == k || y_k == q))) return bad("y_q and y_k may only be q and k");
    if (on_other_strides(y_q, a.oq_row, a.oq_head, q, a.q_row, a.q_head) ||
        on_other_strides(y_k, a.ok_row, a.ok_head, k, a.k_row, a.k_head))
      return bad("an output may be its input only with the same strides");
    hipError_t e;
    BSA_PHASE("rotary.fwd", (hipStream_t)stream,
              e = bsa::launch_rotary_fwd(a, q, k, positions, freq, gain_q, gain_k, y_q, y_k, (hipStream_t)stream));
    return launched(e, "bsa_rotary_forward");
  });
}

bsa_status_t bsa_rotary_backward(const bsa_rotary_t* p, const void* q, const void* k, const void* positions, const double* freq,
                                 const float* gain_q, const float* gain_k, const void* dy_q, const void* dy_k, void* dq,
                                 void* dk, float* dgain_q, float* dgain_k, void* ws, size_t ws_bytes, void* stream) {
  return entry([&] {
    bsa::RotaryArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK) return s;
    if (a.kv_heads == 0) k = dy_k = gain_k = nullptr, dk = dgain_k = nullptr;
    if ((dgain_q && !gain_q) || (dgain_k && !gain_k)) return bad("a gain's gradient needs the gain");
    if (a.rows > 0) {
      if (!positions || !freq || !dy_q || !dq) return bad("positions, freq, dy_q and dq must be non-NULL");
      if (a.kv_heads && (!dy_k || !dk)) return bad("dy_k and dk must be non-NULL with key heads");
      if ((gain_q && !q) || (gain_k && !k)) return bad("q and k must be non-NULL with their gains");
      if (dq == dk || (a.kv_heads && (dq == k || dq == dy_k || dk == q || dk == dy_q)))
        return bad("dq may only be q or dy_q, dk only k or dy_k");
      if (on_other_strides(dq, a.oq_row, a.oq_head, gain_q ? q : nullptr, a.q_row, a.q_head) ||
          on_other_strides(dq, a.oq_row, a.oq_head, dy_q, a.dq_row, a.dq_head) ||
          on_other_strides(dk, a.ok_row, a.ok_head, gain_k ? k : nullptr, a.k_row, a.k_head) ||
          on_other_strides(dk, a.ok_row, a.ok_head, dy_k, a.dk_row, a.dk_head))
        return bad("a gradient may be an input only with the same strides");
    }
    const size_t need = gain_q || gain_k ? bsa::rotary_bwd_ws_bytes(a) : 0;
    if (need && (!ws || ws_bytes < need)) return small_ws("rotary backward", need);
    hipError_t e;
    BSA_PHASE("rotary.bwd", (hipStream_t)stream,
              e = bsa::launch_rotary_bwd(a, q, k, positions, freq, gain_q, gain_k, dy_q, dy_k, dq, dk, dgain_q, dgain_k, ws,
                                         (hipStream_t)stream));
    return launched(e, "bsa_rotary_backward");
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
    if (!apart(a.total_q, a.o_row, a.heads, a.o_head, a.hd)) return bad("o's rows and heads may not overlap");
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

bsa_status_t bsa_cache_write(const bsa_cache_t* p, const void* k, const void* v, const int32_t* cu_q, const int32_t* cu_k,
                             const int32_t* used_k, void* cache_k, void* cache_v, uint8_t* exp_k, uint8_t* exp_v, void* stream) {
  return entry([&] {
    bsa::CacheArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK || a.rows == 0 || a.total_k == 0) return s;
    if (!k || !v || !cu_q || !cu_k || !cache_k || !cache_v || !exp_k || !exp_v) return bad("every pointer but used_k must be non-NULL");
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cache_k, 16) || !aligned(cache_v, 16))
      return bad("k, v and the cache must be 16-byte aligned");
    if (on_one(cache_k, {k, v, cache_v}) || on_one(cache_v, {k, v}) || exp_k == exp_v) return bad("the cache may not alias an input or itself");
    hipError_t e;
    BSA_PHASE("cache.write", (hipStream_t)stream,
              e = bsa::launch_cache_write(a, k, v, cu_q, cu_k, used_k, cache_k, cache_v, exp_k, exp_v, (hipStream_t)stream));
    return launched(e, "bsa_cache_write");
  });
}

bsa_status_t bsa_cache_read(const bsa_cache_t* p, const void* cache_k, const void* cache_v, const uint8_t* exp_k,
                            const uint8_t* exp_v, const int32_t* cu_q, const int32_t* cu_k, const int32_t* used_k, void* k,
                            void* v, void* stream) {
  return entry([&] {
    bsa::CacheArgs a;
    bsa_status_t s = check(p, &a);
    if (s != BSA_OK || a.rows == 0) return s;
    if (!k || !v || !cu_q || !cu_k) return bad("k, v, cu_q and cu_k must be non-NULL");
    if (a.total_k > 0 && (!cache_k || !cache_v || !exp_k || !exp_v)) return bad("the cache must be non-NULL");
    if (!aligned(k, 16) || !aligned(v, 16) || !aligned(cache_k, 16) || !aligned(cache_v, 16))
      return bad("k, v and the cache must be 16-byte aligned");
    if (on_one(k, {cache_k, cache_v, v}) || on_one(v, {cache_k, cache_v})) return bad("k and v may not alias the cache or each other");
    if (!apart(a.rows, a.k_row, a.kv_heads, a.k_head, a.hd) || !apart(a.rows, a.v_row, a.kv_heads, a.v_head, a.hd))
      return bad("rows and heads of k and v may not overlap");
    hipError_t e;
    BSA_PHASE("cache.read", (hipStream_t)stream,
              e = bsa::launch_cache_read(a, cache_k, cache_v, exp_k, exp_v, cu_q, cu_k, used_k, k, v, (hipStream_t)stream));
    return launched(e, "bsa_cache_read");
  });
}

bsa_status_t bsa_cache_attention_sizes(const bsa_attention_t* p, size_t* ws_bytes) {
  return entry([&] {
    bsa::AttnArgs a;
    const bsa_status_t s = check_cache(p, &a);
    if (s == BSA_OK && ws_bytes) *ws_bytes = bsa::cache_attention_ws_bytes(a);
    return s;
  });
}

bsa_status_t bsa_cache_attention_forward(const bsa_attention_t* p, const void* q, const void* cache_k, const void* cache_v,
                                         const uint8_t* exp_k, const uint8_t* exp_v, const int32_t* cu_q, const int32_t* cu_k,
                                         const int32_t* used_k, void* o, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return entry([&] {
    bsa::AttnArgs a;
    bsa_status_t s = check_cache(p, &a);
    if (s != BSA_OK || a.total_q == 0) return s;
    if (!bsa::cache_attention_fits(a)) return set_error(BSA_ERR_UNSUPPORTED, kTooManyTiles);
    if (!q || !cu_q || !cu_k || !o || !lse) return bad("q, cu_q, cu_k, o and lse must be non-NULL");
    if (a.total_k > 0 && (!cache_k || !cache_v || !exp_k || !exp_v)) return bad("the cache must be non-NULL");
    if (on_one(o, {q, cache_k, cache_v})) return bad("o may not alias an input");
    if (!apart(a.total_q, a.o_row, a.heads, a.o_head, a.hd)) return bad("o's rows and heads may not overlap");
    if (!aligned(q, 16) || !aligned(cache_k, 16) || !aligned(cache_v, 16) || !aligned(o, 16))
      return bad("q, the cache and o must be 16-byte aligned");
    const size_t need = bsa::cache_attention_ws_bytes(a);
    if (need && (!ws || ws_bytes < need)) return small_ws("cache attention", need);
    if (need && !aligned(ws, 16)) return bad("ws must be 16-byte aligned");
    hipError_t e;
    BSA_PHASE("cache.attn", (hipStream_t)stream,
              e = bsa::launch_cache_attention(a, q, cache_k, cache_v, exp_k, exp_v, cu_q, cu_k, used_k, o, lse, ws,
                                              (hipStream_t)stream));
    return launched(e, "bsa_cache_attention_forward");
  });
}

}  // extern "C"
