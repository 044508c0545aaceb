// Entry points of the stand-alone operators: argument checks and launches.
#include <math.h>

#include <algorithm>

#include "host.hpp"
#include "ops.hpp"

using namespace cs;

static int elem(int dtype) { return dtype == CS_BF16 ? 2 : dtype == CS_I8 ? 1 : 4; }
static bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

static cs_status check_dtype(int dtype) {
  CHECK(dtype == CS_BF16 || dtype == CS_FP32, CS_E_INVAL, "dtype must be CS_BF16 or CS_FP32");
  return CS_OK;
}

static cs_status check_tensor(const void* p, const char* name) {
  CHECK(p, CS_E_INVAL, "%s is NULL", name);
  CHECK(aligned(p), CS_E_INVAL, "%s must be 16-byte aligned", name);
  return CS_OK;
}

// Stride of an axis with n entries: whole 16-byte units, the axis within 2^60
// bytes.  An axis of one entry may have any stride.
static cs_status check_stride(long s, long n, int esz, const char* name) {
  if (n <= 1) return CS_OK;
  CHECK(s >= 0 && s % (16 / esz) == 0, CS_E_INVAL, "stride %s must be a non-negative multiple of 16 bytes", name);
  CHECK(s < (1L << 60) / n / esz, CS_E_UNSUPPORTED, "stride %s is too large", name);
  return CS_OK;
}

// The same of an output: its entries lie apart.
static cs_status check_out_stride(long s, long n, int esz, const char* name) {
  TRY(check_stride(s, n, esz, name));
  CHECK(n <= 1 || s > 0, CS_E_INVAL, "output stride %s must be positive", name);
  return CS_OK;
}

// A tensor that may be absent.
static cs_status check_optional(const void* p, const char* name) { return p ? check_tensor(p, name) : CS_OK; }

static cs_status check_work(const void* work, size_t bytes, size_t need) {
  if (need == 0) return CS_OK;
  CHECK(work && aligned(work), CS_E_INVAL, "a 16-byte aligned workspace is needed");
  CHECK(bytes >= need, CS_E_INVAL, "the workspace holds %zu bytes, %zu needed", bytes, need);
  return CS_OK;
}

extern "C" {

cs_status cs_qk_norm_rope(const cs_qk_norm_desc* d, const void* q, const void* k, void* q_out, void* k_out,
                          const float* q_gain, const float* k_gain, const float* rope, const int32_t* pos,
                          void* stream) {
  GUARD({
    CHECK(d, CS_E_INVAL, "desc is NULL");
    TRY(check_dtype(d->dtype));
    CHECK(d->tokens >= 0 && d->heads_q >= 0 && d->heads_k >= 0, CS_E_INVAL, "tokens and heads must not be negative");
    CHECK(d->head_dim >= 16, CS_E_INVAL, "head_dim must be at least 16");
    CHECK(d->head_dim % 16 == 0 && d->head_dim <= 256, CS_E_UNSUPPORTED,
          "head_dim must be a multiple of 16 up to 256");
    CHECK(d->rot_dim >= 0 && d->rot_dim <= d->head_dim, CS_E_INVAL, "rot_dim must be in 0..head_dim");
    CHECK(d->rot_dim % 16 == 0, CS_E_UNSUPPORTED, "rot_dim must be a multiple of 16");
    CHECK(d->rope_style == CS_ROPE_PAIRS || d->rope_style == CS_ROPE_HALVES, CS_E_INVAL, "unknown rope_style %d",
          d->rope_style);
    CHECK(d->rot_dim == 0 || d->rope_rows >= 1, CS_E_INVAL, "rope_rows must be positive");
    CHECK(d->eps >= 0.0f && isfinite(d->eps), CS_E_INVAL, "eps must be finite and not negative");
    const int e = elem(d->dtype);
    if (d->heads_q > 0) {
      TRY(check_stride(d->q_row, d->tokens, e, "q_row"));
      TRY(check_stride(d->q_head, d->heads_q, e, "q_head"));
      TRY(check_out_stride(d->qo_row, d->tokens, e, "qo_row"));
      TRY(check_out_stride(d->qo_head, d->heads_q, e, "qo_head"));
      TRY(check_stride(d->q_gain_head, d->heads_q, 4, "q_gain_head"));
    }
    if (d->heads_k > 0) {
      TRY(check_stride(d->k_row, d->tokens, e, "k_row"));
      TRY(check_stride(d->k_head, d->heads_k, e, "k_head"));
      TRY(check_out_stride(d->ko_row, d->tokens, e, "ko_row"));
      TRY(check_out_stride(d->ko_head, d->heads_k, e, "ko_head"));
      TRY(check_stride(d->k_gain_head, d->heads_k, 4, "k_gain_head"));
    }
    if (d->tokens == 0 || (d->heads_q == 0 && d->heads_k == 0)) return CS_OK;
    if (d->heads_q > 0) {
      TRY(check_tensor(q, "q"));
      TRY(check_tensor(q_out, "q_out"));
      TRY(check_tensor(q_gain, "q_gain"));
    }
    if (d->heads_k > 0) {
      TRY(check_tensor(k, "k"));
      TRY(check_tensor(k_out, "k_out"));
      TRY(check_tensor(k_gain, "k_gain"));
    }
    if (d->rot_dim > 0) TRY(check_tensor(rope, "rope"));
    QkNormArgs a = {q, k, q_out, k_out, q_gain, k_gain, rope, pos, *d};
    if (d->rot_dim == 0) a.d.rope_rows = 0;
    hipError_t s = d->dtype == CS_BF16 ? qk_norm_rope<bf16>(a, (hipStream_t)stream)
                                       : qk_norm_rope<float>(a, (hipStream_t)stream);
    CHECK(s != hipErrorInvalidConfiguration, CS_E_UNSUPPORTED, "too many tokens and heads for one call");
    HIPC(s);
    return CS_OK;
  })
}

// ------------------------------------------------------------ 4-bit cache
static cs_status check_cache(const cs_kv4_cache* c) {
  CHECK(c, CS_E_INVAL, "cache is NULL");
  CHECK(c->n_kv >= 1 && c->heads >= 1 && c->cap >= 1, CS_E_INVAL, "cache dimensions must be positive");
  CHECK(c->head_dim == 32 || c->head_dim == 64 || c->head_dim == 128, CS_E_UNSUPPORTED,
        "head_dim must be 32, 64 or 128");
  CHECK((long)c->n_kv * c->cap < (1L << 31), CS_E_UNSUPPORTED, "n_kv * cap must be below 2^31");
  TRY(check_tensor(c->k_codes, "k_codes"));
  TRY(check_tensor(c->k_scales, "k_scales"));
  TRY(check_tensor(c->v_codes, "v_codes"));
  TRY(check_tensor(c->v_scales, "v_scales"));
  return CS_OK;
}

static cs_status kv4_rows_call(const cs_kv4_cache* c, const cs_kv4_rows* r, const void* k, const void* v, void* ko,
                               void* vo, const int32_t* slots, bool store, void* stream) {
  TRY(check_cache(c));
  CHECK(r, CS_E_INVAL, "rows is NULL");
  TRY(check_dtype(r->dtype));
  CHECK(r->n_rows >= 0, CS_E_INVAL, "n_rows must not be negative");
  CHECK(slots || (long)r->n_rows <= (long)c->n_kv * c->cap, CS_E_INVAL, "%d rows without slots, the cache has %ld",
        r->n_rows, (long)c->n_kv * c->cap);
  const int e = elem(r->dtype);
  const auto check = store ? check_stride : check_out_stride;
  TRY(check(r->k_row, r->n_rows, e, "k_row"));
  TRY(check(r->k_head, c->heads, e, "k_head"));
  TRY(check(r->v_row, r->n_rows, e, "v_row"));
  TRY(check(r->v_head, c->heads, e, "v_head"));
  if (r->n_rows == 0) return CS_OK;
  TRY(check_tensor(store ? k : ko, "k"));
  TRY(check_tensor(store ? v : vo, "v"));
  const Kv4RowsArgs a = {*c, *r, k, v, ko, vo, slots, nullptr, nullptr};
  hipStream_t st = (hipStream_t)stream;
  hipError_t s;
  if (r->dtype == CS_BF16)
    s = store ? kv4_store<bf16>(a, st) : kv4_load<bf16>(a, st);
  else
    s = store ? kv4_store<float>(a, st) : kv4_load<float>(a, st);
  CHECK(s != hipErrorInvalidConfiguration, CS_E_UNSUPPORTED, "too many rows and heads for one call");
  HIPC(s);
  return CS_OK;
}

cs_status cs_kv4_store(const cs_kv4_cache* cache, const cs_kv4_rows* rows, const void* k, const void* v,
                       const int32_t* slots, void* stream) {
  GUARD({ return kv4_rows_call(cache, rows, k, v, nullptr, nullptr, slots, true, stream); })
}

cs_status cs_kv4_load(const cs_kv4_cache* cache, const cs_kv4_rows* rows, void* k, void* v, const int32_t* slots,
                      void* stream) {
  GUARD({ return kv4_rows_call(cache, rows, nullptr, nullptr, k, v, slots, false, stream); })
}

// -------------------------------------------------------------- attention
static cs_status check_attn(const cs_attn_desc* d, bool kv4) {
  CHECK(d, CS_E_INVAL, "desc is NULL");
  TRY(check_dtype(d->dtype));
  CHECK(d->n_q >= 0 && d->lq >= 0 && d->lk >= 0, CS_E_INVAL, "n_q, lq and lk must not be negative");
  CHECK(d->n_kv >= 1 || d->n_q == 0, CS_E_INVAL, "n_kv must be positive");
  CHECK(d->heads_q >= 1 && d->heads_kv >= 1, CS_E_INVAL, "heads must be positive");
  CHECK(d->heads_q % d->heads_kv == 0, CS_E_INVAL, "heads_q must be a multiple of heads_kv");
  CHECK(d->head_dim == 32 || d->head_dim == 64 || d->head_dim == 128, CS_E_UNSUPPORTED,
        "head_dim must be 32, 64 or 128");
  CHECK(d->scale > 0.0f && d->scale < 1e38f, CS_E_INVAL, "scale must be positive and below 1e38");
  CHECK(d->mask_b >= 0, CS_E_INVAL, "stride mask_b must not be negative");
  // rows of a set: queries x the heads that share a key head
  CHECK((long)d->lq * (d->heads_q / d->heads_kv) < (1L << 30) && d->lk < (1 << 30), CS_E_UNSUPPORTED,
        "lq x heads and lk must be below 2^30");
  // what grids and workspaces are computed from stays in 64 bits
  CHECK((double)d->n_q * d->heads_q * std::max(d->lq, 1) < 0x1p40, CS_E_UNSUPPORTED,
        "too many queries and heads for one call");
  CHECK(!kv4 || (double)d->n_kv * d->lk < 0x1p31, CS_E_UNSUPPORTED, "n_kv * lk must be below 2^31");
  // offsets inside a tile of keys are 32-bit byte counts
  CHECK(kv4 || d->lk <= 1 || (d->k_r <= (1 << 23) && d->v_r <= (1 << 23)), CS_E_UNSUPPORTED,
        "strides k_r and v_r must be at most 2^23");
  CHECK(!kv4 || (long)d->heads_kv * d->head_dim <= (1 << 23), CS_E_UNSUPPORTED, "heads_kv * head_dim must be at most 2^23");
  CHECK((d->lq <= 1 || (d->q_r < (1L << 31) && d->o_r < (1L << 31))) &&
            (d->heads_q <= 1 || (d->q_h < (1L << 31) && d->o_h < (1L << 31))),
        CS_E_UNSUPPORTED, "strides q_r, q_h, o_r and o_h must be below 2^31");
  const int e = elem(d->dtype);
  TRY(check_stride(d->q_b, d->n_q, e, "q_b"));
  TRY(check_stride(d->q_r, d->lq, e, "q_r"));
  TRY(check_stride(d->q_h, d->heads_q, e, "q_h"));
  TRY(check_out_stride(d->o_b, d->n_q, e, "o_b"));
  TRY(check_out_stride(d->o_r, d->lq, e, "o_r"));
  TRY(check_out_stride(d->o_h, d->heads_q, e, "o_h"));
  if (!kv4) {
    TRY(check_stride(d->k_b, d->n_kv, e, "k_b"));
    TRY(check_stride(d->k_r, d->lk, e, "k_r"));
    TRY(check_stride(d->k_h, d->heads_kv, e, "k_h"));
    TRY(check_stride(d->v_b, d->n_kv, e, "v_b"));
    TRY(check_stride(d->v_r, d->lk, e, "v_r"));
    TRY(check_stride(d->v_h, d->heads_kv, e, "v_h"));
  }
  return CS_OK;
}

static cs_status attn_call(const cs_attn_desc* d, const void* q, const void* k, const void* v,
                           const cs_kv4_cache* cache, const int32_t* kv_of, const int32_t* kv_len,
                           const uint8_t* kv_mask, void* o, void* work, size_t work_bytes, void* stream) {
  const bool kv4 = cache != nullptr;
  CHECK(kv_of || d->n_kv >= d->n_q, CS_E_INVAL, "%d query sets and %d contexts need kv_of", d->n_q, d->n_kv);
  if (d->n_q == 0 || d->lq == 0) return CS_OK;
  TRY(check_tensor(q, "q"));
  TRY(check_tensor(o, "o"));
  if (!kv4 && d->lk > 0) {
    TRY(check_tensor(k, "k"));
    TRY(check_tensor(v, "v"));
  }
  TRY(check_work(work, work_bytes, xattn_workspace(*d, kv4)));
  XAttnArgs a = {q, k, v, o, kv_of, kv_len, false, kv_mask, {}, *d, (float)(1.4426950408889634 * d->scale)};
  if (kv4) a.c = *cache;
  if (d->lk == 1) a.d.k_r = a.d.v_r = d->head_dim;   // never checked
  hipStream_t st = (hipStream_t)stream;
  const hipError_t s = d->dtype == CS_BF16 ? xattn<bf16>(a, kv4, work, st) : xattn<float>(a, kv4, work, st);
  CHECK(s != hipErrorInvalidConfiguration, CS_E_UNSUPPORTED, "too many queries and heads for one call");
  HIPC(s);
  return CS_OK;
}

cs_status cs_cross_attention_workspace(const cs_attn_desc* desc, size_t* bytes) {
  GUARD({
    TRY(check_attn(desc, false));
    CHECK(bytes, CS_E_INVAL, "bytes is NULL");
    *bytes = xattn_workspace(*desc, false);
    return CS_OK;
  })
}

cs_status cs_cross_attention(const cs_attn_desc* desc, const void* q, const void* k, const void* v,
                             const int32_t* kv_of, const int32_t* kv_len, const uint8_t* kv_mask, void* o,
                             void* work, size_t work_bytes, void* stream) {
  GUARD({
    TRY(check_attn(desc, false));
    return attn_call(desc, q, k, v, nullptr, kv_of, kv_len, kv_mask, o, work, work_bytes, stream);
  })
}

cs_status cs_kv4_attention_workspace(const cs_attn_desc* desc, size_t* bytes) {
  GUARD({
    TRY(check_attn(desc, true));
    CHECK(bytes, CS_E_INVAL, "bytes is NULL");
    *bytes = xattn_workspace(*desc, true);
    return CS_OK;
  })
}

cs_status cs_kv4_attention(const cs_attn_desc* desc, const void* q, const cs_kv4_cache* cache, const int32_t* kv_of,
                           const int32_t* kv_len, const uint8_t* kv_mask, void* o, void* work, size_t work_bytes,
                           void* stream) {
  GUARD({
    TRY(check_attn(desc, true));
    TRY(check_cache(cache));
    CHECK(desc->n_kv == cache->n_kv && desc->lk == cache->cap && desc->heads_kv == cache->heads &&
              desc->head_dim == cache->head_dim,
          CS_E_INVAL, "n_kv, lk, heads_kv and head_dim must be the cache's");
    return attn_call(desc, q, nullptr, nullptr, cache, kv_of, kv_len, kv_mask, o, work, work_bytes, stream);
  })
}

// A launch that does not fit a grid, or the error it ended with.
static cs_status launched(hipError_t s, const char* what) {
  CHECK(s != hipErrorInvalidConfiguration, CS_E_UNSUPPORTED, "too many %s for one call", what);
  HIPC(s);
  return CS_OK;
}

// ------------------------------------------------------------- layer norm
// What the two descriptors have in common.
static cs_status check_norm_rows(int x_dtype, int groups, int rows, int dim, int unit_offset, long w_group) {
  CHECK(x_dtype == CS_BF16 || x_dtype == CS_FP32, CS_E_INVAL, "x_dtype must be CS_BF16 or CS_FP32");
  CHECK(groups >= 0 && rows >= 0, CS_E_INVAL, "groups and rows must not be negative");
  CHECK((long)groups * rows < (1L << 30), CS_E_UNSUPPORTED, "groups * rows must be below 2^30");
  CHECK(dim >= 1, CS_E_INVAL, "dim must be positive");
  CHECK(dim <= LN_MAX_DIM, CS_E_UNSUPPORTED, "dim must be at most %d", LN_MAX_DIM);
  CHECK(unit_offset == 0 || unit_offset == 1, CS_E_INVAL, "unit_offset must be 0 or 1");
  return check_stride(w_group, groups, 4, "w_group");
}

cs_status cs_layer_norm(const cs_layer_norm_desc* d, const void* x, const float* weight, const float* bias, void* y,
                        float* y_scale, float* mean, float* rstd, void* stream) {
  GUARD({
    CHECK(d, CS_E_INVAL, "desc is NULL");
    TRY(check_norm_rows(d->x_dtype, d->groups, d->rows, d->dim, d->unit_offset, d->w_group));
    CHECK(d->y_dtype == CS_BF16 || d->y_dtype == CS_FP32 || d->y_dtype == CS_I8, CS_E_INVAL,
          "y_dtype must be CS_BF16, CS_FP32 or CS_I8");
    CHECK(d->eps >= 0.0f && isfinite(d->eps), CS_E_INVAL, "eps must be finite and not negative");
    const long total = (long)d->groups * d->rows;
    TRY(check_stride(d->b_group, d->groups, 4, "b_group"));
    TRY(check_stride(d->x_row, total, elem(d->x_dtype), "x_row"));
    TRY(check_out_stride(d->y_row, total, elem(d->y_dtype), "y_row"));
    if (total == 0) return CS_OK;
    TRY(check_tensor(x, "x"));
    TRY(check_tensor(y, "y"));
    TRY(check_optional(weight, "weight"));
    TRY(check_optional(bias, "bias"));
    if (d->y_dtype == CS_I8) TRY(check_tensor(y_scale, "y_scale"));
    TRY(check_optional(mean, "mean"));
    TRY(check_optional(rstd, "rstd"));
    return launched(layer_norm({x, weight, bias, y, y_scale, mean, rstd, *d}, (hipStream_t)stream), "rows");
  })
}

static cs_status check_norm_grad(const cs_layer_norm_grad_desc* d) {
  CHECK(d, CS_E_INVAL, "desc is NULL");
  TRY(check_norm_rows(d->x_dtype, d->groups, d->rows, d->dim, d->unit_offset, d->w_group));
  CHECK(d->y_dtype == CS_BF16 || d->y_dtype == CS_FP32, CS_E_INVAL, "y_dtype must be CS_BF16 or CS_FP32");
  const long total = (long)d->groups * d->rows;
  TRY(check_stride(d->x_row, total, elem(d->x_dtype), "x_row"));
  TRY(check_stride(d->dy_row, total, elem(d->y_dtype), "dy_row"));
  return CS_OK;
}

cs_status cs_layer_norm_backward_workspace(const cs_layer_norm_grad_desc* desc, size_t* bytes) {
  GUARD({
    TRY(check_norm_grad(desc));
    CHECK(bytes, CS_E_INVAL, "bytes is NULL");
    *bytes = layer_norm_backward_workspace(*desc);
    return CS_OK;
  })
}

cs_status cs_layer_norm_backward(const cs_layer_norm_grad_desc* d, const void* x, const void* dy, const float* weight,
                                 const float* mean, const float* rstd, void* dx, float* dweight, float* dbias,
                                 void* work, size_t work_bytes, void* stream) {
  GUARD({
    TRY(check_norm_grad(d));
    const long total = (long)d->groups * d->rows;
    if (dx) TRY(check_out_stride(d->dx_row, total, elem(d->x_dtype), "dx_row"));
    if (dweight) TRY(check_out_stride(d->dw_group, d->groups, 4, "dw_group"));
    if (dbias) TRY(check_out_stride(d->db_group, d->groups, 4, "db_group"));
    if (d->groups == 0 || (!dx && !dweight && !dbias)) return CS_OK;
    if (total > 0) {
      TRY(check_tensor(x, "x"));
      TRY(check_tensor(dy, "dy"));
      TRY(check_tensor(mean, "mean"));
      TRY(check_tensor(rstd, "rstd"));
    }
    TRY(check_optional(weight, "weight"));
    TRY(check_optional(dx, "dx"));
    TRY(check_optional(dweight, "dweight"));
    TRY(check_optional(dbias, "dbias"));
    float* part = nullptr;
    if (dweight || dbias) {
      TRY(check_work(work, work_bytes, layer_norm_backward_workspace(*d)));
      part = (float*)work;
    }
    return launched(layer_norm_backward({x, dy, weight, mean, rstd, dx, dweight, dbias, part, *d}, (hipStream_t)stream),
                    "groups and rows");
  })
}

// ------------------------------------------------------------------ 8 bits
static cs_status i8_rows_call(const cs_i8_rows* r, const void* x, void* x_out, const int8_t* codes, const float* scales,
                              bool store, void* stream) {
  CHECK(r, CS_E_INVAL, "rows is NULL");
  TRY(check_dtype(r->dtype));
  CHECK(r->rows >= 0, CS_E_INVAL, "rows must not be negative");
  CHECK(r->dim >= 1, CS_E_INVAL, "dim must be positive");
  CHECK(r->dim <= I8_MAX_DIM, CS_E_UNSUPPORTED, "dim must be at most %d", I8_MAX_DIM);
  TRY((store ? check_stride : check_out_stride)(r->x_row, r->rows, elem(r->dtype), "x_row"));
  TRY((store ? check_out_stride : check_stride)(r->q_row, r->rows, 1, "q_row"));
  if (r->rows == 0) return CS_OK;
  TRY(check_tensor(store ? x : x_out, "x"));
  TRY(check_tensor(codes, "codes"));
  TRY(check_tensor(scales, "scales"));
  const I8RowsArgs a = {x, x_out, (int8_t*)codes, (float*)scales, *r};
  return launched(store ? i8_quantise(a, (hipStream_t)stream) : i8_dequantise(a, (hipStream_t)stream), "rows");
}

cs_status cs_i8_quantise(const cs_i8_rows* rows, const void* x, int8_t* codes, float* scales, void* stream) {
  GUARD({ return i8_rows_call(rows, x, nullptr, codes, scales, true, stream); })
}

cs_status cs_i8_dequantise(const cs_i8_rows* rows, const int8_t* codes, const float* scales, void* x, void* stream) {
  GUARD({ return i8_rows_call(rows, nullptr, x, codes, scales, false, stream); })
}

static cs_status check_weight_size(int n, int k) {
  CHECK(n >= 1 && k >= 1, CS_E_INVAL, "n and k must be positive");
  CHECK(n <= (1 << 24), CS_E_UNSUPPORTED, "n must be at most 2^24");
  CHECK(k <= I8_MAX_DIM, CS_E_UNSUPPORTED, "k must be at most %d", I8_MAX_DIM);
  return CS_OK;
}

static cs_status check_weight(const cs_i8_weight* w) {
  CHECK(w, CS_E_INVAL, "weight is NULL");
  TRY(check_weight_size(w->n, w->k));
  TRY(check_tensor(w->codes, "weight codes"));
  TRY(check_tensor(w->scales, "weight scales"));
  return CS_OK;
}

cs_status cs_i8_weight_bytes(int32_t n, int32_t k, size_t* bytes) {
  GUARD({
    TRY(check_weight_size(n, k));
    CHECK(bytes, CS_E_INVAL, "bytes is NULL");
    *bytes = (size_t)i8_weight_bytes(n, k);
    return CS_OK;
  })
}

cs_status cs_i8_weight_pack(const cs_i8_weight* weight, int32_t dtype, const void* w, int64_t w_row,
                            const float* w_scales, void* stream) {
  GUARD({
    TRY(check_weight(weight));
    CHECK(dtype == CS_BF16 || dtype == CS_FP32 || dtype == CS_I8, CS_E_INVAL,
          "dtype must be CS_BF16, CS_FP32 or CS_I8");
    TRY(check_stride(w_row, weight->n, elem(dtype), "w_row"));
    TRY(check_tensor(w, "w"));
    CHECK(dtype == CS_I8 || !w_scales, CS_E_INVAL, "w_scales belong to CS_I8 codes only");
    if (dtype == CS_I8) TRY(check_tensor(w_scales, "w_scales"));
    HIPC(i8_weight_pack(*weight, dtype, w, w_row, w_scales, (hipStream_t)stream));
    return CS_OK;
  })
}

static cs_status check_matmul(const cs_matmul_i8_desc* d) {
  CHECK(d, CS_E_INVAL, "desc is NULL");
  CHECK(d->out_dtype == CS_BF16 || d->out_dtype == CS_FP32, CS_E_INVAL, "out_dtype must be CS_BF16 or CS_FP32");
  CHECK(d->rows >= 0, CS_E_INVAL, "rows must not be negative");
  CHECK(d->rows <= (1 << 30), CS_E_UNSUPPORTED, "rows must be at most 2^30");
  TRY(check_weight_size(d->n, d->k));
  CHECK(d->act == CS_ACT_NONE || d->act == CS_ACT_GELU, CS_E_INVAL, "unknown act %d", d->act);
  TRY(check_stride(d->a_row, d->rows, 1, "a_row"));
  // offsets inside a tile of rows are 32-bit byte counts
  CHECK(d->rows <= 1 || d->a_row <= (1 << 22), CS_E_UNSUPPORTED, "stride a_row must be at most 2^22");
  return check_out_stride(d->o_row, d->rows, elem(d->out_dtype), "o_row");
}

cs_status cs_matmul_i8_workspace(const cs_matmul_i8_desc* desc, size_t* bytes) {
  GUARD({
    TRY(check_matmul(desc));
    CHECK(bytes, CS_E_INVAL, "bytes is NULL");
    *bytes = matmul_i8_workspace(*desc);
    return CS_OK;
  })
}

cs_status cs_matmul_i8(const cs_matmul_i8_desc* d, const int8_t* a, const float* a_scales, const cs_i8_weight* weight,
                       const float* bias, void* out, void* work, size_t work_bytes, void* stream) {
  GUARD({
    TRY(check_matmul(d));
    TRY(check_weight(weight));
    CHECK(weight->n == d->n && weight->k == d->k, CS_E_INVAL, "n and k must be the weight's");
    if (d->rows == 0) return CS_OK;
    TRY(check_tensor(a, "a"));
    TRY(check_tensor(a_scales, "a_scales"));
    TRY(check_optional(bias, "bias"));
    TRY(check_tensor(out, "out"));
    TRY(check_work(work, work_bytes, matmul_i8_workspace(*d)));
    MatmulI8Args m = {a, a_scales, bias, *weight, out, *d};
    if (d->rows == 1) m.d.a_row = round_up(d->k, 16), m.d.o_row = round_up(d->n, 8);   // never checked
    return launched(matmul_i8(m, work, (hipStream_t)stream), "rows and outputs");
  })
}

}  // extern "C"
