// Entry points of the stand-alone operators: argument checks and launches.
#include <math.h>

#include <algorithm>

#include "host.hpp"
#include "ops.hpp"

using namespace cs;

static int elem(int dtype) { return dtype == CS_BF16 ? 2 : 4; }
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
  const size_t need = xattn_workspace(*d, kv4);
  if (need > 0) {
    CHECK(work && aligned(work), CS_E_INVAL, "a 16-byte aligned workspace is needed");
    CHECK(work_bytes >= need, CS_E_INVAL, "the workspace holds %zu bytes, %zu needed", work_bytes, need);
  }
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

}  // extern "C"
