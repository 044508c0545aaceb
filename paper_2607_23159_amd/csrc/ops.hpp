// Launchers of the stand-alone operators (cs_qk_norm_rope, cs_cross_attention,
// cs_kv4_*).  Arguments are validated by ops.hip before any launch.
#pragma once
#include "../../include/cs.h"
#include "common.hpp"

namespace cs {

// Division by d of numbers below 2^31: with 2^s >= d, the quotient is (umulhi(n, m) +
// n) >> s for m = ceil(2^32 (2^s - d) / d), rounded up past exact values.
struct FastDiv {
  uint32_t d, m, s;
  FastDiv() = default;
  explicit FastDiv(uint32_t d_) : d(d_), m(0), s(0) {
    while ((1ull << s) < d) ++s;
    m = (uint32_t)((((1ull << s) - d) << 32) / d + 1);
  }
  CS_DEV int div(int n) const { return (int)((__umulhi((uint32_t)n, m) + (uint32_t)n) >> s); }
};

// ---- per-head norms with rotation (k_qk_norm.hip)
struct QkNormArgs {
  const void *q, *k;
  void *qo, *ko;
  const float *q_gain, *k_gain, *rope;
  const int* pos;
  cs_qk_norm_desc d;
};
template <typename T> hipError_t qk_norm_rope(const QkNormArgs& a, hipStream_t st);

// A launch counts its work items in 32 bits.
inline hipError_t check_grid(long blocks, int threads) {
  return blocks * threads < (1L << 32) ? hipSuccess : hipErrorInvalidConfiguration;
}

// ---- layer norm (k_layer_norm.hip)
constexpr int LN_MAX_DIM = 16384;
struct LayerNormArgs {
  const void* x;
  const float *weight, *bias;    // NULL: 1 and 0
  void* y;
  float *y_scale, *mean, *rstd;  // y_scale: CS_I8 only; mean, rstd may be NULL
  cs_layer_norm_desc d;
};
hipError_t layer_norm(const LayerNormArgs& a, hipStream_t st);

struct LayerNormGradArgs {
  const void *x, *dy;
  const float *weight, *mean, *rstd;
  void* dx;                      // may be NULL
  float *dweight, *dbias;        // may be NULL
  float* part;                   // layer_norm_backward_workspace bytes
  cs_layer_norm_grad_desc d;
};
size_t layer_norm_backward_workspace(const cs_layer_norm_grad_desc& d);
hipError_t layer_norm_backward(const LayerNormGradArgs& a, hipStream_t st);

// ---- 8-bit rows and weights (k_i8_rows.hip)
constexpr int I8_MAX_DIM = 65536;
struct I8RowsArgs {
  const void* x;                 // quantised rows
  void* x_out;                   // read-back rows
  int8_t* codes;
  float* scales;
  cs_i8_rows d;
};
hipError_t i8_quantise(const I8RowsArgs& a, hipStream_t st);
hipError_t i8_dequantise(const I8RowsArgs& a, hipStream_t st);
long i8_weight_bytes(int n, int k);
// dtype of w: bf16, fp32, or CS_I8 with its scales given.
hipError_t i8_weight_pack(const cs_i8_weight& o, int dtype, const void* w, long w_row, const float* given,
                          hipStream_t st);

// ---- product of 8-bit rows and weights (k_matmul_i8.hip)
struct MatmulI8Args {
  const int8_t* a;
  const float *a_scale, *bias;   // bias may be NULL
  cs_i8_weight w;
  void* out;
  cs_matmul_i8_desc d;
};
size_t matmul_i8_workspace(const cs_matmul_i8_desc& d);
hipError_t matmul_i8(const MatmulI8Args& a, void* work, hipStream_t st);

// ---- rows of the 4-bit cache (k_kv4.hip)
struct Kv4RowsArgs {
  cs_kv4_cache c;
  cs_kv4_rows r;
  const void *k, *v;     // stored rows
  void *ko, *vo;         // loaded rows
  const int* slots;
  // kv4_unpack only
  const int* len;        // rows of each context, or NULL: further ones are skipped
  const int* ctx_of;     // the context that context i of the rows stands for, or NULL: i
};
template <typename T> hipError_t kv4_store(const Kv4RowsArgs& a, hipStream_t st);
template <typename T> hipError_t kv4_load(const Kv4RowsArgs& a, hipStream_t st);
hipError_t kv4_unpack(const Kv4RowsArgs& a, hipStream_t st);   // to bf16, slots not read

// ---- attention to contexts (k_xattn*.hip)
// The queries of a set that share a key head are the rows of one problem: row r is
// query r / group, head (key head) * group + r % group.
struct XAttnArgs {
  const void *q, *k, *v;
  void* o;
  const int *kv_of, *kv_len;
  bool by_set;           // k and v hold a context for each set (kv_len and mask do not)
  const uint8_t* mask;
  cs_kv4_cache c;        // 4-bit keys and values (k, v not read)
  cs_attn_desc d;
  float scale_log2;      // log2(e) * scale
  int rows, group;       // lq * group, heads_q / heads_kv
  FastDiv by_group, by_parts, by_heads;   // group, parts, heads_kv
  // Long contexts: a context's keys are cut into at most `parts` parts of xattn_part
  // keys.  A part leaves its outputs relative to its maximum m and its sums l: part_o
  // [problem][part][rows][head_dim], part_ml [problem][part][rows] (m, l).
  int parts;
  float* part_o;
  float2* part_ml;
};
size_t xattn_workspace(const cs_attn_desc& d, bool kv4);
// work: xattn_workspace bytes.
template <typename T> hipError_t xattn(XAttnArgs a, bool kv4, void* work, hipStream_t st);

// The kernels' launchers: few rows (k_xattn_rows.hip), many rows in bf16
// (k_xattn_tile.hip), fp32 in few and in many workgroups (k_xattn_f32.hip,
// k_xattn_split.hip).
template <typename T> hipError_t xattn_rows(const XAttnArgs& a, bool kv4, hipStream_t st);
hipError_t xattn_tile(const XAttnArgs& a, hipStream_t st);
hipError_t xattn_f32(const XAttnArgs& a, hipStream_t st);
hipError_t xattn_split(const XAttnArgs& a, hipStream_t st);

// Keys of the context of query set i, and the context's index (0 keys if kv_of is out
// of range).  i is wave-uniform; the index tensors are only read by these kernels, so
// they are read through the scalar cache.
CS_DEV int xattn_context(const XAttnArgs& a, int i, int* len) {
  typedef const __attribute__((address_space(4))) int const_int;
  const int j = a.kv_of ? ((const_int*)a.kv_of)[i] : i;
  if (j < 0 || j >= a.d.n_kv) {
    *len = 0;
    return 0;
  }
  *len = a.kv_len ? max(0, min(((const_int*)a.kv_len)[j], a.d.lk)) : a.d.lk;
  return j;
}

// Keys of a part of a context of len keys: whole tiles, a workgroup's worth at least.
CS_DEV int xattn_part(const XAttnArgs& a, int len) {
  if (a.parts == 1) return len;
  return max(128, (a.by_parts.div(len + a.parts - 1) + 63) & ~63);
}

// LDS by its own address (a generic pointer's conversion checks for null).
typedef __attribute__((address_space(3))) char lds_char;

// The direct load of buffer_load_lds16 as an instruction the compiler does not
// count.  It makes every transposing LDS read wait for all direct loads that it
// knows of, the next tiles' among them; here the kernels' own waits say which tile
// has to be there.  (No register is written, and the operands are read at issue.)
// base and bytes are wave-uniform.
CS_DEV void load_lds16(const void* base, int bytes, lds_char* lds, int voff) {
  const uint64_t b = (uint64_t)base;
  const i32x4 rsrc = {__builtin_amdgcn_readfirstlane((int)b), __builtin_amdgcn_readfirstlane((int)(b >> 32)) & 0xFFFF,
                      __builtin_amdgcn_readfirstlane(bytes), 0x00020000};
  const int at = __builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(voff), "s"(rsrc)
               : "memory", "m0");
}

// Transposing read: of the 4 rows of 16 values that 16 lanes address (8 bytes each,
// lane i row i / 4), lane i gets column i.
CS_DEV bf16x4 lds_read_tr(const lds_char* p) {
  typedef __attribute__((address_space(3))) bf16x4 lds_t;
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_t*)p);
}

// Offset of row r of problem (set, key head) in q or o (strides below 2^31).
CS_DEV long xattn_row(const XAttnArgs& a, int r, int head, long stride_r, long stride_h) {
  if (a.group == 1) return (long)r * (int)stride_r + (long)head * (int)stride_h;
  const int t = a.by_group.div(r);
  return (long)t * (int)stride_r + (long)(head * a.group + (r - t * a.group)) * (int)stride_h;
}

// ---- 4-bit values: e2m1 codes and their scale bytes.
typedef float f32x2 __attribute__((ext_vector_type(2)));
// Scale byte of a group whose largest magnitude has these fp32 bits: exponent of
// the power of two that puts it into [3.5, 7).  A quarter added to the mantissa
// carries into the exponent from 1.75 on.  255 for an infinity or a NaN.
CS_DEV uint32_t kv4_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return 255;
  return (uint32_t)max(1, (int)((amax_bits + 0x200000u) >> 23) - 2);
}
// Scale 2^(b - 127) of byte b; 255 gives infinity, which the conversions below turn into NaN.
CS_DEV float kv4_scale(uint32_t b) { return __uint_as_float(b << 23); }
// Eight codes of four bytes to bf16 (exact: a code has two significant bits).
CS_DEV bf16x8 kv4_decode8(uint32_t codes, float scale) {
  union { bf16x8 v; bf16x2 p[4]; } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return r.v;
}

}  // namespace cs
