// Rows of keys and values into the 4-bit cache and back.
#include "ops.hpp"

namespace cs {

// Four lanes share a group of 32 channels, 8 channels (16 bytes of bf16, 4 bytes
// of codes) each; LH = head_dim / 8 lanes make a row of a head, and a wave takes
// 64 / LH consecutive rows of one head, whose codes are neighbours in the cache.
struct Kv4Place {
  long row, slot;   // row of the call, row of the cache
  int head, li, ctx, pos;
  bool live;
};

template <int LH> CS_DEV Kv4Place kv4_place(const Kv4RowsArgs& a, long item) {
  constexpr int RW = 64 / LH;
  Kv4Place p;
  const int lane = threadIdx.x & 63;
  const long blk = item / a.c.heads;
  p.head = (int)(item - blk * a.c.heads);
  p.row = blk * RW + lane / LH;
  p.li = lane % LH;
  p.live = p.row < a.r.n_rows;
  p.slot = p.live ? (a.slots ? (long)a.slots[p.row] : p.row) : -1;
  p.live = p.slot >= 0 && p.slot < (long)a.c.n_kv * a.c.cap;
  if (!p.live) p.slot = 0;
  p.ctx = (int)(p.slot / a.c.cap);
  p.pos = (int)(p.slot - (long)p.ctx * a.c.cap);
  return p;
}

template <typename T, int LH> __global__ __launch_bounds__(256) void k_kv4_store(Kv4RowsArgs a) {
  const bool is_v = blockIdx.y != 0;
  const Kv4Place p = kv4_place<LH>(a, (long)blockIdx.x * 4 + (threadIdx.x >> 6));
  if (p.head >= a.c.heads || !p.live) return;   // whole rows: the four lanes of a group go together
  const T* src = is_v ? (const T*)a.v + p.row * a.r.v_row + p.head * a.r.v_head
                      : (const T*)a.k + p.row * a.r.k_row + p.head * a.r.k_head;
  src += 8 * p.li;
  uint32_t amax = 0, codes = 0;
  const long at = ((long)p.ctx * a.c.heads + p.head) * a.c.cap + p.pos;
  uint8_t* dc = (is_v ? a.c.v_codes : a.c.k_codes) + at * (4 * LH) + 4 * p.li;
  uint8_t* ds = (is_v ? a.c.v_scales : a.c.k_scales) + at * (LH / 4) + p.li / 4;
  if constexpr (sizeof(T) == 2) {
    union { uint4 q; uint32_t u[4]; bf16x2 b[4]; } x;
    x.q = *reinterpret_cast<const uint4*>(src);
#pragma unroll
    for (int i = 0; i < 4; ++i) amax = max(amax, max(x.u[i] & 0x7FFF0000u, (x.u[i] & 0x7FFFu) << 16));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1, WAVE));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2, WAVE));
    const uint32_t sb = kv4_scale_byte(amax);
    const float s = kv4_scale(sb == 255 ? 127 : sb);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, x.b[0], s, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, x.b[1], s, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, x.b[2], s, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, x.b[3], s, 3);
    *reinterpret_cast<uint32_t*>(dc) = codes;
    if ((p.li & 3) == 0) *ds = (uint8_t)sb;
  } else {
    union { uint4 q[2]; uint32_t u[8]; float f[8]; } x;
    x.q[0] = reinterpret_cast<const uint4*>(src)[0];
    x.q[1] = reinterpret_cast<const uint4*>(src)[1];
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, x.u[i] & 0x7FFFFFFFu);
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1, WAVE));
    amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2, WAVE));
    const uint32_t sb = kv4_scale_byte(amax);
    const float s = kv4_scale(sb == 255 ? 127 : sb);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x.f[0], x.f[1], s, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x.f[2], x.f[3], s, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x.f[4], x.f[5], s, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x.f[6], x.f[7], s, 3);
    *reinterpret_cast<uint32_t*>(dc) = codes;
    if ((p.li & 3) == 0) *ds = (uint8_t)sb;
  }
}

template <typename T, int LH> __global__ __launch_bounds__(256) void k_kv4_load(Kv4RowsArgs a) {
  const bool is_v = blockIdx.y != 0;
  const Kv4Place p = kv4_place<LH>(a, (long)blockIdx.x * 4 + (threadIdx.x >> 6));
  if (p.head >= a.c.heads || !p.live) return;
  const long at = ((long)p.ctx * a.c.heads + p.head) * a.c.cap + p.pos;
  const uint32_t codes =
      *reinterpret_cast<const uint32_t*>((is_v ? a.c.v_codes : a.c.k_codes) + at * (4 * LH) + 4 * p.li);
  const float s = kv4_scale((is_v ? a.c.v_scales : a.c.k_scales)[at * (LH / 4) + p.li / 4]);
  T* dst = is_v ? (T*)a.vo + p.row * a.r.v_row + p.head * a.r.v_head : (T*)a.ko + p.row * a.r.k_row + p.head * a.r.k_head;
  dst += 8 * p.li;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<bf16x8*>(dst) = kv4_decode8(codes, s);
  } else {
    const f32x2 u0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0);
    const f32x2 u1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
    const f32x2 u2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2);
    const f32x2 u3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
    reinterpret_cast<f32x4*>(dst)[0] = f32x4{u0[0], u0[1], u1[0], u1[1]};
    reinterpret_cast<f32x4*>(dst)[1] = f32x4{u2[0], u2[1], u3[0], u3[1]};
  }
}

template <typename T, int LH, bool STORE> static hipError_t launch(const Kv4RowsArgs& a, hipStream_t st) {
  const long items = (long)cdiv(a.r.n_rows, 64 / LH) * a.c.heads, blocks = (items + 3) / 4;
  if (blocks > 0xFFFFFFL) return hipErrorInvalidConfiguration;
  if constexpr (STORE)
    hipLaunchKernelGGL((k_kv4_store<T, LH>), dim3((unsigned)blocks, 2), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_kv4_load<T, LH>), dim3((unsigned)blocks, 2), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename T, bool STORE> static hipError_t rows(const Kv4RowsArgs& a, hipStream_t st) {
  switch (a.c.head_dim) {
    case 128: return launch<T, 16, STORE>(a, st);
    case 64: return launch<T, 8, STORE>(a, st);
    case 32: return launch<T, 4, STORE>(a, st);
    default: return hipErrorInvalidValue;
  }
}

template <typename T> hipError_t kv4_store(const Kv4RowsArgs& a, hipStream_t st) { return rows<T, true>(a, st); }
template <typename T> hipError_t kv4_load(const Kv4RowsArgs& a, hipStream_t st) { return rows<T, false>(a, st); }
template hipError_t kv4_store<bf16>(const Kv4RowsArgs&, hipStream_t);
template hipError_t kv4_store<float>(const Kv4RowsArgs&, hipStream_t);
template hipError_t kv4_load<bf16>(const Kv4RowsArgs&, hipStream_t);
template hipError_t kv4_load<float>(const Kv4RowsArgs&, hipStream_t);

}  // namespace cs
