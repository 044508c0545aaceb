// Rows held in registers: the row kernels (k_layer_norm.hip, k_i8_rows.hip) read a row
// once, reduce it as often as they need and write it once.
//
// A row belongs to WPR waves (1 or 4 of a workgroup of 4, or 16 of 16); a lane holds NV
// chunks of U consecutive channels, chunk i of lane t (0 <= t < 64 WPR) at channel
// U (64 WPR i + t), so that a wave's access is one run of memory.  U is 8 for bf16 rows and 4
// for fp32 ones (16 bytes a lane).  Channels past the row's end read as zero and
// are not written; a row's last, partial chunk moves by elements.
#pragma once
#include "common.hpp"

namespace cs {

template <typename T, int U> struct Chunk { typedef T vec __attribute__((ext_vector_type(U))); };

template <typename T, int U>
CS_DEV typename Chunk<T, U>::vec load_chunk(const T* __restrict__ p, int left) {
  typename Chunk<T, U>::vec v = {};
  if (left >= U) {
    v = *reinterpret_cast<const typename Chunk<T, U>::vec*>(p);
  } else {
#pragma unroll
    for (int e = 0; e < U - 1; ++e)
      if (e < left) v[e] = p[e];
  }
  return v;
}

// y: U values, rounded to T.
template <typename T, int U> CS_DEV void store_chunk(T* __restrict__ p, int left, const float* y) {
  typename Chunk<T, U>::vec v;
#pragma unroll
  for (int e = 0; e < U; ++e) v[e] = to_t<T>(y[e]);
  if (left >= U) {
    *reinterpret_cast<typename Chunk<T, U>::vec*>(p) = v;
  } else {
#pragma unroll
    for (int e = 0; e < U - 1; ++e)
      if (e < left) p[e] = v[e];
  }
}

// The same of integer codes -127..127, given as floats.
template <int U> CS_DEV void store_codes(int8_t* __restrict__ p, int left, const float* y) {
  union { uint32_t w[U / 4]; int8_t b[U]; } v;
#pragma unroll
  for (int i = 0; i < U / 4; ++i) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int)y[4 * i + e] & 255u) << (8 * e);
    v.w[i] = w;
  }
  if (left >= U) {
    if constexpr (U == 8) *reinterpret_cast<uint2*>(p) = make_uint2(v.w[0], v.w[1]);
    else *reinterpret_cast<uint32_t*>(p) = v.w[0];
  } else {
#pragma unroll
    for (int e = 0; e < U - 1; ++e)
      if (e < left) p[e] = v.b[e];
  }
}

// Sums (maxima) of the WPR waves of a row; every lane gets them.  Waves add up in a fixed
// order.  Each use needs LDS of its own or a barrier between two.
template <int WPR> CS_DEV float row_sum(float v, float* lds, int wave) {
  v = wave_sum(v);
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < WPR; ++i) v += lds[i];
  }
  return v;
}

template <int WPR> CS_DEV uint32_t row_max(uint32_t v, uint32_t* lds, int wave) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, WAVE));
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WPR; ++i) v = max(v, lds[i]);
  }
  return v;
}

// ---- 8-bit rows: scale = largest magnitude / 127 in fp32, code = the integer nearest to
// x / scale, halfway ones to the even one.
struct I8Scale {
  float scale, unit, half, inv, up;   // unit = scale * up, up a power of two
  // amax: bits of the row's largest magnitude.  A row that is not finite gets scale NaN and
  // codes 0, so that it reads back as NaN; one whose scale underflows gets codes 0.
  CS_DEV explicit I8Scale(uint32_t amax) {
    const bool ok = amax < 0x7F800000u;
    scale = ok ? __uint_as_float(amax) / 127.0f : __uint_as_float(0x7FC00000u);
    // Scales near the smallest numbers are moved up, where their inverse is finite and no
    // difference below underflows.
    up = scale < 0x1p-90f ? 0x1p100f : 1.0f;
    unit = scale * up;
    half = 0.5f * unit;
    inv = ok && scale > 0.0f ? 1.0f / unit : 0.0f;
  }
  // x * inv is off by less than 2^-15, so its nearest integer c is the quotient's or next to
  // it, and is wrong only next to a halfway value.  x - c scale is exact (a difference of
  // multiples of one unit in the last place, below scale): it decides.
  CS_DEV float code(float x) const {
    if (inv == 0.0f) return 0.0f;
    x *= up;
    float c = rintf(x * inv);
    const float t = fmaf(-c, unit, x), a = fabsf(t);
    const bool odd = ((int)c & 1) != 0;
    if (a > half || (a == half && odd)) c += copysignf(1.0f, t);
    return fminf(fmaxf(c, -127.0f), 127.0f);
  }
};

CS_DEV uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

}  // namespace cs
