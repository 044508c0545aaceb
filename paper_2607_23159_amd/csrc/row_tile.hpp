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

// Shape of a kernel for rows of a length: waves of a row, chunks of a lane, and whether the
// length is not a multiple of U.
template <int WPR_, int NV_, bool TAIL_> struct RowShape {
  static constexpr int WPR = WPR_, NV = NV_;
  static constexpr bool TAIL = TAIL_;
};

// Calls f with the shape for rows of dim channels, up to 16,384: the least chunks that hold a row (a
// lane's idle chunks cost registers, and with them waves in flight).  A wave a row up to 2048
// channels, 4 beyond.
template <int U, class F> static hipError_t with_row_shape(int dim, F f) {
  constexpr int L = U == 4 ? 4 : 2;   // chunks per 16 channels of a lane
  if (dim % U != 0) {
    if (dim <= 512) return f(RowShape<1, L / 2, true>{});
    if (dim <= 2048) return f(RowShape<1, 2 * L, true>{});
    if (dim <= 8192) return f(RowShape<4, 2 * L, true>{});
    return f(RowShape<4, 4 * L, true>{});
  }
#define CS_SHAPE(WPR, N) \
  if (nv <= N) return f(RowShape<WPR, N, false>{});
  if (dim <= 2048) {
    const int nv = (dim / U + 63) / 64;
    CS_SHAPE(1, 1) CS_SHAPE(1, 2) CS_SHAPE(1, 3) CS_SHAPE(1, 4)
    if constexpr (U == 4) {
      CS_SHAPE(1, 6) CS_SHAPE(1, 8)
    }
  }
  const int nv = (dim / U + 255) / 256;
  if constexpr (U == 8) {
    CS_SHAPE(4, 2)
  }
  CS_SHAPE(4, 3) CS_SHAPE(4, 4) CS_SHAPE(4, 5) CS_SHAPE(4, 6) CS_SHAPE(4, 8)
  if constexpr (U == 4) {
    CS_SHAPE(4, 12) CS_SHAPE(4, 16)
  }
#undef CS_SHAPE
  return hipErrorInvalidValue;
}

// Calls of more than one and a half times the last cache (256 MB) pass it by, both ways: their rows
// are gone before they are wanted again.  (8 x 32,760 x 1536, norm from fp32 to bf16: 411 -> 390 us;
// 32,760 x 5120 from 8 bits 85 -> 72.  32,760 x 1536 in bf16, 200 MB, would go from 33 to 39.)
inline bool past_caches(double bytes) { return bytes > 384e6; }

template <typename T, int U, bool TAIL, bool NT = false>
CS_DEV typename Chunk<T, U>::vec load_chunk(const T* __restrict__ p, int left) {
  typename Chunk<T, U>::vec v = {};
  if (left >= U) {
    const auto* q = reinterpret_cast<const typename Chunk<T, U>::vec*>(p);
    if constexpr (NT) v = __builtin_nontemporal_load(q);
    else v = *q;
  } else if constexpr (TAIL) {
#pragma unroll
    for (int e = 0; e < U - 1; ++e)
      if (e < left) v[e] = p[e];
  }
  return v;
}

// y: U values, rounded to T.
template <typename T, int U, bool TAIL, bool NT = false>
CS_DEV void store_chunk(T* __restrict__ p, int left, const float* y) {
  typename Chunk<T, U>::vec v;
#pragma unroll
  for (int e = 0; e < U; ++e) v[e] = to_t<T>(y[e]);
  if (left >= U) {
    if (NT) __builtin_nontemporal_store(v, reinterpret_cast<typename Chunk<T, U>::vec*>(p));
    else *reinterpret_cast<typename Chunk<T, U>::vec*>(p) = v;
  } else if constexpr (TAIL) {
#pragma unroll
    for (int e = 0; e < U - 1; ++e)
      if (e < left) p[e] = v[e];
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

// Two sums at once.
template <int WPR> CS_DEV float2 row_sums(float a, float b, float2* lds, int wave) {
  float2 v = make_float2(wave_sum(a), wave_sum(b));
  if constexpr (WPR > 1) {
    if ((threadIdx.x & 63) == 0) lds[wave] = v;
    __syncthreads();
    v = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < WPR; ++i) {
      v.x += lds[i].x;
      v.y += lds[i].y;
    }
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
  CS_DEV bool plain() const { return inv != 0.0f && up == 1.0f; }
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

// The larger of m and the magnitudes' bits of a chunk: fp32, or two bf16 to a word.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
CS_DEV void max_bits(uint32_t& m, const f32x4& v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) m = max(m, abs_bits(v[e]));
}
CS_DEV void max_bits(u16x2& m, const bf16x8& v) {
  union { bf16x8 v; uint32_t w[4]; u16x2 h[4]; } u = {v};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    u.w[e] &= 0x7FFF7FFFu;
    m = __builtin_elementwise_max(m, u.h[e]);
  }
}
CS_DEV uint32_t fp32_bits(uint32_t m) { return m; }
CS_DEV uint32_t fp32_bits(u16x2 m) { return (uint32_t)max(m[0], m[1]) << 16; }

// Four low bytes to one word.
CS_DEV uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0C0C0400u), hi = __builtin_amdgcn_perm(d, c, 0x0C0C0400u);
  return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// Codes of a lane's chunks of a row of dim values, value(i, e) element e of chunk i, stored to p
// (the row's codes).  The sum x inv + 1.5 2^23 has the nearest integer in its low bits, and what x -
// c scale leaves says whether it is the quotient's.  Values of 24 bits lie next to a halfway value once
// in a few hundred chunks: the largest remainder is kept, and where it reaches half a scale in
// a wave the codes are made again, one by one.  Values of 8 bits (COARSE) do in most rows (half the
// largest magnitude is one): there a step up or down follows from the remainder.  Exact halves are
// left for the second way: an odd number of half scales that has 8 significant bits is there only if
// the scale has no more.  With all of code()'s steps for every value the vector unit was
// the bound: 32,760 x 8960 in bf16 took 215 us.
template <int U, int NV, int WPR, bool TAIL, bool COARSE, class F>
CS_DEV void store_codes(const I8Scale& s, int8_t* __restrict__ p, int dim, int t, F value) {
  constexpr float MAGIC = 12582912.0f;
  uint32_t w[NV][U / 4];
  float worst = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    // a chunk after the other: widened all at once, bf16 values take twice the registers
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int h = 0; h < U / 4; ++h) {
      uint32_t b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = value(i, 4 * h + e), f = fmaf(x, s.inv, MAGIC);
        const float left = fmaf(MAGIC - f, s.unit, x);
        b[e] = __float_as_uint(f);
        if constexpr (COARSE) {
          b[e] += left > s.half ? 1u : 0u;
          b[e] -= left < -s.half ? 1u : 0u;
        } else {
          worst = fmaxf(worst, fabsf(left));
        }
      }
      w[i][h] = pack_bytes(b[0], b[1], b[2], b[3]);
    }
  }
  if (!s.plain() || (COARSE ? (__float_as_uint(s.scale) & 0xFFFFu) == 0 : __any(worst >= s.half))) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int h = 0; h < U / 4; ++h) {
        uint32_t b[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = (uint32_t)(int)s.code(value(i, 4 * h + e));
        w[i][h] = pack_bytes(b[0], b[1], b[2], b[3]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = U * (64 * WPR * i + t), left = dim - c;
    if (left >= U) {
      if constexpr (U == 8) *reinterpret_cast<uint2*>(p + c) = make_uint2(w[i][0], w[i][1]);
      else *reinterpret_cast<uint32_t*>(p + c) = w[i][0];
    } else if constexpr (TAIL) {
#pragma unroll
      for (int e = 0; e < U - 1; ++e)
        if (e < left) p[c + e] = (int8_t)(w[i][e / 4] >> (8 * (e % 4)));
    }
  }
}

}  // namespace cs
