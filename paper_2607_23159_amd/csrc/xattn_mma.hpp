// Attention of queries to contexts: what the kernels on 16 x 16 x 32 bf16 products share.
#pragma once
#include "ops.hpp"

namespace cs {

CS_DEV f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Maximum / sum over lanes l, l ^ 16, l ^ 32, l ^ 48.
CS_DEV float max_groups16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_lane_pair32(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
CS_DEV float sum_groups16(float x) {
  x += __shfl_xor(x, 16, WAVE);
  return x + __shfl_xor(x, 32, WAVE);
}

// Eight elements as sums of NS bf16 terms, the largest first: three hold all 24 bits of
// an fp32 number (below bf16's largest, 3.39e38).
template <int NS> CS_DEV void split_bf16(const float* x, bf16x8* t) {
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float a = x[i], b = x[i + 1];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const bf16x2 y = {(bf16)a, (bf16)b};
      t[n][i] = y[0];
      t[n][i + 1] = y[1];
      const uint32_t u = __builtin_bit_cast(uint32_t, y);
      a -= __uint_as_float(u << 16);
      b -= __uint_as_float(u & 0xFFFF0000u);
    }
  }
}

typedef __attribute__((address_space(3))) bf16x8 lds_vec8;
// Keys or values of a tile in LDS: rows of DH bf16, whose 16-byte chunks are permuted by the
// row (chunk c of row r at c ^ swz(r)): 16 rows' writes of one chunk, and 8 rows'
// reads of two, meet every bank once.
template <int DH> struct LdsRows {
  static constexpr int NC = DH / 8, BYTES = 2 * DH, PER256 = DH == 128 ? 0 : DH == 64 ? 1 : 2;   // log2 rows in 256 bytes
  static CS_DEV int swz(int r) { return 2 * ((r >> PER256) & (NC / 2 - 1)) | ((r >> 3) & 1); }
  static CS_DEV void put(lds_char* rows, int r, int chunk, bf16x8 v) {
    *(lds_vec8*)(rows + r * BYTES + 16 * (chunk ^ swz(r))) = v;
  }
  static CS_DEV bf16x8 get(const lds_char* rows, int r, int chunk) {
    return *(const lds_vec8*)(rows + r * BYTES + 16 * (chunk ^ swz(r)));
  }
  // V^T operand of 16 channels ct over the 32 rows from `rows` on
  static CS_DEV bf16x8 operand(const lds_char* rows, int lane, int ct) {
    const int r = 4 * (lane >> 4) + ((lane & 15) >> 2);
    const lds_char* p = rows + r * BYTES + 16 * ((2 * ct + ((lane >> 1) & 1)) ^ swz(r)) + 8 * (lane & 1);
    const bf16x4 x = lds_read_tr(p), y = lds_read_tr(p + 16 * BYTES);   // row + 16 is permuted alike
    return bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  }
};

// Keys of a tile (bit i: key kv0 + i) that are left: below k1 and not masked.
template <int KEYS, bool MASK>
CS_DEV uint64_t tile_bits(const uint8_t* mask, int kv0, int k1, int lane) {
  if constexpr (MASK) {
    const int key = kv0 + lane;
    return __ballot(lane < KEYS && key < k1 && mask[min(key, k1 - 1)] != 0);
  } else {
    const int n = min(KEYS, k1 - kv0);
    return n == 64 ? ~0ull : (1ull << n) - 1;
  }
}

}  // namespace cs
