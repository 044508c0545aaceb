// Rows of keys and values into the 4-bit cache and back.
#include "ops.hpp"

namespace cs {

// Four lanes share a group of 32 channels, 8 channels (16 bytes of bf16, 4 bytes of
// codes) each; LH = head_dim / 8 lanes make a row of a head.  A wave takes U times 64 /
// LH consecutive rows of one head: their codes are neighbours in the cache where their
// slots are.  All of a wave's rows are asked for before the first is waited for.
// Bound by moving the rows and their codes once: 478 MB, in 78 us into the cache (6.1
// TB/s) and 70 us back (6.8).
template <int LH, int U> struct Kv4Items {
  static constexpr int RW = 64 / LH;
  int head, li;
  int row[U];       // row of the call; negative: none, or its slot is not in the cache
  long at[U];       // row of the head in the cache

  // UNPACK: row i is row i % cap of context i / cap, or of ctx_of[i / cap], as far as that goes.
  template <bool UNPACK> CS_DEV bool set(const Kv4RowsArgs& a, FastDiv by_heads, FastDiv by_cap, int items) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = blockIdx.x * 4 + wave;
    if (item >= items) return false;
    const int block = by_heads.div(item);
    head = item - block * (int)by_heads.d;
    li = lane % LH;
    const long slots = (long)a.c.n_kv * a.c.cap;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      row[u] = (block * U + u) * RW + lane / LH;
      const int slot = row[u] >= a.r.n_rows ? -1 : !UNPACK && a.slots ? a.slots[row[u]] : row[u];
      if (slot < 0 || slot >= slots) row[u] = -1;
      int ctx = by_cap.div(row[u] < 0 ? 0 : slot);
      const int r = slot - ctx * a.c.cap;
      if constexpr (UNPACK) {
        if (a.ctx_of) ctx = a.ctx_of[ctx];
        if (ctx < 0 || ctx >= a.c.n_kv) {
          row[u] = -1;
          ctx = 0;
        }
        if (a.len && r >= a.len[ctx]) row[u] = -1;
      }
      at[u] = ((long)ctx * a.c.heads + head) * a.c.cap + r;
    }
    return true;
  }
};

template <typename T> struct Row8 {
  typedef T V __attribute__((ext_vector_type(8), aligned(16)));
};

// Codes and scale byte of a lane's 8 channels (the byte is the group's, alike in its lanes).
CS_DEV uint32_t kv4_encode(Row8<bf16>::V x, uint32_t* byte) {
  union { Row8<bf16>::V v; uint32_t u[4]; bf16x2 b[4]; } r;
  r.v = x;
  uint32_t amax = 0, codes = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) amax = max(amax, max(r.u[i] & 0x7FFF0000u, (r.u[i] & 0x7FFFu) << 16));
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1, WAVE));
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2, WAVE));
  *byte = kv4_scale_byte(amax);
  const float s = kv4_scale(*byte == 255 ? 127 : *byte);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, r.b[0], s, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, r.b[1], s, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, r.b[2], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, r.b[3], s, 3);
}
CS_DEV uint32_t kv4_encode(Row8<float>::V x, uint32_t* byte) {
  uint32_t amax = 0, codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 1, WAVE));
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 2, WAVE));
  *byte = kv4_scale_byte(amax);
  const float s = kv4_scale(*byte == 255 ? 127 : *byte);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], s, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], s, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], s, 3);
}

template <typename T, int LH, int U>
__global__ __launch_bounds__(256) void k_kv4_store(Kv4RowsArgs a, FastDiv by_heads, FastDiv by_cap, int items) {
  typedef typename Row8<T>::V V;
  const bool is_v = blockIdx.y != 0;
  Kv4Items<LH, U> it;
  if (!it.template set<false>(a, by_heads, by_cap, items)) return;
  const T* src = (is_v ? (const T*)a.v + it.head * a.r.v_head : (const T*)a.k + it.head * a.r.k_head) + 8 * it.li;
  const long stride = is_v ? a.r.v_row : a.r.k_row;
  uint8_t *codes = is_v ? a.c.v_codes : a.c.k_codes, *scales = is_v ? a.c.v_scales : a.c.k_scales;
  V x[U] = {};
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (it.row[u] >= 0) x[u] = __builtin_nontemporal_load(reinterpret_cast<const V*>(src + it.row[u] * stride));
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t byte;
    const uint32_t c = kv4_encode(x[u], &byte);
    if (it.row[u] < 0) continue;   // whole rows: the four lanes of a group go together
    *reinterpret_cast<uint32_t*>(codes + it.at[u] * (4 * LH) + 4 * it.li) = c;
    if ((it.li & 3) == 0) scales[it.at[u] * (LH / 4) + it.li / 4] = (uint8_t)byte;
  }
}

// Loaded rows are not read again soon and are written as streaming; unpacked ones are read
// next.  (With the choice made in the kernel, a load of 61,440 rows took 105 us instead of 70.)
template <typename T, int LH, int U, bool UNPACK>
__global__ __launch_bounds__(256) void k_kv4_load(Kv4RowsArgs a, FastDiv by_heads, FastDiv by_cap, int items) {
  typedef typename Row8<T>::V V;
  const bool is_v = blockIdx.y != 0;
  Kv4Items<LH, U> it;
  if (!it.template set<UNPACK>(a, by_heads, by_cap, items)) return;
  T* dst = (is_v ? (T*)a.vo + it.head * a.r.v_head : (T*)a.ko + it.head * a.r.k_head) + 8 * it.li;
  const long stride = is_v ? a.r.v_row : a.r.k_row;
  const uint8_t *codes = is_v ? a.c.v_codes : a.c.k_codes, *scales = is_v ? a.c.v_scales : a.c.k_scales;
  uint32_t c[U] = {}, b[U] = {};
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (it.row[u] >= 0) {
      c[u] = *reinterpret_cast<const uint32_t*>(codes + it.at[u] * (4 * LH) + 4 * it.li);
      b[u] = scales[it.at[u] * (LH / 4) + it.li / 4];
    }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (it.row[u] < 0) continue;
    const float s = kv4_scale(b[u]);
    V y;
    if constexpr (sizeof(T) == 2) {
      y = kv4_decode8(c[u], s);
    } else {
      const f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], s, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[u], s, 3)};
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = p[i / 2][i % 2];
    }
    V* to = reinterpret_cast<V*>(dst + it.row[u] * stride);
    if constexpr (UNPACK) *to = y;
    else __builtin_nontemporal_store(y, to);
  }
}

enum Kv4Move { STORE, LOAD, UNPACK };

template <typename T, int LH, int U, Kv4Move MOVE> static hipError_t launch(const Kv4RowsArgs& a, hipStream_t st) {
  const long items = (long)cdiv(a.r.n_rows, U * (64 / LH)) * a.c.heads, blocks = (items + 3) / 4;
  if (blocks > 0xFFFFFFL) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks, 2), block(256);
  const FastDiv by_heads(a.c.heads), by_cap(a.c.cap);
  if constexpr (MOVE == STORE)
    hipLaunchKernelGGL((k_kv4_store<T, LH, U>), grid, block, 0, st, a, by_heads, by_cap, (int)items);
  else
    hipLaunchKernelGGL((k_kv4_load<T, LH, U, MOVE == UNPACK>), grid, block, 0, st, a, by_heads, by_cap, (int)items);
  return hipGetLastError();
}

// Four steps a wave once that leaves every SIMD a few waves; one before, where latency
// counts (12 heads of 128, store and load, four / one: 2,048 rows 6.3 and 6.3 / 6.4 and 6.3
// us, 8,192 rows 15.5 and 11.8 / 19.0 and 12.6, 61,440 rows 78 and 70 / 119 and 76).
template <typename T, int LH, Kv4Move MOVE> static hipError_t launch_u(const Kv4RowsArgs& a, hipStream_t st) {
  return (long)cdiv(a.r.n_rows, 64 / LH) * a.c.heads >= 4 * 4096 ? launch<T, LH, 4, MOVE>(a, st)
                                                                : launch<T, LH, 1, MOVE>(a, st);
}

template <typename T, Kv4Move MOVE> static hipError_t rows(const Kv4RowsArgs& a, hipStream_t st) {
  switch (a.c.head_dim) {
    case 128: return launch_u<T, 16, MOVE>(a, st);
    case 64: return launch_u<T, 8, MOVE>(a, st);
    case 32: return launch_u<T, 4, MOVE>(a, st);
    default: return hipErrorInvalidValue;
  }
}

template <typename T> hipError_t kv4_store(const Kv4RowsArgs& a, hipStream_t st) { return rows<T, STORE>(a, st); }
template <typename T> hipError_t kv4_load(const Kv4RowsArgs& a, hipStream_t st) { return rows<T, LOAD>(a, st); }
hipError_t kv4_unpack(const Kv4RowsArgs& a, hipStream_t st) { return rows<bf16, UNPACK>(a, st); }
template hipError_t kv4_store<bf16>(const Kv4RowsArgs&, hipStream_t);
template hipError_t kv4_store<float>(const Kv4RowsArgs&, hipStream_t);
template hipError_t kv4_load<bf16>(const Kv4RowsArgs&, hipStream_t);
template hipError_t kv4_load<float>(const Kv4RowsArgs&, hipStream_t);

}  // namespace cs
