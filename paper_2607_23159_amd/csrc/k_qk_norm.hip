// RMS norm of q and k per head with the position rotation in the same pass.
#include "ops.hpp"

namespace cs {

typedef float f32x8 __attribute__((ext_vector_type(8), aligned(16)));   // rows are 16-byte aligned

// 8 channels as they come from memory.  q and k are read once and written once: both
// are marked as streaming.
template <typename T> struct Chunk8 {
  typedef T V __attribute__((ext_vector_type(8), aligned(16)));
  V v;
  CS_DEV void load(const T* p) { v = __builtin_nontemporal_load(reinterpret_cast<const V*>(p)); }
  CS_DEV f32x8 get() const { return __builtin_convertvector(v, f32x8); }
  static CS_DEV void store(T* p, const float* f) {
    V o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = to_t<T>(f[i]);
    __builtin_nontemporal_store(o, reinterpret_cast<V*>(p));
  }
};

// A lane owns 16 channels of a head, in two chunks of 8: both members of its
// pairs, whatever the style, and neighbouring lanes' first chunks (and second ones)
// lie next to each other, so that an access covers whole lines.  Halves: a chunk of
// each half of the rotated channels, or of the others; adjacent pairs: a chunk of
// each half of the head.  GL lanes (the power of two that holds
// head_dim / 16) make a head, so a wave takes 64 / GL heads of a token at a time
// ("pass"), and the same heads of TT tokens: their gains are read once.
//
// Bound by moving q and k once each way.  Per lane and token 64 bytes of them meet 64
// bytes of table and 64 / TT of gains, which come from L1 and L2.
template <typename T, int GL, int TT, bool HALVES>
__global__ __launch_bounds__(256) void k_qk_norm(QkNormArgs a, FastDiv by_passes, int items) {
  const cs_qk_norm_desc& d = a.d;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int item = blockIdx.x * 4 + wave;
  if (item >= items) return;
  const int block = by_passes.div(item), pass = item - block * (int)by_passes.d;
  const int t0 = block * TT;
  const int head = pass * (64 / GL) + lane / GL, li = lane % GL;
  const bool live = head < d.heads_q + d.heads_k && 16 * li < d.head_dim;
  const bool is_q = head < d.heads_q;
  const int h = is_q ? head : head - d.heads_q;
  int c0 = 8 * li, c1 = c0 + d.head_dim / 2;
  if (HALVES) {
    const bool in_rot = 16 * li < d.rot_dim;
    c0 = in_rot ? 8 * li : d.rot_dim + 8 * (li - d.rot_dim / 16);
    c1 = c0 + (in_rot ? d.rot_dim : d.head_dim - d.rot_dim) / 2;
  }
  const bool turns0 = c0 < d.rot_dim, turns1 = c1 < d.rot_dim;   // alike with halves
  // the chunks' entries of a row of the table
  const int e0 = HALVES ? 2 * c0 : c0, e1 = HALVES ? 2 * c0 + 8 : c1;
  const T* src = is_q ? (const T*)a.q + h * d.q_head : (const T*)a.k + h * d.k_head;
  T* dst = is_q ? (T*)a.qo + h * d.qo_head : (T*)a.ko + h * d.ko_head;
  const long in_row = is_q ? d.q_row : d.k_row, out_row = is_q ? d.qo_row : d.ko_row;

  // the row of the table of each token; negative: the token is skipped
  int row[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const int tok = t0 + t;
    row[t] = tok >= d.tokens ? -1 : a.pos ? a.pos[tok] : (d.rope_rows > 0 ? (int)((uint32_t)tok % (uint32_t)d.rope_rows) : 0);
  }
  Chunk8<T> u[TT], v[TT];
  if (live) {
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const T* x = src + min(t0 + t, d.tokens - 1) * in_row;
      u[t].load(x + c0);
      v[t].load(x + c1);
    }
  }
  f32x8 g0 = {}, g1 = {};
  if (live) {
    const float* gain = is_q ? a.q_gain + h * d.q_gain_head : a.k_gain + h * d.k_gain_head;
    g0 = *reinterpret_cast<const f32x8*>(gain + c0);
    g1 = *reinterpret_cast<const f32x8*>(gain + c1);
  }
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    if (row[t] < 0) continue;
    const bool in = row[t] < d.rope_rows;
    f32x8 e[2] = {};   // cos, sin of four pairs each
    const float* tab = a.rope + (long)(in ? row[t] : 0) * d.rot_dim;
    if (live && turns0) e[0] = *reinterpret_cast<const f32x8*>(tab + e0);
    if (live && turns1) e[1] = *reinterpret_cast<const f32x8*>(tab + e1);
    float x[16] = {};   // first chunk, second chunk
    if (live) {
      const f32x8 x0 = u[t].get(), x1 = v[t].get();
#pragma unroll
      for (int i = 0; i < 8; ++i) { x[i] = x0[i]; x[8 + i] = x1[i]; }
    }
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s = fmaf(x[i], x[i], s);
#pragma unroll
    for (int o = GL / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, WAVE);
    if (!live) continue;
    const float r = 1.0f / sqrtf(s / (float)d.head_dim + d.eps);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = x[i] * r * (i < 8 ? g0[i & 7] : g1[i & 7]);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      if (!(p < 4 ? turns0 : turns1)) continue;
      const int i = HALVES ? p : 2 * p, j = HALVES ? p + 8 : 2 * p + 1;
      const float c = e[p / 4][2 * (p % 4)], sn = e[p / 4][2 * (p % 4) + 1];
      const float f = x[i], w = x[j];
      x[i] = f * c - w * sn;
      x[j] = f * sn + w * c;
    }
    if (d.rot_dim > 0 && !in) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = NAN;
    }
    T* o = dst + (t0 + t) * out_row;
    Chunk8<T>::store(o + c0, x);
    Chunk8<T>::store(o + c1, x + 8);
  }
}

template <typename T, int GL, int TT> static hipError_t launch(const QkNormArgs& a, hipStream_t st) {
  const long passes = cdiv((long)a.d.heads_q + a.d.heads_k, 64 / GL), items = cdiv(a.d.tokens, TT) * passes;
  const long blocks = (items + 3) / 4;
  if (blocks > 0xFFFFFFL) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks), block(256);
  if (a.d.rope_style == CS_ROPE_HALVES)
    hipLaunchKernelGGL((k_qk_norm<T, GL, TT, true>), grid, block, 0, st, a, FastDiv(passes), (int)items);
  else
    hipLaunchKernelGGL((k_qk_norm<T, GL, TT, false>), grid, block, 0, st, a, FastDiv(passes), (int)items);
  return hipGetLastError();
}

// Two tokens a wave once that still leaves every SIMD eight waves; one before, where
// latency counts.  32,760 tokens of 40 + 40 heads of 128, bf16 (1.36 GB): 232 us, 5.9
// TB/s; four tokens 235, eight 248; without the streaming marks 255; 16 neighbouring
// channels a lane, so that an access takes every other half line, 288; one head group
// of one token a wave so 329.
template <typename T, int GL> static hipError_t launch_gl(const QkNormArgs& a, hipStream_t st) {
  const long passes = cdiv((long)a.d.heads_q + a.d.heads_k, 64 / GL);
  return a.d.tokens * passes >= 2 * 8192 ? launch<T, GL, 2>(a, st) : launch<T, GL, 1>(a, st);
}

template <typename T> hipError_t qk_norm_rope(const QkNormArgs& a, hipStream_t st) {
  const int lanes = a.d.head_dim / 16;
  if (lanes <= 2) return launch_gl<T, 2>(a, st);
  if (lanes <= 4) return launch_gl<T, 4>(a, st);
  if (lanes <= 8) return launch_gl<T, 8>(a, st);
  return launch_gl<T, 16>(a, st);
}

template hipError_t qk_norm_rope<bf16>(const QkNormArgs&, hipStream_t);
template hipError_t qk_norm_rope<float>(const QkNormArgs&, hipStream_t);

}  // namespace cs
