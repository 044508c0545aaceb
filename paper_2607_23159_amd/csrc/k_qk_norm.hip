// RMS norm of q and k per head with the position rotation in the same pass.
#include "ops.hpp"

namespace cs {

// 16 channels of a lane as two chunks of 8.
template <typename T> struct Chunk8;
template <> struct Chunk8<bf16> {
  bf16x8 v;
  CS_DEV void load(const bf16* p) { v = *reinterpret_cast<const bf16x8*>(p); }
  CS_DEV void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
  }
  static CS_DEV void store(bf16* p, const float* f) {
    bf16x8 o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = (bf16)f[i];
    *reinterpret_cast<bf16x8*>(p) = o;
  }
};
template <> struct Chunk8<float> {
  f32x4 a, b;
  CS_DEV void load(const float* p) {
    a = reinterpret_cast<const f32x4*>(p)[0];
    b = reinterpret_cast<const f32x4*>(p)[1];
  }
  CS_DEV void get(float* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[4 + i] = b[i]; }
  }
  static CS_DEV void store(float* p, const float* f) {
    reinterpret_cast<f32x4*>(p)[0] = f32x4{f[0], f[1], f[2], f[3]};
    reinterpret_cast<f32x4*>(p)[1] = f32x4{f[4], f[5], f[6], f[7]};
  }
};

// A lane owns 16 channels of a head, in two chunks of 8: both members of its
// pairs, whatever the style.  With adjacent pairs (and beyond rot_dim) they are 16
// consecutive channels, with halves 8 of each half; the table's entries for the
// 8 pairs are consecutive either way.  GL lanes (the power of two that holds
// head_dim / 16) make a head, so a wave takes 64 / GL heads of one token at a time.
template <typename T, int GL>
__global__ __launch_bounds__(256) void k_qk_norm(QkNormArgs a) {
  const cs_qk_norm_desc& d = a.d;
  const int lane = threadIdx.x & 63;
  const int hw = 64 / GL, heads = d.heads_q + d.heads_k, passes = (heads + hw - 1) / hw;
  const long item = (long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long tok = item / passes;
  if (tok >= d.tokens) return;
  const int head = (int)(item - tok * passes) * hw + lane / GL;
  const int li = lane % GL;
  const int row = a.pos ? a.pos[tok] : (d.rope_rows > 0 ? (int)(tok % d.rope_rows) : 0);
  if (row < 0) return;
  const bool live = head < heads && 16 * li < d.head_dim;
  const bool is_q = head < d.heads_q;
  const int h = is_q ? head : head - d.heads_q;
  const bool turns = 16 * li < d.rot_dim;
  const bool halves = turns && d.rope_style == CS_ROPE_HALVES;
  const int c0 = halves ? 8 * li : 16 * li, c1 = halves ? c0 + d.rot_dim / 2 : c0 + 8;

  float x[16], g[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.0f;
  if (live) {
    const T* src = is_q ? (const T*)a.q + tok * d.q_row + h * d.q_head : (const T*)a.k + tok * d.k_row + h * d.k_head;
    Chunk8<T> u, v;
    u.load(src + c0);
    v.load(src + c1);
    u.get(x);
    v.get(x + 8);
  }
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s = fmaf(x[i], x[i], s);
#pragma unroll
  for (int o = GL / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, WAVE);
  if (!live) return;
  const float r = 1.0f / sqrtf(s / (float)d.head_dim + d.eps);
  const float* gain = is_q ? a.q_gain + h * d.q_gain_head : a.k_gain + h * d.k_gain_head;
  Chunk8<float> t;
  t.load(gain + c0);
  t.get(g);
  t.load(gain + c1);
  t.get(g + 8);
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = x[i] * r * g[i];
  if (turns) {
    float e[16];
    const bool in = row < d.rope_rows;
    const float* tab = a.rope + (long)(in ? row : 0) * d.rot_dim + 16 * li;
    t.load(tab);
    t.get(e);
    t.load(tab + 8);
    t.get(e + 8);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const float c = in ? e[2 * p] : NAN, sn = in ? e[2 * p + 1] : NAN;
      const float f = halves ? x[p] : x[2 * p], w = halves ? x[8 + p] : x[2 * p + 1];
      const float y0 = f * c - w * sn, y1 = f * sn + w * c;
      if (halves) { x[p] = y0; x[8 + p] = y1; }
      else { x[2 * p] = y0; x[2 * p + 1] = y1; }
    }
  } else if (a.pos && d.rot_dim > 0 && row >= d.rope_rows) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = NAN;
  }
  T* dst = is_q ? (T*)a.qo + tok * d.qo_row + h * d.qo_head : (T*)a.ko + tok * d.ko_row + h * d.ko_head;
  Chunk8<T>::store(dst + c0, x);
  Chunk8<T>::store(dst + c1, x + 8);
}

template <typename T, int GL> static hipError_t launch(const QkNormArgs& a, hipStream_t st) {
  const int hw = 64 / GL, passes = (a.d.heads_q + a.d.heads_k + hw - 1) / hw;
  const long blocks = ((long)a.d.tokens * passes + 3) / 4;
  if (blocks > 0xFFFFFFL) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((k_qk_norm<T, GL>), dim3((unsigned)blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename T> hipError_t qk_norm_rope(const QkNormArgs& a, hipStream_t st) {
  const int lanes = a.d.head_dim / 16;
  if (lanes <= 2) return launch<T, 2>(a, st);
  if (lanes <= 4) return launch<T, 4>(a, st);
  if (lanes <= 8) return launch<T, 8>(a, st);
  return launch<T, 16>(a, st);
}

template hipError_t qk_norm_rope<bf16>(const QkNormArgs&, hipStream_t);
template hipError_t qk_norm_rope<float>(const QkNormArgs&, hipStream_t);

}  // namespace cs
