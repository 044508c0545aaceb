// Attention of queries to contexts of their own lengths, over keys and values in
// the compute type or in 4 bits.
#include "ops.hpp"

namespace cs {

// Channel values of key rows, per storage.
template <typename T> struct KvPlain {
  const T *k, *v;
  long k_r, v_r;
  CS_DEV KvPlain(const XAttnArgs& a, int ctx, int head)
      : k((const T*)a.k + ctx * a.d.k_b + head * a.d.k_h), v((const T*)a.v + ctx * a.d.v_b + head * a.d.v_h),
        k_r(a.d.k_r), v_r(a.d.v_r) {}
  CS_DEV void key8(int key, int c, float* f) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)k[key * k_r + c + i];
  }
  CS_DEV float value(int key, int c) const { return (float)v[key * v_r + c]; }
};

template <int DH> struct Kv4Rows {
  const uint8_t *kc, *ks, *vc, *vs;
  CS_DEV Kv4Rows(const XAttnArgs& a, int ctx, int head) {
    const long at = ((long)ctx * a.c.heads + head) * a.c.cap;
    kc = a.c.k_codes + at * (DH / 2);
    vc = a.c.v_codes + at * (DH / 2);
    ks = a.c.k_scales + at * (DH / 32);
    vs = a.c.v_scales + at * (DH / 32);
  }
  CS_DEV void key8(int key, int c, float* f) const {
    const uint32_t codes = *reinterpret_cast<const uint32_t*>(kc + (long)key * (DH / 2) + c / 2);
    const bf16x8 v = kv4_decode8(codes, kv4_scale(ks[(long)key * (DH / 32) + c / 32]));
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
  }
  CS_DEV float value(int key, int c) const {
    const uint32_t code = vc[(long)key * (DH / 2) + c / 2] >> (4 * (c & 1));
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, kv4_scale(vs[(long)key * (DH / 32) + c / 32]), 0)[0];
  }
};

CS_DEV float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, WAVE));
  return v;
}

// One wave per query and head: 64 keys at a time, a lane per key for the scores
// (online softmax across the wave), a lane per channel for the values.
template <typename T, int DH, typename KV>
__global__ __launch_bounds__(256) void k_xattn_wave(XAttnArgs a) {
  __shared__ float s_q[4][DH];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long item = (long)blockIdx.x * 4 + wave, n = (long)a.d.n_q * a.d.lq * a.d.heads_q;
  const long it = item < n ? item : n - 1;
  const int head = (int)(it % a.d.heads_q);
  const long row = it / a.d.heads_q;
  const int set = (int)(row / a.d.lq), qi = (int)(row - (long)set * a.d.lq);
  int len;
  const int ctx = xattn_context(a, set, &len);
  const KV kv(a, ctx, head / (a.d.heads_q / a.d.heads_kv));
  const uint8_t* mask = a.mask ? a.mask + ctx * a.d.mask_b : nullptr;
  const T* q = (const T*)a.q + set * a.d.q_b + qi * a.d.q_r + head * a.d.q_h;
  for (int c = lane; c < DH; c += 64) s_q[wave][c] = (float)q[c];
  __syncthreads();

  constexpr int NC = (DH + 63) / 64;
  float m = -INFINITY, l = 0.0f, o[NC] = {};
  for (int base = 0; base < len; base += 64) {
    const int key = base + lane;
    const bool left = key < len && (!mask || mask[key] != 0);
    float s = -INFINITY;
    if (left) {
      s = 0.0f;
      for (int c = 0; c < DH; c += 8) {
        float f[8];
        kv.key8(key, c, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(s_q[wave][c + i], f[i], s);
      }
      s *= a.scale_log2;
    }
    const float m_new = fmaxf(m, wave_max(s));
    if (m_new == -INFINITY) continue;
    const float alpha = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    const float p = left ? (float)to_t<T>(__builtin_amdgcn_exp2f(s - m)) : 0.0f;
    l = l * alpha + wave_sum(p);
#pragma unroll
    for (int i = 0; i < NC; ++i) o[i] *= alpha;
    for (int j = 0; j < 64 && base + j < len; ++j) {
      const float pj = __shfl(p, j, WAVE);
      if (pj == 0.0f) continue;
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (lane + 64 * i < DH) o[i] = fmaf(pj, kv.value(base + j, lane + 64 * i), o[i]);
    }
  }
  if (item >= n) return;
  T* dst = (T*)a.o + set * a.d.o_b + qi * a.d.o_r + head * a.d.o_h;
#pragma unroll
  for (int i = 0; i < NC; ++i)
    if (lane + 64 * i < DH) dst[lane + 64 * i] = to_t<T>(l > 0.0f ? o[i] / l : 0.0f);
}

size_t xattn_workspace(const cs_attn_desc&, bool) { return 0; }

template <typename T, int DH> static hipError_t launch(const XAttnArgs& a, bool kv4, hipStream_t st) {
  const long blocks = ((long)a.d.n_q * a.d.lq * a.d.heads_q + 3) / 4;
  if (blocks > 0xFFFFFFL) return hipErrorInvalidConfiguration;
  if (kv4)
    hipLaunchKernelGGL((k_xattn_wave<T, DH, Kv4Rows<DH>>), dim3((unsigned)blocks), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_xattn_wave<T, DH, KvPlain<T>>), dim3((unsigned)blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename T> hipError_t xattn(const XAttnArgs& a, bool kv4, hipStream_t st) {
  switch (a.d.head_dim) {
    case 128: return launch<T, 128>(a, kv4, st);
    case 64: return launch<T, 64>(a, kv4, st);
    case 32: return launch<T, 32>(a, kv4, st);
    default: return hipErrorInvalidValue;
  }
}
template hipError_t xattn<bf16>(const XAttnArgs&, bool, hipStream_t);
template hipError_t xattn<float>(const XAttnArgs&, bool, hipStream_t);

}  // namespace cs
