// Attention of queries to contexts: choice of the kernel, workspace, join of the
// parts of long contexts.
#include "ops.hpp"

#include <algorithm>

namespace cs {

// A problem's keys are cut into parts by its own sizes, never by the batch, so that
// results do not depend on it.
static void cut(XAttnArgs& a, bool kv4) {
  a.group = a.d.heads_q / a.d.heads_kv;
  a.rows = a.d.lq * a.group;
  a.parts = 1;
  // Keys of a full context's part: half as many bytes again in 4 bits (16 contexts of up
  // to 32,768 rows: 512 keys 72.7 us, 1,024 66.6, 2,048 82.6; bf16, 8 of up to 8,192: 256
  // keys 35.3, 512 34.2, 1,024 35.8).
  const int keys = kv4 ? 1024 : 512, most = 128;
  if (a.rows <= 1024 && a.d.lk > keys) a.parts = std::min(most, cdiv(a.d.lk, keys));
  a.by_group = FastDiv(a.group);
  a.by_parts = FastDiv(a.parts);
  a.by_heads = FastDiv(a.d.heads_kv);
}

struct Work {
  size_t part_o = 0, part_ml = 0, k = 0, v = 0, bytes = 0;
};
static Work layout(const XAttnArgs& a, bool kv4) {
  Work w;
  auto take = [&](size_t n) {
    const size_t at = w.bytes;
    w.bytes += (size_t)round_up((long)n, 256);
    return at;
  };
  if (a.d.n_q == 0 || a.rows == 0) return w;
  if (a.parts > 1) {
    const size_t rows = (size_t)a.d.n_q * a.d.heads_kv * a.parts * a.rows;
    w.part_o = take(rows * a.d.head_dim * sizeof(float));
    w.part_ml = take(rows * sizeof(float2));
  }
  if (kv4 && a.rows > XATTN_FEW_ROWS) {
    const size_t n = (size_t)a.d.n_kv * a.d.lk * a.d.heads_kv * a.d.head_dim * (a.d.dtype == CS_BF16 ? 2 : 4);
    w.k = take(n);
    w.v = take(n);
  }
  return w;
}

size_t xattn_workspace(const cs_attn_desc& d, bool kv4) {
  XAttnArgs a = {};
  a.d = d;
  cut(a, kv4);
  return layout(a, kv4).bytes;
}

// One row: the parts' outputs, each weighted with 2^(m_p - m).  Sixteen waves
// take every sixteenth part, lanes the channels.
template <typename T, int DH> __global__ __launch_bounds__(1024) void k_xattn_join(XAttnArgs a) {
  constexpr int NW = 16, MAXP = 128;
  __shared__ float s_w[MAXP], s_o[NW][DH], s_red[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long pr = blockIdx.x / a.rows;              // problem
  const int r = (int)(blockIdx.x - pr * a.rows);
  const int set = (int)(pr / a.d.heads_kv), head = (int)(pr - (long)set * a.d.heads_kv);
  int len;
  xattn_context(a, set, &len);
  const int pk = xattn_part(a, len), n = len > 0 ? (len + pk - 1) / pk : 0;
  const long base = pr * a.parts * a.rows + r;
  constexpr int NC = (DH + 63) / 64;
  float o[MAXP / NW][NC];
#pragma unroll
  for (int i = 0; i < MAXP / NW; ++i) {
    const int p = wave + NW * i;
#pragma unroll
    for (int c = 0; c < NC; ++c)
      o[i][c] = p < n && lane + 64 * c < DH ? a.part_o[(base + (long)p * a.rows) * DH + lane + 64 * c] : 0.0f;
  }
  if (wave == 0) {
    float m[2], l[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = lane + 64 * i;
      const float2 ml = p < n ? a.part_ml[base + (long)p * a.rows] : make_float2(-INFINITY, 0.0f);
      m[i] = ml.x;
      l[i] = ml.y;
    }
    float mx = fmaxf(m[0], m[1]);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor(mx, s, WAVE));
    if (mx == -INFINITY) mx = 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float w = __builtin_amdgcn_exp2f(m[i] - mx);
      s_w[lane + 64 * i] = w;
      sum = fmaf(w, l[i], sum);
    }
    sum = wave_sum(sum);
    if (lane == 0) s_red[0] = sum;
  }
  __syncthreads();
  float acc[NC] = {};
#pragma unroll
  for (int i = 0; i < MAXP / NW; ++i)
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (wave + NW * i < n) acc[c] = fmaf(s_w[wave + NW * i], o[i][c], acc[c]);
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (lane + 64 * c < DH) s_o[wave][lane + 64 * c] = acc[c];
  __syncthreads();
  if (tid < DH) {
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += s_o[w][tid];
    const float l = s_red[0];
    T* dst = (T*)a.o + set * a.d.o_b + xattn_row(a, r, head, a.d.o_r, a.d.o_h);
    dst[tid] = to_t<T>(l != 0.0f ? v / l : 0.0f);
  }
}

template <typename T> static hipError_t join(const XAttnArgs& a, hipStream_t st) {
  const long blocks = (long)a.d.n_q * a.d.heads_kv * a.rows;
  if (blocks > 0x3FFFFFL) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)blocks), block(1024);
  switch (a.d.head_dim) {
    case 128: hipLaunchKernelGGL((k_xattn_join<T, 128>), grid, block, 0, st, a); break;
    case 64: hipLaunchKernelGGL((k_xattn_join<T, 64>), grid, block, 0, st, a); break;
    default: hipLaunchKernelGGL((k_xattn_join<T, 32>), grid, block, 0, st, a); break;
  }
  return hipGetLastError();
}

template <typename T> hipError_t xattn(XAttnArgs a, bool kv4, void* work, hipStream_t st) {
  cut(a, kv4);
  const Work w = layout(a, kv4);
  a.part_o = (float*)((char*)work + w.part_o);
  a.part_ml = (float2*)((char*)work + w.part_ml);
  if (a.parts > 1 && (long)a.d.n_q * a.d.heads_kv * a.rows > 0x3FFFFFL) return hipErrorInvalidConfiguration;
  hipError_t e;
  if (a.rows <= XATTN_FEW_ROWS && (kv4 || sizeof(T) == 2)) {
    e = xattn_rows<T>(a, kv4, st);
  } else {
    if (kv4) {
      // many queries meet every key: unpack the cache once
      Kv4RowsArgs l = {};
      l.c = a.c;
      const long hd = (long)a.d.heads_kv * a.d.head_dim;
      l.r = {a.d.dtype, a.d.n_kv * a.d.lk, hd, a.d.head_dim, hd, a.d.head_dim};
      l.ko = (char*)work + w.k;
      l.vo = (char*)work + w.v;
      e = kv4_load<T>(l, st);
      if (e != hipSuccess) return e;
      a.k = l.ko;
      a.v = l.vo;
      a.d.k_r = a.d.v_r = hd;
      a.d.k_h = a.d.v_h = a.d.head_dim;
      a.d.k_b = a.d.v_b = hd * a.d.lk;
    }
    if constexpr (sizeof(T) == 2)
      e = xattn_tile(a, st);
    else
      e = xattn_f32(a, st);
  }
  if (e == hipSuccess && a.parts > 1) e = join<T>(a, st);
  return e;
}
template hipError_t xattn<bf16>(XAttnArgs, bool, void*, hipStream_t);
template hipError_t xattn<float>(XAttnArgs, bool, void*, hipStream_t);

}  // namespace cs
