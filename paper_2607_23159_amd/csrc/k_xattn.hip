// Attention of queries to contexts: choice of the kernel, workspace, join of the
// parts of long contexts.
#include "ops.hpp"

#include <algorithm>

namespace cs {

// Whether a problem goes to k_xattn_rows, which takes its rows 32 at a time and reads
// the keys once for each 32.
//   bf16: if that is once (8 contexts of 8,192 rows, 8 key heads, here / in k_xattn_tile: 32
//     rows 54.1 / 53.5 us, 36 rows 66.2 / 54.8, 64 rows 75.8 / 60.7).
//   4 bits, bf16 rows: k_xattn_tile wants the cache unpacked first, which pays once the
//     rows are many (16 contexts of 32,768 rows, 8 key heads, here / there: 64 rows 320 /
//     1,024 us, 128 rows 608 / 1,136, 192 rows 917 / 1,244, 256 rows 1,216 / 1,345, 384 rows
//     1,823 / 1,773).  Contexts that many queries share would turn earlier.
//   4 bits, fp32 rows: always.  The queries' and weights' three bf16 terms meet exact
//     bf16 keys at 220 TFLOP/s, the fp32 products of k_xattn_f32 reach 85 (96 tokens of
//     4 heads each: 3.8 ms, 9.7 there).
static bool few_rows(const XAttnArgs& a, bool kv4) {
  if (a.d.dtype != CS_BF16) return kv4;
  return a.rows <= (kv4 ? 192 : 32);
}

// A problem's keys are cut into parts by its own sizes, never by the batch, so that
// results do not depend on it.
static void cut(XAttnArgs& a, bool kv4) {
  a.group = a.d.heads_q / a.d.heads_kv;
  a.rows = a.d.lq * a.group;
  a.parts = 1;
  // Keys of a full context's part: half as many bytes again in 4 bits (16 contexts of up
  // to 32,768 rows: 512 keys 72.7 us, 1,024 66.6, 2,048 82.6; bf16, 8 of up to 8,192: 256
  // keys 35.3, 512 34.2, 1,024 35.8).
  // In fp32, where a workgroup takes long over its keys, 4,096 keys once the rows are many
  // (one set of 12 heads, 1,560 rows, 32,760 keys: 3,319 us whole, 1,690 in parts).
  // Else many rows of enough heads fill the card by themselves.  Fewer workgroups a set than
  // half the CUs take parts of 2,048 keys, as many as go round once (bf16, one set, whole
  // / parts: 1,032 rows of one head, 131,072 keys 2,242 / 121 us, of 8 heads
  // 2,527 / 894; 1,100 rows of 2 heads of 64, 8,192 keys 125 / 41.  Batches that fill the card pay
  // for the join: 64 sets of 1,100 rows of 2 heads, 8,192 keys 692 / 775).
  const bool many = a.rows > 1024, f32 = a.d.dtype == CS_FP32 && !kv4;
  const int keys = !many ? kv4 ? 1024 : 512 : f32 ? 4096 : 2048;
  long most = 128;
  if (many && !f32) most = std::min(most, 256 / ((long)a.d.heads_kv * cdiv(a.rows, few_rows(a, kv4) ? 32 : 128)));
  if (a.d.lk > keys && most > 1) a.parts = (int)std::min<long>(most, cdiv(a.d.lk, keys));
  a.by_group = FastDiv(a.group);
  a.by_parts = FastDiv(a.parts);
  a.by_heads = FastDiv(a.d.heads_kv);
}

// Which of the fp32 kernels.  k_xattn_split does a product in bf16 terms, at twice the
// rate, but its workgroups take 128 rows and all keys in turn where those of k_xattn_f32
// take 32 rows and split the keys between their waves: it wants 64 workgroups a set (12
// heads of 128, 512 keys, here / there: 400 rows 60.7 / 29.3 us, 800 rows 62.4 / 55.1, 1,560
// rows 63.0 / 79.0; 8 such sets: 89.9 / 126, 138 / 245, 220 / 466).
static bool split_f32(const XAttnArgs& a) { return a.rows > 64 && (long)a.rows * a.d.heads_kv >= 64 * 128; }

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
  if (kv4 && !few_rows(a, kv4)) {
    // the contexts unpacked, or each set's where sets are fewer
    const size_t n = (size_t)std::min(a.d.n_q, a.d.n_kv) * a.d.lk * a.d.heads_kv * a.d.head_dim * sizeof(bf16);
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

// One row: the parts' outputs, each weighted with 2^(m_p - m).  NW waves take every
// NW-th of at most MAXP parts, lanes the channels.  Latency is all there is to it (16
// parts 4.4 us, 128 parts 4.3 us): the loads do not wait for the context's length, what
// lies past its parts is dropped after.
template <typename T, int DH, int NW, int MAXP> __global__ __launch_bounds__(64 * NW) void k_xattn_join(XAttnArgs a) {
  __shared__ float s_w[MAXP], s_o[NW][DH], s_sum;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t total = (uint32_t)(a.d.n_q * a.d.heads_kv) * a.rows;   // below 2^31
  for (uint32_t row = blockIdx.x; row < total; row += gridDim.x) {
    if (row != blockIdx.x) __syncthreads();   // s_sum is read
    const int pr = (int)(row / (uint32_t)a.rows);   // problem
    const int r = (int)row - pr * a.rows;
    const int set = a.by_heads.div(pr), head = pr - set * a.d.heads_kv;
    const long base = (long)pr * a.parts * a.rows + r;
    constexpr int NC = (DH + 63) / 64, NP = MAXP / NW, NM = (MAXP + 63) / 64;
    float o[NP][NC];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int p = min(wave + NW * i, a.parts - 1);
#pragma unroll
      for (int c = 0; c < NC; ++c)
        o[i][c] = lane + 64 * c < DH ? a.part_o[(base + (long)p * a.rows) * DH + lane + 64 * c] : 0.0f;
    }
    float2 ml[NM];
#pragma unroll
    for (int i = 0; i < NM; ++i) ml[i] = a.part_ml[base + (long)min(lane + 64 * i, a.parts - 1) * a.rows];
    int len;
    xattn_context(a, set, &len);
    const int pk = xattn_part(a, len), n = len > 0 ? (len + pk - 1) / pk : 0;
    if (wave == 0) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        if (lane + 64 * i >= n) ml[i] = make_float2(-INFINITY, 0.0f);
        mx = fmaxf(mx, ml[i].x);
      }
#pragma unroll
      for (int s = 32; s > 0; s >>= 1) mx = fmaxf(mx, __shfl_xor(mx, s, WAVE));
      if (mx == -INFINITY) mx = 0.0f;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        const float w = __builtin_amdgcn_exp2f(ml[i].x - mx);
        if (lane + 64 * i < MAXP) s_w[lane + 64 * i] = w;
        sum = fmaf(w, ml[i].y, sum);
      }
      sum = wave_sum(sum);
      if (lane == 0) s_sum = sum;
    }
    __syncthreads();
    float acc[NC] = {};
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (wave + NW * i < n) acc[c] = fmaf(s_w[wave + NW * i], o[i][c], acc[c]);
#pragma unroll
    for (int c = 0; c < NC; ++c)
      if (lane + 64 * c < DH) s_o[wave][lane + 64 * c] = acc[c];
    __syncthreads();
    for (int c = tid; c < DH; c += 64 * NW) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < NW; ++w) v += s_o[w][c];
      T* dst = (T*)a.o + set * a.d.o_b + xattn_row(a, r, head, a.d.o_r, a.d.o_h);
      dst[c] = to_t<T>(s_sum != 0.0f ? v / s_sum : 0.0f);
    }
  }
}

template <typename T, int DH> static void launch_join(const XAttnArgs& a, unsigned blocks, hipStream_t st) {
  if (a.parts <= 16)
    hipLaunchKernelGGL((k_xattn_join<T, DH, 4, 16>), dim3(blocks), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_xattn_join<T, DH, 16, 128>), dim3(blocks), dim3(1024), 0, st, a);
}

template <typename T> static hipError_t join(const XAttnArgs& a, hipStream_t st) {
  const long blocks = std::min((long)a.d.n_q * a.d.heads_kv * a.rows, 0x3FFFFFL);
  switch (a.d.head_dim) {
    case 128: launch_join<T, 128>(a, (unsigned)blocks, st); break;
    case 64: launch_join<T, 64>(a, (unsigned)blocks, st); break;
    default: launch_join<T, 32>(a, (unsigned)blocks, st); break;
  }
  return hipGetLastError();
}

template <typename T> hipError_t xattn(XAttnArgs a, bool kv4, void* work, hipStream_t st) {
  cut(a, kv4);
  const Work w = layout(a, kv4);
  a.part_o = (float*)((char*)work + w.part_o);
  a.part_ml = (float2*)((char*)work + w.part_ml);
  // grids, before anything is enqueued
  const long pr = (long)a.d.n_q * a.d.heads_kv;
  const bool few = few_rows(a, kv4), stream = !few && sizeof(T) == 2;
  if ((a.parts > 1 && pr * a.rows > 0x7FFFFFFFL) ||
      pr * a.parts * cdiv(a.rows, few ? 16 : 32) > (stream ? 0x3FFFFFFFL : 0xFFFFFFL))
    return hipErrorInvalidConfiguration;
  hipError_t e;
  if (few) {
    e = xattn_rows<T>(a, kv4, st);
  } else {
    if constexpr (sizeof(T) == 2) {
      if (kv4) {
        // many queries meet every key: unpack them once, and only the sets' contexts where
        // sets are fewer (one set of 256 rows on one of 64 contexts of 16,384 rows, 8 heads
        // of 128: 52 us and 80 MB of workspace, unpacking all of them 1,365 us and 4.1 GB)
        Kv4RowsArgs l = {};
        l.c = a.c;
        a.by_set = a.d.n_q < a.d.n_kv;
        if (a.by_set) l.ctx_of = a.kv_of;
        const long hd = (long)a.d.heads_kv * a.d.head_dim;
        l.r = {a.d.dtype, std::min(a.d.n_q, a.d.n_kv) * a.d.lk, hd, a.d.head_dim, hd, a.d.head_dim};
        l.len = a.kv_len;
        l.ko = (char*)work + w.k;
        l.vo = (char*)work + w.v;
        e = kv4_unpack(l, st);
        if (e != hipSuccess) return e;
        a.k = l.ko;
        a.v = l.vo;
        a.d.k_r = a.d.v_r = hd;
        a.d.k_h = a.d.v_h = a.d.head_dim;
        a.d.k_b = a.d.v_b = hd * a.d.lk;
      }
      e = xattn_tile(a, st);
    } else {
      e = split_f32(a) ? xattn_split(a, st) : xattn_f32(a, st);
    }
  }
  if (e == hipSuccess && a.parts > 1) e = join<T>(a, st);
  return e;
}
template hipError_t xattn<bf16>(XAttnArgs, bool, void*, hipStream_t);
template hipError_t xattn<float>(XAttnArgs, bool, void*, hipStream_t);

}  // namespace cs
