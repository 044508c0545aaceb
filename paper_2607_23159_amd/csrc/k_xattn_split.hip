// fp32 attention of many queries to contexts, in bf16 products.
//
// An fp32 number is a sum of three bf16 terms x0 + x1 + x2 of 8 bits each, so a product
// x y is x0 y0 + (x0 y1 + x1 y0) + (x0 y2 + x1 y1 + x2 y0) and terms below 2^-23 |x y|,
// which are left out.  Six bf16 products of 16 x 16 x 32 take 2.7 times less time than one
// in fp32.
//
// A workgroup's four waves take 32 rows each; they split the keys and values of a block of
// 32 between them, once for all 128 rows, and leave the terms in LDS.  Scores, softmax and
// value product as in k_xattn_rows.  Two workgroups share a CU: one's splitting and
// softmax run under the other's products.  12 heads of 128, 1,560 rows: one set of 32,760
// keys 1,594 us (197 TFLOP/s; a library fp32 product reaches 153, k_xattn_f32 111), 8 sets
// of 512 keys 220 us (178 TFLOP/s, matrix pipe 46% busy).  Splitting in the registers of every wave, 32 rows at a
// time, measured 65 TFLOP/s: twice as many instructions go to the terms as to the rest.
#include "xattn_mma.hpp"

namespace cs {

template <int DH, bool MASK> __global__ __launch_bounds__(256, 2) void k_xattn_split(XAttnArgs a, FastDiv by_blocks) {
  typedef LdsRows<DH> Rows;
  constexpr int NW = 4, NS = 3, RT = 2, KEYS = 32, KS = DH / 32, NC = DH / 8, NCT = DH / 16;
  constexpr int PLANE = KEYS * Rows::BYTES, PER = (KEYS * NC + 255) / 256;
  __shared__ __attribute__((aligned(1024))) char smem[2 * NS * PLANE];
  lds_char *const lk = (lds_char*)smem, *const lv = lk + NS * PLANE;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int id = xcd_contiguous(blockIdx.x, gridDim.x);
  const int at = by_blocks.div(id), r0 = (id - at * (int)by_blocks.d) * 16 * RT * NW + 16 * RT * wave;
  const int pr = a.by_parts.div(at), part = at - pr * a.parts;
  const int set = a.by_heads.div(pr), head = pr - set * a.d.heads_kv;
  int len;
  const int ctx = xattn_context(a, set, &len);
  const int pk = xattn_part(a, len), k0 = part * pk, k1 = min(len, k0 + pk);
  if (k0 >= k1 && a.parts > 1) return;   // the join does not read it

  const char* kb = (const char*)((const float*)a.k + ctx * a.d.k_b + head * a.d.k_h);
  const char* vb = (const char*)((const float*)a.v + ctx * a.d.v_b + head * a.d.v_h);
  const int k_b = 4 * (int)a.d.k_r, v_b = 4 * (int)a.d.v_r;
  const uint8_t* mask = MASK ? a.mask + ctx * a.d.mask_b : nullptr;

  // Q^T operands
  bf16x8 qf[NS][RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = min(r0 + 16 * rt + l16, a.rows - 1);
    const float* src = (const float*)a.q + set * a.d.q_b + xattn_row(a, r, head, a.d.q_r, a.d.q_h);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float x[8];
      bf16x8 t[NS];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = src[32 * ks + 8 * g + i];
      split_bf16<NS>(x, t);
#pragma unroll
      for (int n = 0; n < NS; ++n) qf[n][rt][ks] = t[n];
    }
  }

  f32x4 o[RT][NCT];
  float m_run[RT], l_run[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m_run[rt] = -INFINITY;
    l_run[rt] = 0.0f;
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) o[rt][ct] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // chunk i of this thread: 8 channels of a row
  f32x4 kr[PER][2], vr[PER][2];
  auto request = [&](int kv0) {
    const int last = k1 - 1 - kv0;   // past the last: the last again
    const char *kt = kb + (long)kv0 * k_b, *vt = vb + (long)kv0 * v_b;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = tid + 256 * i, row = min(c / NC, last);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        kr[i][h] = *reinterpret_cast<const f32x4*>(kt + (uint32_t)(row * k_b + 32 * (c % NC) + 16 * h));
        vr[i][h] = *reinterpret_cast<const f32x4*>(vt + (uint32_t)(row * v_b + 32 * (c % NC) + 16 * h));
      }
    }
  };
  auto stage = [&](lds_char* rows, int c, const f32x4* raw, bool left) {
    float x[8];
    bf16x8 t[NS];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = raw[i / 4][i % 4];
    split_bf16<NS>(x, t);
#pragma unroll
    for (int n = 0; n < NS; ++n) Rows::put(rows + n * PLANE, c / NC, c % NC, left ? t[n] : bf16x8{});
  };

  if (k0 < k1) request(k0);
  for (int kv0 = k0; kv0 < k1; kv0 += KEYS) {
    const uint64_t bits = tile_bits<KEYS, MASK>(mask, kv0, k1, lane);
    const bool some = bits != (1ull << KEYS) - 1;
    __syncthreads();   // the block before is read
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = tid + 256 * i;
      if (KEYS * NC % 256 != 0 && c >= KEYS * NC) break;
      stage(lk, c, kr[i], true);
      stage(lv, c, vr[i], bits >> (c / NC) & 1);   // those that are left out may hold anything: zeros
    }
    __syncthreads();
    if (kv0 + KEYS < k1) request(kv0 + KEYS);

    f32x4 sc[2][RT];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) sc[t][rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        bf16x8 kf[NS];
#pragma unroll
        for (int n = 0; n < NS; ++n) kf[n] = Rows::get(lk + n * PLANE, 16 * t + l16, 4 * ks + g);
#pragma unroll
        for (int s = NS - 1; s >= 0; --s)
#pragma unroll
          for (int n = 0; n <= s; ++n)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) sc[t][rt] = mma16(kf[s - n], qf[n][rt][ks], sc[t][rt]);
      }
    }
    if (some) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!(bits >> (16 * t + 4 * g + j) & 1))
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) sc[t][rt][j] = -INFINITY;
    }
    bf16x8 pf[NS][RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sc[t][rt][j]);
      mx = max_groups16(mx) * a.scale_log2;
      const bool moves = mx > m_run[rt] + 8.0f;   // see k_xattn_rows
      if (__any(moves)) {
        const float m_new = moves ? mx : m_run[rt];
        const float alpha = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[rt] - m_new);
        m_run[rt] = m_new;
        l_run[rt] *= alpha;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) o[rt][ct] *= alpha;
      }
      const float m_use = m_run[rt] == -INFINITY ? 0.0f : m_run[rt];
      float p[8], lsum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i / 4][rt][i % 4], a.scale_log2, -m_use));
        lsum += p[i];
      }
      l_run[rt] += lsum;
      bf16x8 t[NS];
      split_bf16<NS>(p, t);
#pragma unroll
      for (int n = 0; n < NS; ++n) pf[n][rt] = t[n];
    }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      bf16x8 vf[NS];
#pragma unroll
      for (int n = 0; n < NS; ++n) vf[n] = Rows::operand(lv + n * PLANE, lane, ct);
#pragma unroll
      for (int s = NS - 1; s >= 0; --s)
#pragma unroll
        for (int n = 0; n <= s; ++n)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) o[rt][ct] = mma16(vf[s - n], pf[n][rt], o[rt][ct]);
    }
  }

#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = sum_groups16(l_run[rt]);
    const int r = r0 + 16 * rt + l16;
    if (r >= a.rows) continue;
    if (a.parts > 1) {
      const long at = ((long)pr * a.parts + part) * a.rows + r;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) *reinterpret_cast<f32x4*>(a.part_o + at * DH + 16 * ct + 4 * g) = o[rt][ct];
      if (g == 0) a.part_ml[at] = make_float2(m_run[rt], l);
    } else {
      float* dst = (float*)a.o + set * a.d.o_b + xattn_row(a, r, head, a.d.o_r, a.d.o_h) + 4 * g;
      const float inv = l != 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) *reinterpret_cast<f32x4*>(dst + 16 * ct) = o[rt][ct] * inv;
    }
  }
}

template <int DH> static hipError_t launch(const XAttnArgs& a, hipStream_t st) {
  const FastDiv by_blocks(cdiv(a.rows, 128));
  const dim3 grid((unsigned)((long)a.d.n_q * a.d.heads_kv * a.parts * by_blocks.d)), block(256);
  if (a.mask)
    hipLaunchKernelGGL((k_xattn_split<DH, true>), grid, block, 0, st, a, by_blocks);
  else
    hipLaunchKernelGGL((k_xattn_split<DH, false>), grid, block, 0, st, a, by_blocks);
  return hipGetLastError();
}

hipError_t xattn_split(const XAttnArgs& a, hipStream_t st) {
  switch (a.d.head_dim) {
    case 128: return launch<128>(a, st);
    case 64: return launch<64>(a, st);
    case 32: return launch<32>(a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace cs
