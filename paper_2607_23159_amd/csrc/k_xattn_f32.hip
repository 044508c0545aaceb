// fp32 attention to contexts where workgroups are few.
//
// The four waves of a workgroup share 32 rows and split the keys in blocks of 32;
// every fragment comes straight from L2, as in the fp32 self-attention: the fp32
// products (32 x 32 x 2) are the limit, not the loads.  The contraction of the
// value product visits the keys in the order in which the accumulators of S^T =
// K Q^T hold them; its channels are dealt to the output tiles in turn (tile dt
// takes channels NDT i + dt), so that a lane reads NDT neighbouring channels of a
// row of V with one load and holds NDT neighbours of O.  85-90 TFLOP/s where the card
// is full (two row tiles a wave spill: 60-80; two waves a SIMD without reads ahead: 75-90);
// its calls are mostly short: 2 sets of 297 rows, 77 keys, 4 heads of 64 take 8.7 us.
#include "ops.hpp"

namespace cs {

template <int DH, bool MASK> __global__ __launch_bounds__(256, 1) void k_xattn_f32(XAttnArgs a) {
  typedef Mfma32<float> MF;
  constexpr int NW = 4, NG = DH / 8, NDT = DH / 32, OLD = DH + 4;
  typedef float vrow __attribute__((ext_vector_type(NDT)));
  __shared__ __attribute__((aligned(16))) float s_o[NW][32 * OLD];
  __shared__ float s_m[NW][32], s_l[NW][32];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int n_qt = (a.rows + 31) / 32;
  int id = blockIdx.x;
  const int qt = id % n_qt;
  id /= n_qt;
  const int part = id % a.parts, pr = id / a.parts;
  const int set = pr / a.d.heads_kv, head = pr - set * a.d.heads_kv;
  int len;
  const int ctx = xattn_context(a, set, &len);
  const int pk = xattn_part(a, len), k0 = part * pk, k1 = min(len, k0 + pk);
  if (k0 >= k1 && a.parts > 1) return;   // the join does not read it
  const int r0 = qt * 32;

  const float* kb = (const float*)a.k + ctx * a.d.k_b + head * a.d.k_h + 4 * half;
  const float* vb = (const float*)a.v + ctx * a.d.v_b + head * a.d.v_h + NDT * l32;
  const uint8_t* mask = MASK ? a.mask + ctx * a.d.mask_b : nullptr;

  // lane: row l32, channels 8g + 4 half + e in qf[g][e]
  f32x4 qf[NG];
  {
    const int r = min(r0 + l32, a.rows - 1);
    const float* src = (const float*)a.q + set * a.d.q_b + xattn_row(a, r, head, a.d.q_r, a.d.q_h) + 4 * half;
#pragma unroll
    for (int g = 0; g < NG; ++g) qf[g] = *reinterpret_cast<const f32x4*>(src + 8 * g);
  }
  f32x16 o[NDT];
  float m_run = -INFINITY, l_run = 0.0f;
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;

  f32x4 kf[NG];
  auto load_k = [&](int kv0) {
    const float* src = kb + min(kv0 + l32, k1 - 1) * a.d.k_r;
#pragma unroll
    for (int g = 0; g < NG; ++g) kf[g] = *reinterpret_cast<const f32x4*>(src + 8 * g);
  };
  auto block_bits = [&](int kv0) -> uint32_t {
    if constexpr (MASK) {
      const int key = kv0 + l32;
      return (uint32_t)__ballot(key < k1 && mask[min(key, k1 - 1)] != 0);
    } else {
      return k1 - kv0 >= 32 ? ~0u : (1u << (k1 - kv0)) - 1;
    }
  };
  const int first = k0 + 32 * wave;
  if (first < k1) load_k(first);
  for (int kv0 = first; kv0 < k1; kv0 += 32 * NW) {
    const uint32_t bits = block_bits(kv0);
    vrow vf[16];   // key 8(r/4) + 4 half + r%4 of the block
#pragma unroll
    for (int r = 0; r < 16; ++r)
      vf[r] = *reinterpret_cast<const vrow*>(vb + min(kv0 + acc_row(r, lane), k1 - 1) * a.d.v_r);
    f32x16 sc[2];
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[c][r] = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[e & 1] = MF::mma(kf[g][e], qf[g][e], sc[e & 1]);
    if (kv0 + 32 * NW < k1) load_k(kv0 + 32 * NW);
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[0][r] += sc[1][r];
    if (bits != ~0u) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(bits >> acc_row(r, lane) & 1)) {
          sc[0][r] = -INFINITY;
#pragma unroll
          for (int dt = 0; dt < NDT; ++dt) vf[r][dt] = 0.0f;   // may hold anything
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[0][r]);
    mx = max_lane_pair32(mx) * a.scale_log2;
    const bool moves = mx > m_run + 8.0f;   // see k_xattn_rows
    if (__any(moves)) {
      const float m_new = moves ? mx : m_run;
      const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.0f : m_run;
    float p[16], lsum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = __builtin_amdgcn_exp2f(fmaf(sc[0][r], a.scale_log2, -m_use));
      lsum += p[r];
    }
    l_run += lsum;
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) o[dt] = MF::mma(vf[r][dt], p[r], o[dt]);
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32, WAVE);
  if (half == 0) {
    s_m[wave][l32] = m_run;
    s_l[wave][l32] = l_tot;
  }
  __syncthreads();
  float m_all = s_m[0][l32];
#pragma unroll
  for (int w = 1; w < NW; ++w) m_all = fmaxf(m_all, s_m[w][l32]);
  const float f = __builtin_amdgcn_exp2f(m_run - (m_all == -INFINITY ? 0.0f : m_all));
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    vrow y;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) y[dt] = o[dt][r] * f;
    *reinterpret_cast<vrow*>(&s_o[wave][l32 * OLD + NDT * acc_row(r, lane)]) = y;
  }
  __syncthreads();
  for (int i = tid; i < 32 * DH / 4; i += 64 * NW) {
    const int q = i / (DH / 4), c = 4 * (i % (DH / 4)), row = r0 + q;
    if (row >= a.rows) break;
    float m = s_m[0][q], l = 0.0f;
#pragma unroll
    for (int w = 1; w < NW; ++w) m = fmaxf(m, s_m[w][q]);
    const float mu = m == -INFINITY ? 0.0f : m;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      v += *reinterpret_cast<const f32x4*>(&s_o[w][q * OLD + c]);
      l = fmaf(s_l[w][q], __builtin_amdgcn_exp2f(s_m[w][q] - mu), l);
    }
    if (a.parts > 1) {
      const long at = ((long)pr * a.parts + part) * a.rows + row;
      *reinterpret_cast<f32x4*>(a.part_o + at * DH + c) = v;
      if (c == 0) a.part_ml[at] = make_float2(m, l);
    } else {
      float* dst = (float*)a.o + set * a.d.o_b + xattn_row(a, row, head, a.d.o_r, a.d.o_h) + c;
      *reinterpret_cast<f32x4*>(dst) = v * (l != 0.0f ? 1.0f / l : 0.0f);
    }
  }
}

template <int DH> static hipError_t launch(const XAttnArgs& a, hipStream_t st) {
  const long blocks = (long)a.d.n_q * a.d.heads_kv * a.parts * cdiv(a.rows, 32);
  if (a.mask)
    hipLaunchKernelGGL((k_xattn_f32<DH, true>), dim3((unsigned)blocks), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_xattn_f32<DH, false>), dim3((unsigned)blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t xattn_f32(const XAttnArgs& a, hipStream_t st) {
  switch (a.d.head_dim) {
    case 128: return launch<128>(a, st);
    case 64: return launch<64>(a, st);
    case 32: return launch<32>(a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace cs
