// bf16 attention of many queries to contexts: tiles of 64 keys shared by the waves
// of a workgroup through LDS, 32 rows per wave, online softmax.
//
// Orientation.  S^T = K Q^T and O^T = V^T P^T with 32x32x16 products, so that the
// softmax weights already sit in the operand layout of the value product: lane l holds
// row l % 32 and, in accumulator register j, key 8 (j / 4) + 4 (l / 32) + j % 4.
// Values come as rows [key][channel], and the operand V^T wants 8 keys of one
// channel per lane: two transposing LDS reads (ds_read_b64_tr_b16), of keys 4 (l / 32)
// + 0..3 and 8 + 4 (l / 32) + 0..3 of each 16, the order the registers hold them in.
//
// LDS layout.  Direct loads place 16-byte chunks anywhere in the 1 KB an instruction
// fills.  K rows are padded by one chunk, which spreads 16 rows over all banks.  A
// transposing read touches 64 bytes of four consecutive rows at a time: the 64-byte
// blocks of a V row are permuted by the row (block b of row r at b ^ vswz(r)), so
// that the four land on different banks without padding.
#include "ops.hpp"

namespace cs {

template <int DH> CS_DEV int vswz(int row) { return DH == 128 ? row & 3 : DH == 64 ? (row >> 1) & 1 : 0; }

CS_DEV bf16x4 tile_read_tr(const char* p) {
  typedef __attribute__((address_space(3))) bf16x4 lds_t;
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_t*)p);
}

template <int DH, int NW, int OCC, bool MASK> __global__ __launch_bounds__(64 * NW, OCC) void k_xattn_tile(XAttnArgs a) {
  typedef Mfma32<bf16> MF;
  typedef MF::frag frag;
  constexpr int KVT = 64, STAGES = 3;
  constexpr int CK = DH / 8 + 1, KRS = CK * 16, VRS = DH * 2;
  constexpr int K_INSTR = KVT * CK / 64, V_INSTR = KVT * DH / 8 / 64;
  static_assert(K_INSTR * 64 == KVT * CK, "whole 1 KB loads");
  constexpr int KB = K_INSTR * 1024, STAGE = KB + V_INSTR * 1024;
  constexpr int TOT = K_INSTR + V_INSTR, NPW = (TOT + NW - 1) / NW, NBUSY = TOT - (NPW - 1) * NW;
  constexpr int NKT = KVT / 32, NDT = DH / 32, NKS = DH / 16, NPS = 2;
  __shared__ __attribute__((aligned(1024))) char smem[STAGES * STAGE];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int n_qt = (a.rows + NW * 32 - 1) / (NW * 32);
  int id = xcd_contiguous(blockIdx.x, gridDim.x);
  const int qt = id % n_qt;
  id /= n_qt;
  const int part = id % a.parts, pr = id / a.parts;
  const int set = pr / a.d.heads_kv, head = pr - set * a.d.heads_kv;
  int len;
  const int ctx = xattn_context(a, set, &len);
  const int k0 = part * a.part_keys, k1 = min(len, k0 + a.part_keys);
  if (k0 >= k1 && a.parts > 1) return;   // the join does not read it
  const int r0 = (qt * NW + wave) * 32;
  const bf16* kb = (const bf16*)a.k + ctx * a.d.k_b + head * a.d.k_h;
  const bf16* vb = (const bf16*)a.v + ctx * a.d.v_b + head * a.d.v_h;
  const uint8_t* mask = MASK ? a.mask + ctx * a.d.mask_b : nullptr;
  const int k_r = (int)a.d.k_r, v_r = (int)a.d.v_r;

  // load instruction i of this wave fills slots [64g, 64g + 64) of the stage, g = wave + NW i
  int voff[NPW];
#pragma unroll
  for (int i = 0; i < NPW; ++i) {
    const int g = wave + NW * i;
    if (g < K_INSTR) {
      const int p = g * 64 + lane, row = p / CK, ch = p % CK;
      voff[i] = ch < CK - 1 ? (row * k_r + ch * 8) * 2 : 0x7FFFFFF0;   // the padding loads nothing
    } else {
      const int p = (g - K_INSTR) * 64 + lane, row = p / (DH / 8), ch = p % (DH / 8);
      voff[i] = (row * v_r + (ch ^ (vswz<DH>(row) << 2)) * 8) * 2;
    }
  }
  const bool busy = wave < NBUSY;
  auto issue = [&](int tile, int st) {
    const int kv0 = k0 + tile * KVT, last = min(KVT, k1 - kv0) - 1;   // keys past k1 load as zeros
    const bf16* kt = kb + (long)kv0 * k_r;
    const bf16* vt = vb + (long)kv0 * v_r;
    char* base = smem + st * STAGE;
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
      const int g = wave + NW * i;
      if (i < NPW - 1 || busy) {
        if (g < K_INSTR)
          buffer_load_lds16(kt, (last * k_r + DH) * 2, base + g * 1024, voff[i], 0);
        else
          buffer_load_lds16(vt, (last * v_r + DH) * 2, base + g * 1024, voff[i], 0);
      }
    }
  };

  f32x16 o[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  float m_run = -INFINITY, l_run = 0.0f;

  const int ntiles = k1 > k0 ? (k1 - k0 + KVT - 1) / KVT : 0;
  if (ntiles > 0) issue(0, 0);
  frag qf[NKS];
  {
    const int r = min(r0 + l32, a.rows - 1);
    const bf16* src = (const bf16*)a.q + set * a.d.q_b + xattn_row(a, r, head, a.d.q_r, a.d.q_h) + 8 * half;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) qf[ks] = MF::load(src + ks * 16);
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks) asm volatile("" : "+v"(qf[ks]));
  }
#pragma unroll
  for (int t = 1; t < STAGES - 1; ++t)
    if (t < ntiles) issue(t, t);

  const int lane_k = l32 * KRS + half * 16;
  // transposing reads: 16 lanes address four rows of 32 bytes; of the two groups of a
  // half, the second takes the next 16 channels
  const int vrow = 4 * half + ((lane & 15) >> 2);
  int lane_v[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
    lane_v[dt] = KB + vrow * VRS + (dt ^ vswz<DH>(vrow)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  const bf16x2 one = {(bf16)1.0f, (bf16)1.0f};

  for (int t = 0; t < ntiles; ++t) {
    // tile t has landed once only the next one is in flight; past the barrier every
    // wave has read tile t - 1, whose stage the load below refills
    if (t + 1 < ntiles) {
      if (busy) wait_all_barrier<NPW>();
      else wait_all_barrier<NPW - 1>();
    } else {
      wait_all_barrier<0>();
    }
    if (t + STAGES - 1 < ntiles) issue(t + STAGES - 1, (t + STAGES - 1) % STAGES);
    const char* pk = smem + (t % STAGES) * STAGE + lane_k;
    const char* pv = smem + (t % STAGES) * STAGE;
    const int kv0 = k0 + t * KVT;
    uint64_t bits = ~0ull;
    if constexpr (MASK) {
      const int key = kv0 + lane;
      bits = __ballot(key < k1 && mask[min(key, k1 - 1)] != 0);
    } else if (k1 - kv0 < KVT) {
      bits = (1ull << (k1 - kv0)) - 1;
    }

    f32x16 sc[NKT];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[kt][r] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
        sc[kt] = MF::mma(MF::load(reinterpret_cast<const bf16*>(pk + kt * 32 * KRS + ks * 32)), qf[ks], sc[kt]);
    if (bits != ~0ull) {
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!(bits >> (kt * 32 + acc_row(r, lane)) & 1)) sc[kt][r] = -INFINITY;
    }

    frag pf[NKT][NPS];
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[kt][r]);
    mx = max_lane_pair32(mx) * a.scale_log2;
    if (__any(mx > m_run + 8.0f)) {   // see k_xattn_rows
      const float m_new = fmaxf(m_run, mx);
      const float alpha = m_run == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= alpha;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.0f : m_run;
    float lsum = 0.0f;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
      float p[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(sc[kt][r], a.scale_log2, -m_use));
#pragma unroll
      for (int ps = 0; ps < NPS; ++ps) {
        frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (bf16)p[ps * 8 + i];
        pf[kt][ps] = f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const bf16x2 pr2 = {f[i], f[i + 1]};
          lsum = __builtin_amdgcn_fdot2_f32_bf16(pr2, one, lsum, false);
        }
      }
    }
    l_run += lsum;

#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int ps = 0; ps < NPS; ++ps)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          const char* p = pv + lane_v[dt] + (kt * 32 + ps * 16) * VRS;
          union { bf16x4 h[2]; frag f; uint32_t u[4]; } v;
          v.h[0] = tile_read_tr(p);
          v.h[1] = tile_read_tr(p + 8 * VRS);
          if constexpr (MASK) {
            if (bits != ~0ull) {   // rows that are left out may hold NaN: zeros
              const uint32_t b = (uint32_t)(bits >> (kt * 32 + ps * 16 + 4 * half));
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int at = i < 2 ? 2 * i : 4 + 2 * i;   // keys 0..3, 8..11
                v.u[i] &= (b >> at & 1 ? 0xFFFFu : 0u) | (b >> (at + 1) & 1 ? 0xFFFF0000u : 0u);
              }
            }
          }
          o[dt] = MF::mma(v.f, pf[kt][ps], o[dt]);
        }
  }

  const float l_tot = l_run + __shfl_xor(l_run, 32, WAVE);
  const int r = r0 + l32;
  if (a.parts > 1) {
    if (r < a.rows) {
      const long at = ((long)pr * a.parts + part) * a.rows + r;
      float* dst = a.part_o + at * DH + 4 * half;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<f32x4*>(dst + dt * 32 + 8 * g) =
              f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
      if (half == 0) a.part_ml[at] = make_float2(m_run, l_tot);
    }
    return;
  }
  bf16* dst = (bf16*)a.o + set * a.d.o_b + xattn_row(a, min(r, a.rows - 1), head, a.d.o_r, a.d.o_h);
  store_o_rows(o, l_tot != 0.0f ? 1.0f / l_tot : 0.0f, dst, half, r < a.rows);
}

template <int DH, int NW, int OCC> static hipError_t launch_nw(const XAttnArgs& a, hipStream_t st) {
  const long blocks = (long)a.d.n_q * a.d.heads_kv * a.parts * cdiv(a.rows, NW * 32);
  if (blocks * 64 * NW > 0xFFFFFFFFL) return hipErrorInvalidConfiguration;
  if (a.mask)
    hipLaunchKernelGGL((k_xattn_tile<DH, NW, OCC, true>), dim3((unsigned)blocks), dim3(64 * NW), 0, st, a);
  else
    hipLaunchKernelGGL((k_xattn_tile<DH, NW, OCC, false>), dim3((unsigned)blocks), dim3(64 * NW), 0, st, a);
  return hipGetLastError();
}

hipError_t xattn_tile(const XAttnArgs& a, hipStream_t st) {
  switch (a.d.head_dim) {
    case 128: return launch_nw<128, 8, 2>(a, st);
    case 64: return launch_nw<64, 8, 2>(a, st);
    case 32: return launch_nw<32, 8, 2>(a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace cs
