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
//
// Bound by the products and the LDS reads that feed them, of which one wave's softmax
// covers the other's: 1.1-1.2 PFLOP/s over long contexts (8 x 32,760 rows, 4,096 keys,
// 12 heads of 128: 5.64 ms), 85% of a large library product.  What stays outside is
// each item's queries and outputs, about 4.5 us: 512 keys 0.85-0.98 ms.
#include "ops.hpp"

#include <algorithm>

namespace cs {

template <int DH> CS_DEV int vswz(int row) { return DH == 128 ? row & 3 : DH == 64 ? (row >> 1) & 1 : 0; }

// Waits in a form that the compiler counts: it then knows that the register loads
// from before have landed, and adds no wait of its own among the direct loads behind.
CS_DEV void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }   // vmcnt 0
CS_DEV void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }     // lgkmcnt 0

// One item of work: 32 NW rows of one part of a problem.
struct TileItem {
  int set, head, part, r0, k0, k1;
  const bf16 *kb, *vb;
  const uint8_t* mask;
};

template <int DH, int NW, int OCC, bool MASK> __global__ __launch_bounds__(64 * NW, OCC) void k_xattn_tile(XAttnArgs a, FastDiv by_qt, int n_items, int sorted) {
  typedef Mfma32<bf16> MF;
  typedef MF::frag frag;
  constexpr int KVT = 64, CK = DH / 8 + 1, KRS = CK * 16, VRS = DH * 2;
  constexpr int K_INSTR = KVT * CK / 64, V_INSTR = KVT * DH / 8 / 64;   // 1 KB each
  constexpr int K_NPW = (K_INSTR + NW - 1) / NW, V_NPW = (V_INSTR + NW - 1) / NW;
  constexpr int KB = K_INSTR * 1024, STAGE = KB + V_INSTR * 1024;
  constexpr int NKT = KVT / 32, NDT = DH / 32, NKS = DH / 16, NPS = 2;
  // Rows of q and o cross the wave's part of this on their way, 128 bytes of 32 rows at
  // a time, so that memory sees whole lines (64 bytes with head dim 32, and with four
  // waves, of which two workgroups share a CU's LDS).
  constexpr int SEG = DH == 32 || NW == 4 ? 64 : 128, SRS = SEG + 16, NSEG = 2 * DH / SEG, CPS = SEG / 16, RPI = 64 / CPS;
  constexpr int SI = 32 / RPI;   // instructions of a segment
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE + NW * 32 * SRS];

  lds_char* const lds = (lds_char*)smem;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int k_r = (int)a.d.k_r, v_r = (int)a.d.v_r;

  auto row_offset = [&](const TileItem& it, int row, long stride_r, long stride_h) {
    return xattn_row(a, min(it.r0 + wave * 32 + row, a.rows - 1), it.head, stride_r, stride_h);
  };
  // f(i, offset) of row i * RPI + lane / CPS of this wave, i = 0 .. SI - 1: one step apart
  // where every query is a row and none lies past the last
  auto each_row = [&](const TileItem& it, int lane, long stride_r, long stride_h, auto f) {
    if (a.group == 1 && it.r0 + wave * 32 + 32 <= a.rows) {
      const long at = (long)(it.r0 + wave * 32 + lane / CPS) * (int)stride_r + (long)it.head * (int)stride_h;
#pragma unroll
      for (int i = 0; i < SI; ++i) f(i, at + i * (RPI * stride_r));
    } else {
#pragma unroll
      for (int i = 0; i < SI; ++i) f(i, row_offset(it, i * RPI + lane / CPS, stride_r, stride_h));
    }
  };
  // Sets in the order of their contexts' lengths, the longest first: a workgroup's items of
  // the rounds then add up to much the same (8 sets of 1,560 queries, 4 prompts of up to 512
  // rows, 12 heads of 128: 41.2 us, 47.1 in the sets' own order with rounds one way, 42.3 back
  // and forth).  At most 64 sets, one a lane: 64 of 400 queries, up to 512 keys, take 73.4
  // us, 80.7 in their own order, which 65 keep (89.5).
  __shared__ int s_order[64];
  if (sorted) {
    if (wave == 0) {
      int len = 0, rank = 0;
      if (lane < a.d.n_q) {
        const int j = a.kv_of ? a.kv_of[lane] : lane;
        if (j >= 0 && j < a.d.n_kv) len = max(0, min(a.kv_len[j], a.d.lk));
      }
      for (int i = 0; i < a.d.n_q; ++i) {
        const int other = __builtin_amdgcn_readlane(len, i);
        rank += other > len || (other == len && i < lane);
      }
      if (lane < a.d.n_q) s_order[rank] = lane;
    }
    __syncthreads();
  }

  // The next item of this workgroup with keys to read, from index i on; items without
  // any get their zeros (in parts: nothing, the join does not read them).  Rows past
  // the last are copies of it: every load is in bounds, and the last row gets its zeros
  // several times.
  const int place = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);   // an XCD takes neighbouring items
  auto find = [&](int& i, TileItem& it) {
    for (;; ++i) {
      // back and forth, so that who has a long item of one round has a short one of the next
      const int id = i * (int)gridDim.x + (i & 1 ? (int)gridDim.x - 1 - place : place);
      if (id >= n_items) return false;
      const int n = by_qt.div(id), qt = id - n * by_qt.d;
      const int pr = a.by_parts.div(n);
      it.part = n - pr * a.parts;
      it.set = a.by_heads.div(pr);
      it.head = pr - it.set * a.d.heads_kv;
      if (sorted) it.set = __builtin_amdgcn_readfirstlane(s_order[it.set]);
      it.r0 = qt * NW * 32;
      int len;
      const int ctx = xattn_context(a, it.set, &len);
      const int pk = xattn_part(a, len);
      it.k0 = it.part * pk;
      it.k1 = min(len, it.k0 + pk);
      const int kv = a.by_set ? it.set : ctx;
      it.kb = (const bf16*)a.k + kv * a.d.k_b + it.head * a.d.k_h;
      it.vb = (const bf16*)a.v + kv * a.d.v_b + it.head * a.d.v_h;
      it.mask = MASK ? a.mask + ctx * a.d.mask_b : nullptr;
      if (it.k0 < it.k1) return true;
      if (a.parts == 1) {
        bf16* dst = (bf16*)a.o + it.set * a.d.o_b + row_offset(it, l32, a.d.o_r, a.d.o_h) + 8 * half;
#pragma unroll
        for (int c = 0; c < DH; c += 16) *reinterpret_cast<uint4*>(dst + c) = make_uint4(0, 0, 0, 0);
      }
    }
  };

  // load instruction i of this wave fills slots [64g, 64g + 64) of a tile, g = wave + NW i
  int koff[K_NPW], voff[V_NPW];
#pragma unroll
  for (int i = 0; i < K_NPW; ++i) {
    const int p = (wave + NW * i) * 64 + lane, row = p / CK, ch = p % CK;
    koff[i] = ch < CK - 1 ? (row * k_r + ch * 8) * 2 : 0x7FFFFFF0;   // the padding loads nothing
  }
#pragma unroll
  for (int i = 0; i < V_NPW; ++i) {
    const int p = (wave + NW * i) * 64 + lane, row = p / (DH / 8), ch = p % (DH / 8);
    voff[i] = (row * v_r + (ch ^ (vswz<DH>(row) << 2)) * 8) * 2;
  }
  auto issue = [&](const bf16* kb, const bf16* vb, int kv0, int k1, int st) {
    const int last = min(KVT, k1 - kv0) - 1;   // keys past k1 load as zeros
    const bf16 *ks = kb + (long)kv0 * k_r, *vs = vb + (long)kv0 * v_r;
    lds_char* base = lds + st * STAGE + wave * 1024;
#pragma unroll
    for (int i = 0; i < K_NPW; ++i)
      if ((i + 1) * NW <= K_INSTR || wave + NW * i < K_INSTR)
        load_lds16(ks, (last * k_r + DH) * 2, base + NW * i * 1024, koff[i]);
#pragma unroll
    for (int i = 0; i < V_NPW; ++i)
      if ((i + 1) * NW <= V_INSTR || wave + NW * i < V_INSTR)
        load_lds16(vs, (last * v_r + DH) * 2, base + KB + NW * i * 1024, voff[i]);
  };
  char* const seg = smem + 2 * STAGE + wave * 32 * SRS;
  static_assert(NSEG * SI == NKS, "as many operands as loads");
  frag qf[NKS];   // between load_q and turn_q: the rows as they come from memory
  auto load_q = [&](const TileItem& it) {
    const bf16* src = (const bf16*)a.q + it.set * a.d.q_b + 8 * (lane % CPS);
    each_row(it, lane, a.d.q_r, a.d.q_h, [&](int i, long at) {
#pragma unroll
      for (int s = 0; s < NSEG; ++s) qf[s * SI + i] = MF::load(src + at + s * (SEG / 2));
    });
  };
  auto turn_q = [&]() {   // to operands: lane row l32, channels 16 ks + 8 half
#pragma unroll
    for (int s = 0; s < NSEG; ++s) {
#pragma unroll
      for (int i = 0; i < SI; ++i)
        *reinterpret_cast<frag*>(seg + (i * RPI + lane / CPS) * SRS + 16 * (lane % CPS)) = qf[s * SI + i];
#pragma unroll
      for (int ks = 0; ks < SI; ++ks)
        qf[s * SI + ks] = *reinterpret_cast<const frag*>(seg + l32 * SRS + 32 * ks + 16 * half);
    }
  };

  TileItem cur, nxt;
  int i = 0;
  if (!find(i, cur)) return;
  issue(cur.kb, cur.vb, cur.k0, cur.k1, 0);
  load_q(cur);
  bool more = find(++i, nxt);

  f32x16 o[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
  float m_run = -INFINITY, l_run = 0.0f;

  const int lane_k = l32 * KRS + half * 16;
  // transposing reads: 16 lanes address four rows of 32 bytes; of the two groups of a
  // half, the second takes the next 16 channels
  const int vrow = 4 * half + ((lane & 15) >> 2);
  int lane_v[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
    lane_v[dt] = KB + vrow * VRS + (dt ^ vswz<DH>(vrow)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
  const bf16x2 one = {(bf16)1.0f, (bf16)1.0f};

  // The tiles of all items in one stream: the next item's first tile and its queries
  // are on their way while this one's last tile is worked on, and its output drains
  // under the next one's.
  int kv0 = cur.k0;
  // a tile's mask bytes, asked for with the tile: read when needed they would have to be
  // waited for, and with them the direct loads before them (8 x 32,760 rows, 512 keys
  // half masked, 12 heads of 128: 1,140 against 1,420 us)
  auto mask_byte = [&](const TileItem& it, int from) { return it.mask[min(from + lane, it.k1 - 1)]; };
  uint8_t mask_here = 0, mask_next = 0;
  if constexpr (MASK) mask_here = mask_byte(cur, kv0);
  turn_q();
  wait_loads();
  for (int st = 0;; st ^= 1) {
    // this wave's loads of the tile have landed (wait_loads below); past the barrier
    // every wave's have, and every wave has read the other stage, which is refilled
    wait_lds();
    asm volatile("s_barrier" ::: "memory");
    const bool last = kv0 + KVT >= cur.k1;
    if (!last || more) {
      issue(last ? nxt.kb : cur.kb, last ? nxt.vb : cur.vb, last ? nxt.k0 : kv0 + KVT, last ? nxt.k1 : cur.k1, st ^ 1);
      if constexpr (MASK) mask_next = last ? mask_byte(nxt, nxt.k0) : mask_byte(cur, kv0 + KVT);
    }
    const char* pk = smem + st * STAGE + lane_k;
    const lds_char* pv = lds + st * STAGE;
    uint64_t bits = ~0ull;
    if constexpr (MASK) {
      bits = __ballot(kv0 + lane < cur.k1 && mask_here != 0);
    } else if (cur.k1 - kv0 < KVT) {
      bits = (1ull << (cur.k1 - kv0)) - 1;
    }

    f32x16 sc[NKT];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[kt][r] = 0.0f;
    // key operands are read four steps ahead of their products, and half of the values
    // ahead of the softmax: read one at a time they leave the products waiting for LDS
#pragma unroll
    for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
        sc[kt] = MF::mma(MF::load(reinterpret_cast<const bf16*>(pk + kt * 32 * KRS + ks * 32)), qf[ks], sc[kt]);
    constexpr int AHEAD = NKS < 4 ? NKS : 4;
    __builtin_amdgcn_sched_group_barrier(0x100, NKT * AHEAD, 0);
#pragma unroll
    for (int ks = 0; ks < NKS - AHEAD; ++ks) {
      __builtin_amdgcn_sched_group_barrier(0x008, NKT, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, NKT, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, NKT * AHEAD, 0);
    union ValueFrag { bf16x4 h[2]; frag f; uint32_t u[4]; };
    auto value = [&](int kt, int ps, int dt) {
      const lds_char* p = pv + lane_v[dt] + (kt * 32 + ps * 16) * VRS;
      ValueFrag v;
      v.h[0] = lds_read_tr(p);
      v.h[1] = lds_read_tr(p + 8 * VRS);
      return v;
    };
    ValueFrag vf[NPS][NDT];
#pragma unroll
    for (int ps = 0; ps < NPS; ++ps)
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt) vf[ps][dt] = value(0, ps, dt);
    asm volatile("" ::: "memory");
    if (last && more) load_q(nxt);
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
    const bool moves = mx > m_run + 8.0f;   // see k_xattn_rows
    if (kv0 == cur.k0) {   // nothing seen yet: nothing to scale
      m_run = mx;
    } else if (__any(moves)) {
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
    float lsum = 0.0f;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int ps = 0; ps < NPS; ++ps) {
        frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          f[i] = (bf16)__builtin_amdgcn_exp2f(fmaf(sc[kt][ps * 8 + i], a.scale_log2, -m_use));
        pf[kt][ps] = f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const bf16x2 pr2 = {f[i], f[i + 1]};
          lsum = __builtin_amdgcn_fdot2_f32_bf16(pr2, one, lsum, false);
        }
      }
    l_run += lsum;

#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int ps = 0; ps < NPS; ++ps)
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
          ValueFrag v = kt == 0 ? vf[ps][dt] : value(kt, ps, dt);
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
    if (!last) {
      kv0 += KVT;
      wait_loads();
      mask_here = mask_next;
      continue;
    }

    // the next item's first tile and queries were asked for a round ago; the stores
    // behind this wait then drain under its work
    wait_loads();
    mask_here = mask_next;
    // Only rows that exist are stored: nothing is written by two waves.
    const int live = a.rows - cur.r0 - wave * 32;   // rows of this wave that exist
    const float l_tot = l_run + __shfl_xor(l_run, 32, WAVE);
    // the lane's number, formed anew: what follows from it is then not kept in registers
    // over the products (the masked and the 12-wave variants spill for it)
    int here = 0;
    asm volatile("" : "+v"(here));
    here = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, here));
    if (a.parts > 1) {
      const int pr = cur.set * a.d.heads_kv + cur.head;
      const long at = ((long)pr * a.parts + cur.part) * a.rows + cur.r0 + wave * 32 + (here & 31);
      float* dst = a.part_o + at * DH + 4 * (here >> 5);
      if ((here & 31) < live) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(dst + dt * 32 + 8 * g) =
                f32x4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
        if (here < 32) a.part_ml[at] = make_float2(m_run, l_tot);
      }
    } else {
      const float inv = l_tot != 0.0f ? 1.0f / l_tot : 0.0f;
      bf16* dst = (bf16*)a.o + cur.set * a.d.o_b + 8 * (here % CPS);
      constexpr int DPS = NDT / NSEG;   // 32-channel blocks of a segment
      long at[SI];
      each_row(cur, here, a.d.o_r, a.d.o_h, [&](int i, long x) { at[i] = x; });
#pragma unroll
      for (int s = 0; s < NSEG; ++s) {
        f32x16 os[DPS];
#pragma unroll
        for (int d = 0; d < DPS; ++d) os[d] = o[s * DPS + d];
        store_o_rows(os, inv, reinterpret_cast<bf16*>(seg + l32 * SRS), half, true);
        frag y[SI];
#pragma unroll
        for (int i = 0; i < SI; ++i) y[i] = *reinterpret_cast<const frag*>(seg + (i * RPI + here / CPS) * SRS + 16 * (here % CPS));
        if (live >= 32) {
#pragma unroll
          for (int i = 0; i < SI; ++i) *reinterpret_cast<frag*>(dst + at[i] + s * (SEG / 2)) = y[i];
        } else {
#pragma unroll
          for (int i = 0; i < SI; ++i)
            if (i * RPI + here / CPS < live) *reinterpret_cast<frag*>(dst + at[i] + s * (SEG / 2)) = y[i];
        }
      }
    }
    if (!more) return;
    turn_q();
    cur = nxt;
    more = find(++i, nxt);
    kv0 = cur.k0;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[dt][r] = 0.0f;
    m_run = -INFINITY;
    l_run = 0.0f;
  }
}

// Items go round the workgroups that fill the chip's 256 CUs: one of 8 or 12 waves each,
// or two of 4.
template <int DH, int NW> static hipError_t launch_nw(const XAttnArgs& a, hipStream_t st) {
  constexpr int OCC = NW == 12 ? 3 : 2;
  const long items = (long)a.d.n_q * a.d.heads_kv * a.parts * cdiv(a.rows, NW * 32);
  const dim3 grid((unsigned)std::min<long>(round_up(items, 8), 256 * (NW == 4 ? 2 : 1))), block(64 * NW);
  const FastDiv by_qt(cdiv(a.rows, NW * 32));
  const int sorted = a.kv_len && a.d.n_q > 1 && a.d.n_q <= 64 && items > grid.x;
  if constexpr (NW < 12) {   // with 12 waves the masks' registers do not fit
    if (a.mask) {
      hipLaunchKernelGGL((k_xattn_tile<DH, NW, OCC, true>), grid, block, 0, st, a, by_qt, (int)items, sorted);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((k_xattn_tile<DH, NW, OCC, false>), grid, block, 0, st, a, by_qt, (int)items, sorted);
  return hipGetLastError();
}

// 8 waves share a tile of keys between twice the rows of 4, which a full chip runs 7%
// faster (8 sets of 32,760 queries, 512 keys, 12 heads of 128: 0.96 against 1.03 ms; 4 x
// 1,560: 39.2 against 40.7 us); 4 waves fill it sooner and leave smaller last rounds
// (1 x 1,560: 14.3 against 17.6 us; 4 x 384, 40 heads: 24.1 against 38.5).  Up to head dim
// 64 three waves fit a SIMD: 12 take 384 rows at 7% less a row (8 x 32,760 x 512, 12 heads
// of 64: 602 against 641 us; 4,096 keys 3.68 against 4.02 ms; 2 x 5,000, 300 keys, 4
// heads: 13.5 against 11.2 us, in one unfilled round).  A wave's arithmetic is the same in
// all of them, so results are bitwise equal.
template <int DH> static hipError_t launch_dh(const XAttnArgs& a, hipStream_t st) {
  const long pr = (long)a.d.n_q * a.d.heads_kv * a.parts;
  const long i4 = pr * cdiv(a.rows, 128);
  const double t4 = i4 <= 256 ? 0.82 : 1.07 * cdiv(i4, 512), t8 = cdiv(pr * cdiv(a.rows, 256), 256);
  if constexpr (DH <= 64) {
    const double t12 = 1.39 * cdiv(pr * cdiv(a.rows, 384), 256);
    if (!a.mask && t12 < t8 && t12 < t4) return launch_nw<DH, 12>(a, st);
  }
  return t4 < t8 ? launch_nw<DH, 4>(a, st) : launch_nw<DH, 8>(a, st);
}

hipError_t xattn_tile(const XAttnArgs& a, hipStream_t st) {
  switch (a.d.head_dim) {
    case 128: return launch_dh<128>(a, st);
    case 64: return launch_dh<64>(a, st);
    case 32: return launch_dh<32>(a, st);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace cs
