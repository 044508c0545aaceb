// Attention of few queries (a token or a handful, with the heads that share a key
// head) to a context, 32 rows at a time: keys and values are read once for them, from
// memory.  Over a 4-bit cache in fp32, of any number of queries.
//
// Work split.  A workgroup takes one part of a problem's keys, its four waves the
// part's tiles in turn, each on its own: no barrier until the waves' outputs are
// joined at the end.
//
// Orientation.  S^T = K Q^T and O^T = V^T P^T with 16x16x32 products: lane l holds
// query l % 16 of a row tile, and keys 4 (l / 16) + j of 16 in accumulator register
// j.  The value product's operand of lane l wants 8 keys of 32: it takes those two
// 16-key score blocks hold there, 4 (l / 16) + j and 16 + 4 (l / 16) + j, and reads
// the same keys of V^T through two transposing LDS reads (ds_read_b64_tr_b16: lane i
// of 16 gets column i of the 4 rows that the 16 lanes address).
//
// Bound by the read of the keys and values: 8 contexts of up to 8,192 rows, 8 key heads
// of 128, one token: 134 MB in 23-28 us (4.8-5.8 TB/s); in 4 bits, 16 of up to 32,768
// rows: 314 MB in 62 us (5.1 TB/s); one of 131,072 rows: 143 MB in 27 us (5.3 TB/s).
// Over 4 bits the conversions and products bound it from 32 rows a key head on: 500
// TFLOP/s, 220 with fp32 queries.
#include "xattn_mma.hpp"

namespace cs {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A tile of 32 keys on its way through the registers of a wave.  Lane l: keys l % 16 and
// 16 + l % 16, every fourth chunk of a row.  Whole tiles are read at constant offsets
// from a uniform address.  Plain loads: marked as streaming they are faster on contexts
// that no cache holds (32 of 8,192 rows, 8 key heads: 180 us against 191) and slower on
// those that a decoding loop meets again in the last-level cache (8: 52.4 against 46.8).
template <int DH, bool MASK> struct TileBf16 {
  static constexpr int KEYS = 32, KS = DH / 32, NC = DH / 8, WAVES = 2;
  const char *kp, *vp;   // row k0
  int k_b, v_b;          // bytes from row to row
  const uint8_t* mask;
  int k1, lane, koff;
  bf16x8 k[2][KS], v[2][KS];
  uint64_t bits;

  CS_DEV TileBf16(const XAttnArgs& a, int ctx, int head, const uint8_t* mask_, int k1_, int lane_)
      : k_b(2 * (int)a.d.k_r), v_b(2 * (int)a.d.v_r), mask(mask_), k1(k1_), lane(lane_) {
    kp = (const char*)((const bf16*)a.k + ctx * a.d.k_b + head * a.d.k_h);
    vp = (const char*)((const bf16*)a.v + ctx * a.d.v_b + head * a.d.v_h);
    koff = (lane & 15) * k_b + 16 * (lane >> 4);
  }
  // channel of element 0 of step ks in lane group g
  static CS_DEV int channel(int ks, int g) { return 32 * ks + 8 * g; }
  static CS_DEV bf16x8 fetch(const char* p) { return *reinterpret_cast<const bf16x8*>(p); }
  CS_DEV void request(int kv0) {
    const bool whole = k1 - kv0 >= KEYS;
    const int last = k1 - 1 - kv0;
    const char *kt = kp + (long)kv0 * k_b, *vt = vp + (long)kv0 * v_b;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint32_t ko = koff + 16 * t * k_b;
      if (!whole) ko = min(16 * t + (lane & 15), last) * k_b + 16 * (lane >> 4);   // past the last: the last again
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) k[t][ks] = fetch(kt + ko + 64 * ks);
    }
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      const uint32_t vo = min(row(i), whole ? KEYS : last) * v_b + 16 * (lane % NC);
      v[i / KS][i % KS] = fetch(vt + vo);
    }
    bits = tile_bits<KEYS, MASK>(mask, kv0, k1, lane);
  }
  CS_DEV int row(int i) const { return (64 / NC) * i + lane / NC; }
  CS_DEV bf16x8 key(int t, int ks) const { return k[t][ks]; }
  // the values of the tile into LDS, whole rows at a time; those that are left out may
  // hold anything: they become zeros
  CS_DEV void stage(lds_char* rows, uint64_t bits, bool some) const {
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      const bool left = !some || (bits >> row(i) & 1);
      LdsRows<DH>::put(rows, row(i), lane % NC, left ? v[i / KS][i % KS] : bf16x8{});
    }
  }
};

// The same of a 4-bit cache, with loads marked as streaming.  A lane reads a quarter of a key's codes, which lie
// together and (from head dim 64 on) under one scale byte; the score product visits
// the channels in that order.
template <int DH, bool MASK> struct TileKv4 {
  static constexpr int KEYS = 32, KS = DH / 32, WAVES = 4;
  const uint8_t *kc, *ks_, *vc, *vs_;   // row 0
  const uint8_t* mask;
  int k1, lane;
  uint32_t k[2][KS], v[2][KS], kb[2], vb[2];
  uint64_t bits;

  CS_DEV TileKv4(const XAttnArgs& a, int ctx, int head, const uint8_t* mask_, int k1_, int lane_)
      : mask(mask_), k1(k1_), lane(lane_) {
    const long at = ((long)ctx * a.c.heads + head) * a.c.cap;
    kc = a.c.k_codes + at * (DH / 2);
    vc = a.c.v_codes + at * (DH / 2);
    ks_ = a.c.k_scales + at * (DH / 32);
    vs_ = a.c.v_scales + at * (DH / 32);
  }
  static CS_DEV int channel(int ks, int g) { return DH / 4 * g + 8 * ks; }
  static CS_DEV void fetch(const uint8_t* p, uint32_t* d) {
    if constexpr (KS == 4) {
      const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
      d[0] = x[0]; d[1] = x[1]; d[2] = x[2]; d[3] = x[3];
    } else if constexpr (KS == 2) {
      const u32x2 x = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
      d[0] = x[0]; d[1] = x[1];
    } else {
      d[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
    }
  }
  CS_DEV void request(int kv0) {
    const bool whole = k1 - kv0 >= KEYS;
    const uint8_t *kt = kc + (long)kv0 * (DH / 2), *vt = vc + (long)kv0 * (DH / 2);
    const uint8_t *kst = ks_ + (long)kv0 * (DH / 32), *vst = vs_ + (long)kv0 * (DH / 32);
    const int g = lane >> 4;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      uint32_t row = 16 * t + (lane & 15);
      if (!whole) row = min((int)row, k1 - 1 - kv0);
      fetch(kt + (row * (DH / 2) + g * (DH / 8)), k[t]);
      fetch(vt + (row * (DH / 2) + g * (DH / 8)), v[t]);
      kb[t] = kst[row * (DH / 32) + g * DH / 128];
      vb[t] = vst[row * (DH / 32) + g * DH / 128];
    }
    bits = tile_bits<KEYS, MASK>(mask, kv0, k1, lane);
  }
  CS_DEV bf16x8 key(int t, int ks) const { return kv4_decode8(k[t][ks], kv4_scale(kb[t])); }
  CS_DEV void stage(lds_char* rows, uint64_t bits, bool some) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = 16 * t + (lane & 15);
      const bool left = !some || (bits >> row & 1);
      const float s = kv4_scale(left ? vb[t] : 127);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        LdsRows<DH>::put(rows, row, DH / 32 * (lane >> 4) + ks, kv4_decode8(left ? v[t][ks] : 0, s));
    }
  }
};

// NS: bf16 terms of a query and of a softmax weight (1: bf16; 3: fp32).
template <typename T, int DH, int RT, int NS, bool MASK, typename Tile>
__global__ __launch_bounds__(256, NS > 1 ? 1 : RT > 1 ? 2 : Tile::WAVES) void k_xattn_rows(XAttnArgs a, FastDiv by_blocks) {
  typedef LdsRows<DH> Rows;
  constexpr int NW = 4, KS = DH / 32, NCT = DH / 16, OLD = DH + 4, KEYS = Tile::KEYS;
  constexpr uint64_t FULL = (1ull << KEYS) - 1;
  constexpr int WAVE_LDS = KEYS * Rows::BYTES;
  constexpr int LDS = WAVE_LDS > 16 * OLD * 4 ? WAVE_LDS * NW : 16 * OLD * 4 * NW;
  __shared__ __attribute__((aligned(1024))) char smem[LDS];
  __shared__ float s_m[NW][16 * RT], s_l[NW][16 * RT];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  // row blocks of one part next to each other, on one XCD: its L2 then reads the part once
  const int id = by_blocks.d > 1 ? xcd_contiguous(blockIdx.x, gridDim.x) : (int)blockIdx.x;
  const int at = by_blocks.div(id), r0 = (id - at * (int)by_blocks.d) * 16 * RT;
  const int pr = a.by_parts.div(at), part = at - pr * a.parts;
  const int set = a.by_heads.div(pr), head = pr - set * a.d.heads_kv;
  int len;
  const int ctx = xattn_context(a, set, &len);
  const int pk = xattn_part(a, len), k0 = part * pk, k1 = min(len, k0 + pk);
  if (k0 >= k1 && a.parts > 1) return;   // the join does not read it

  // Q^T operands
  bf16x8 qf[NS][RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = min(r0 + 16 * rt + l16, a.rows - 1);
    const T* src = (const T*)a.q + set * a.d.q_b + xattn_row(a, r, head, a.d.q_r, a.d.q_h);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const T* p = src + Tile::channel(ks, g);
      if constexpr (NS == 1) {
        qf[0][rt][ks] = *reinterpret_cast<const bf16x8*>(p);
      } else {
        float x[8];
        bf16x8 t[NS];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)p[i];
        split_bf16<NS>(x, t);
#pragma unroll
        for (int n = 0; n < NS; ++n) qf[n][rt][ks] = t[n];
      }
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

  lds_char* const rows = (lds_char*)smem + wave * WAVE_LDS;
  Tile tile(a, ctx, head, MASK ? a.mask + ctx * a.d.mask_b : nullptr, k1, lane);
  const int first = k0 + wave * KEYS, step = NW * KEYS;
  if (first < k1) tile.request(first);
  for (int kv0 = first; kv0 < k1; kv0 += step) {
    // scores, and the values into LDS: the tile's registers are then free for the next
    const uint64_t bits = tile.bits;
    f32x4 sc[2][RT];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      bf16x8 kf[KS];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[ks] = tile.key(t, ks);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int n = NS - 1; n >= 0; --n)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) acc = mma16(kf[ks], qf[n][rt][ks], acc);
        sc[t][rt] = acc;
      }
    }
    const bool some = bits != FULL;
    tile.stage(rows, bits, some);
    if (kv0 + step < k1) tile.request(kv0 + step);
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
      // a row's maximum moves only when it must (weights up to 2^8 lose nothing in fp32), and
      // by the row's own scores alone: a query's output does not depend on the others
      const bool moves = mx > m_run[rt] + 8.0f;
      if (__any(moves)) {
        const float m_new = moves ? mx : m_run[rt];
        // nothing seen yet: the sums are zero whatever the factor, which must not be NaN
        const float alpha = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[rt] - m_new);
        m_run[rt] = m_new;
        l_run[rt] *= alpha;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) o[rt][ct] *= alpha;
      }
      const float m_use = m_run[rt] == -INFINITY ? 0.0f : m_run[rt];
      float p[8], lsum = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i / 4][rt][i % 4], a.scale_log2, -m_use));
      // terms of the weights, which are summed as rounded
      const bf16x2 one = {(bf16)1.0f, (bf16)1.0f};
      bf16x8 t[NS];
      split_bf16<NS>(p, t);
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        pf[n][rt] = t[n];
#pragma unroll
        for (int i = 0; i < 8; i += 2) lsum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{t[n][i], t[n][i + 1]}, one, lsum, false);
      }
      l_run[rt] += lsum;
    }
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct) {
      const bf16x8 vf = Rows::operand(rows, lane, ct);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int n = NS - 1; n >= 0; --n) o[rt][ct] = mma16(vf, pf[n][rt], o[rt][ct]);
    }
  }

  // join the waves: maxima and sums, then the outputs of one row tile at a time
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = sum_groups16(l_run[rt]);
    if (g == 0) {
      s_m[wave][16 * rt + l16] = m_run[rt];
      s_l[wave][16 * rt + l16] = l;
    }
  }
  float(*s_o)[16 * OLD] = reinterpret_cast<float(*)[16 * OLD]>(smem);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (r0 + 16 * rt >= a.rows) break;
    __syncthreads();   // stages and the previous row tile are read
    float m_all = s_m[0][16 * rt + l16];
#pragma unroll
    for (int w = 1; w < NW; ++w) m_all = fmaxf(m_all, s_m[w][16 * rt + l16]);
    const float m_use = m_all == -INFINITY ? 0.0f : m_all;
    const float f = __builtin_amdgcn_exp2f(m_run[rt] - m_use);
#pragma unroll
    for (int ct = 0; ct < NCT; ++ct)
      *reinterpret_cast<f32x4*>(&s_o[wave][l16 * OLD + 16 * ct + 4 * g]) = o[rt][ct] * f;
    __syncthreads();
    for (int i = tid; i < 16 * DH / 4; i += 64 * NW) {
      const int q = i / (DH / 4), c = 4 * (i % (DH / 4)), tr = 16 * rt + q, r = r0 + tr;
      if (r >= a.rows) break;
      float m = s_m[0][tr], l = 0.0f;
#pragma unroll
      for (int w = 1; w < NW; ++w) m = fmaxf(m, s_m[w][tr]);
      const float mu = m == -INFINITY ? 0.0f : m;
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        v += *reinterpret_cast<const f32x4*>(&s_o[w][q * OLD + c]);
        l = fmaf(s_l[w][tr], __builtin_amdgcn_exp2f(s_m[w][tr] - mu), l);
      }
      if (a.parts > 1) {
        const long at = ((long)pr * a.parts + part) * a.rows + r;
        *reinterpret_cast<f32x4*>(a.part_o + at * DH + c) = v;
        if (c == 0) a.part_ml[at] = make_float2(m, l);
      } else {
        T* dst = (T*)a.o + set * a.d.o_b + xattn_row(a, r, head, a.d.o_r, a.d.o_h) + c;
        const float inv = l != 0.0f ? 1.0f / l : 0.0f;
        typedef T out4 __attribute__((ext_vector_type(4)));
        out4 y;
#pragma unroll
        for (int x = 0; x < 4; ++x) y[x] = to_t<T>(v[x] * inv);
        *reinterpret_cast<out4*>(dst) = y;
      }
    }
  }
}

// Blocks of 16 RT rows.
template <typename T, int DH, int RT, bool MASK, bool KV4> static hipError_t launch_rt(const XAttnArgs& a, hipStream_t st) {
  constexpr int NS = sizeof(T) == 2 ? 1 : 3;
  const FastDiv by_blocks(cdiv(a.rows, 16 * RT));
  const dim3 grid((unsigned)((long)a.d.n_q * a.d.heads_kv * a.parts * by_blocks.d)), block(256);
  if constexpr (KV4)
    hipLaunchKernelGGL((k_xattn_rows<T, DH, RT, NS, MASK, TileKv4<DH, MASK>>), grid, block, 0, st, a, by_blocks);
  else
    hipLaunchKernelGGL((k_xattn_rows<T, DH, RT, NS, MASK, TileBf16<DH, MASK>>), grid, block, 0, st, a, by_blocks);
  return hipGetLastError();
}

// One row tile where 16 hold all rows, two else: a third and fourth do not fit the
// registers of two waves a SIMD (64 rows over 16 4-bit contexts of 32,768 rows take 17% longer as
// one block of four tiles than as two blocks of two).
template <typename T, int DH, bool MASK, bool KV4> static hipError_t launch(const XAttnArgs& a, hipStream_t st) {
  return a.rows <= 16 ? launch_rt<T, DH, 1, MASK, KV4>(a, st) : launch_rt<T, DH, 2, MASK, KV4>(a, st);
}

template <typename T, int DH> static hipError_t launch_dh(const XAttnArgs& a, bool kv4, hipStream_t st) {
  if (kv4) return a.mask ? launch<T, DH, true, true>(a, st) : launch<T, DH, false, true>(a, st);
  if constexpr (sizeof(T) == 2)
    return a.mask ? launch<T, DH, true, false>(a, st) : launch<T, DH, false, false>(a, st);
  else
    return hipErrorInvalidValue;
}

template <typename T> hipError_t xattn_rows(const XAttnArgs& a, bool kv4, hipStream_t st) {
  switch (a.d.head_dim) {
    case 128: return launch_dh<T, 128>(a, kv4, st);
    case 64: return launch_dh<T, 64>(a, kv4, st);
    case 32: return launch_dh<T, 32>(a, kv4, st);
    default: return hipErrorInvalidValue;
  }
}
template hipError_t xattn_rows<bf16>(const XAttnArgs&, bool, hipStream_t);
template hipError_t xattn_rows<float>(const XAttnArgs&, bool, hipStream_t);

}  // namespace cs
