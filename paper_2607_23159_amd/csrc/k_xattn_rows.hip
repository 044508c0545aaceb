// Attention of few queries (a token or a handful, with the heads that share a key
// head: at most 64 rows) to a context: keys and values are read once, from memory.
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
#include "ops.hpp"

namespace cs {

CS_DEV f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Maximum / sum over lanes l, l ^ 16, l ^ 32, l ^ 48.
CS_DEV float max_groups16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_lane_pair32(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
CS_DEV float sum_groups16(float x) {
  x += __shfl_xor(x, 16, WAVE);
  return x + __shfl_xor(x, 32, WAVE);
}

// x as a sum of NS bf16 terms, the largest first (three hold all 24 bits).
template <int NS> CS_DEV void split_bf16(float x, bf16* t) {
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    t[i] = (bf16)x;
    x -= (float)t[i];
  }
}

typedef __attribute__((address_space(3))) bf16x8 lds_vec8;

// Keys of a tile (bit i: key kv0 + i) that are left: below k1 and not masked.
template <int KEYS, bool MASK>
CS_DEV uint64_t tile_bits(const uint8_t* mask, int kv0, int k1, int lane) {
  if constexpr (MASK) {
    const int key = kv0 + lane;
    return __ballot(lane < KEYS && key < k1 && mask[min(key, k1 - 1)] != 0);
  } else {
    const int n = min(KEYS, k1 - kv0);
    return n == 64 ? ~0ull : (1ull << n) - 1;
  }
}

// V^T operand of 16 channels ct over 32 rows of VRS bytes in LDS.
template <int VRS> CS_DEV bf16x8 read_values(const lds_char* rows, int lane, int ct) {
  const lds_char* p = rows + (4 * (lane >> 4) + ((lane & 15) >> 2)) * VRS + ct * 32 + (lane & 3) * 8;
  const bf16x4 x = lds_read_tr(p), y = lds_read_tr(p + 16 * VRS);
  return bf16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

// Key tile of 32 keys in bf16: fragments straight from memory, the values through a
// ring of two LDS stages filled by direct loads.
template <int DH, bool MASK> struct TileBf16 {
  static constexpr int H = 1, KEYS = 32 * H, KS = DH / 32, VRS = 2 * DH + 32;   // padded rows: conflict-free reads
  static constexpr int LDS = 2 * KEYS * VRS;                         // bytes per wave
  static constexpr int CV = VRS / 16, V_INST = KEYS * CV / 64;
  static_assert(V_INST * 64 == KEYS * CV, "whole 1 KB loads");
  const bf16 *k, *v;
  long k_r, v_r;
  const uint8_t* mask;
  int k1, lane;
  lds_char* lds;
  bf16x8 kf[2][KS];
  int voff[V_INST];
  uint64_t bits_next;   // keys of the requested tile that are left

  CS_DEV TileBf16(const XAttnArgs& a, int ctx, int head, const uint8_t* mask_, int k1_, int lane_, lds_char* lds_)
      : k((const bf16*)a.k + ctx * a.d.k_b + head * a.d.k_h), v((const bf16*)a.v + ctx * a.d.v_b + head * a.d.v_h),
        k_r(a.d.k_r), v_r(a.d.v_r), mask(mask_), k1(k1_), lane(lane_), lds(lds_) {
#pragma unroll
    for (int i = 0; i < V_INST; ++i) {
      const int p = i * 64 + lane, row = p / CV, ch = p % CV;
      // the padding slots' offset lies past every range: they load nothing
      voff[i] = ch < DH / 8 ? (row * (int)v_r + ch * 8) * 2 : 0x7FFFFFF0;
    }
  }
  // channel of element i of step ks in lane group g
  static CS_DEV int channel(int ks, int g) { return 32 * ks + 8 * g; }
  CS_DEV void request(int kv0, int stage) {
    bits_next = tile_bits<KEYS, MASK>(mask, kv0, k1, lane);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const bf16* src = k + min(kv0 + 16 * kt + (lane & 15), k1 - 1) * k_r + 8 * (lane >> 4);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[kt][ks] = *reinterpret_cast<const bf16x8*>(src + 32 * ks);
    }
    const bf16* base = v + kv0 * v_r;
    const int bytes = ((min(KEYS, k1 - kv0) - 1) * (int)v_r + DH) * 2;
#pragma unroll
    for (int i = 0; i < V_INST; ++i) {
      int off = voff[i];
      if constexpr (MASK) {   // rows that the mask leaves out load as zeros: they may hold NaN
        if (!(bits_next >> ((i * 64 + lane) / CV) & 1)) off = 0x7FFFFFF0;
      }
      load_lds16(base, bytes, lds + stage * KEYS * VRS + i * 1024, off);
    }
  }
  // the requested tile is there: everything in flight was asked for one round ago
  CS_DEV void land(int) { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
  CS_DEV bf16x8 key(int kt, int ks) const { return kf[kt][ks]; }
  // V^T operand of 16 channels ct over 32 keys
  CS_DEV bf16x8 values(int stage, int, int ct) const { return read_values<VRS>(lds + stage * KEYS * VRS, lane, ct); }
};

// The same of a 4-bit cache.  A lane reads a quarter of a key's codes, which lie
// together and (from head dim 64 on) under one scale byte; the score product visits
// the channels in that order.  Values are decoded on their way into LDS.
template <int DH, bool MASK> struct TileKv4 {
  static constexpr int H = 2, KEYS = 32 * H, KT = 2 * H, KS = DH / 32, VRS = 2 * DH + 32;
  static constexpr int LDS = KEYS * VRS;
  const uint8_t *kc, *ks_, *vc, *vs_;
  const uint8_t* mask;
  int k1, lane;
  lds_char* lds;
  uint32_t k[KT][KS], v[KT][KS];
  uint32_t kb[KT], vb[KT];
  uint64_t bits_next;

  CS_DEV TileKv4(const XAttnArgs& a, int ctx, int head, const uint8_t* mask_, int k1_, int lane_, lds_char* lds_)
      : mask(mask_), k1(k1_), lane(lane_), lds(lds_) {
    const long at = ((long)ctx * a.c.heads + head) * a.c.cap;
    kc = a.c.k_codes + at * (DH / 2);
    vc = a.c.v_codes + at * (DH / 2);
    ks_ = a.c.k_scales + at * (DH / 32);
    vs_ = a.c.v_scales + at * (DH / 32);
  }
  static CS_DEV int channel(int ks, int g) { return DH / 4 * g + 8 * ks; }
  static CS_DEV void fetch(const uint8_t* p, uint32_t* d) {
    if constexpr (KS == 4) {
      const uint4 x = *reinterpret_cast<const uint4*>(p);
      d[0] = x.x; d[1] = x.y; d[2] = x.z; d[3] = x.w;
    } else if constexpr (KS == 2) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      d[0] = x.x; d[1] = x.y;
    } else {
      d[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  }
  CS_DEV void request(int kv0, int) {
    const int g = lane >> 4;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const long key = min(kv0 + 16 * kt + (lane & 15), k1 - 1);
      fetch(kc + key * (DH / 2) + g * (DH / 8), k[kt]);
      fetch(vc + key * (DH / 2) + g * (DH / 8), v[kt]);
      kb[kt] = ks_[key * (DH / 32) + g * DH / 128];
      vb[kt] = vs_[key * (DH / 32) + g * DH / 128];
    }
    bits_next = tile_bits<KEYS, MASK>(mask, kv0, k1, lane);
  }
  CS_DEV void land(int) {
    const uint64_t bits = bits_next;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      // rows that are left out may hold anything: they become zeros
      const bool left = bits >> (16 * kt + (lane & 15)) & 1;
      const float s = kv4_scale(left ? vb[kt] : 127);
      lds_char* p = lds + (16 * kt + (lane & 15)) * VRS + (lane >> 4) * (DH / 2);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
        *(lds_vec8*)(p + 16 * ks) = kv4_decode8(left ? v[kt][ks] : 0, s);
    }
  }
  CS_DEV bf16x8 key(int kt, int ks) const { return kv4_decode8(k[kt][ks], kv4_scale(kb[kt])); }
  CS_DEV bf16x8 values(int, int half, int ct) const { return read_values<VRS>(lds + half * 32 * VRS, lane, ct); }
};

// NS: bf16 terms of a query and of a softmax weight (1: bf16; 3: fp32).
template <typename T, int DH, int RT, int NS, bool MASK, typename Tile>
__global__ __launch_bounds__(256, RT > 2 || NS > 1 ? 1 : 2) void k_xattn_rows(XAttnArgs a) {
  constexpr int NW = 4, KS = DH / 32, NCT = DH / 16, OLD = DH + 4, H = Tile::H;
  constexpr uint64_t FULL = Tile::KEYS == 64 ? ~0ull : (1ull << Tile::KEYS) - 1;
  constexpr int LDS = Tile::LDS * NW > NW * 16 * OLD * 4 ? Tile::LDS * NW : NW * 16 * OLD * 4;
  __shared__ __attribute__((aligned(1024))) char smem[LDS];
  __shared__ float s_m[NW][16 * RT], s_l[NW][16 * RT];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int part = blockIdx.x % a.parts, pr = blockIdx.x / a.parts;
  const int set = pr / a.d.heads_kv, head = pr - set * a.d.heads_kv;
  int len;
  const int ctx = xattn_context(a, set, &len);
  const int k0 = part * a.part_keys, k1 = min(len, k0 + a.part_keys);
  if (k0 >= k1 && a.parts > 1) return;   // the join does not read it

  // Q^T operands
  bf16x8 qf[NS][RT][KS];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = min(16 * rt + l16, a.rows - 1);
    const T* src = (const T*)a.q + set * a.d.q_b + xattn_row(a, r, head, a.d.q_r, a.d.q_h);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const T* p = src + Tile::channel(ks, g);
      if constexpr (NS == 1) {
        qf[0][rt][ks] = *reinterpret_cast<const bf16x8*>(p);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          bf16 t[NS];
          split_bf16<NS>((float)p[i], t);
#pragma unroll
          for (int n = 0; n < NS; ++n) qf[n][rt][ks][i] = t[n];
        }
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

  Tile tile(a, ctx, head, MASK ? a.mask + ctx * a.d.mask_b : nullptr, k1, lane, (lds_char*)smem + wave * Tile::LDS);
  const int first = k0 + wave * Tile::KEYS, step = NW * Tile::KEYS;
  if (first < k1) tile.request(first, 0);
  int stage = 0;
  for (int kv0 = first; kv0 < k1; kv0 += step, stage ^= 1) {
    tile.land(stage);
    const uint64_t bits = tile.bits_next;
    f32x4 sc[2 * H][RT];
#pragma unroll
    for (int kt = 0; kt < 2 * H; ++kt)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int n = NS - 1; n >= 0; --n)
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) acc = mma16(tile.key(kt, ks), qf[n][rt][ks], acc);
        sc[kt][rt] = acc;
      }
    // the other stage's reads are long done; ask for the next tile under the softmax
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (kv0 + step < k1) tile.request(kv0 + step, stage ^ 1);
    if (bits != FULL) {
#pragma unroll
      for (int kt = 0; kt < 2 * H; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!(bits >> (16 * kt + 4 * g + j) & 1))
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) sc[kt][rt][j] = -INFINITY;
    }
    bf16x8 pf[NS][RT][H];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2 * H; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j) mx = fmaxf(mx, sc[kt][rt][j]);
      mx = max_groups16(mx) * a.scale_log2;
      // the maximum moves only when it must: weights up to 2^8 lose nothing in fp32
      if (__any(mx > m_run[rt] + 8.0f)) {
        const float m_new = fmaxf(m_run[rt], mx);
        // nothing seen yet: the sums are zero whatever the factor, which must not be NaN
        const float alpha = m_run[rt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[rt] - m_new);
        m_run[rt] = m_new;
        l_run[rt] *= alpha;
#pragma unroll
        for (int ct = 0; ct < NCT; ++ct) o[rt][ct] *= alpha;
      }
      const float m_use = m_run[rt] == -INFINITY ? 0.0f : m_run[rt];
      float lsum = 0.0f;
#pragma unroll
      for (int kt = 0; kt < 2 * H; ++kt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sc[kt][rt][j], a.scale_log2, -m_use));
          bf16 t[NS];
          split_bf16<NS>(p, t);
          float back = 0.0f;
#pragma unroll
          for (int n = NS - 1; n >= 0; --n) {
            pf[n][rt][kt / 2][4 * (kt & 1) + j] = t[n];
            back += (float)t[n];
          }
          lsum += back;   // summed as rounded
        }
      l_run[rt] += lsum;
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int ct = 0; ct < NCT; ++ct) {
        const bf16x8 vf = tile.values(stage, h, ct);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int n = NS - 1; n >= 0; --n) o[rt][ct] = mma16(vf, pf[n][rt][h], o[rt][ct]);
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
    if (16 * rt >= a.rows) break;
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
      const int q = i / (DH / 4), c = 4 * (i % (DH / 4)), r = 16 * rt + q;
      if (r >= a.rows) break;
      float m = s_m[0][r], l = 0.0f;
#pragma unroll
      for (int w = 1; w < NW; ++w) m = fmaxf(m, s_m[w][r]);
      const float mu = m == -INFINITY ? 0.0f : m;
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        v += *reinterpret_cast<const f32x4*>(&s_o[w][q * OLD + c]);
        l = fmaf(s_l[w][r], __builtin_amdgcn_exp2f(s_m[w][r] - mu), l);
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

// Row tiles of 16: as many as the rows need.
template <typename T, int DH, int RT, int NS, bool MASK, bool KV4> static hipError_t launch_rt(const XAttnArgs& a, hipStream_t st) {
  const long blocks = (long)a.d.n_q * a.d.heads_kv * a.parts;
  if (blocks > 0xFFFFFFL) return hipErrorInvalidConfiguration;
  if constexpr (KV4)
    hipLaunchKernelGGL((k_xattn_rows<T, DH, RT, NS, MASK, TileKv4<DH, MASK>>), dim3((unsigned)blocks), dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((k_xattn_rows<T, DH, RT, NS, MASK, TileBf16<DH, MASK>>), dim3((unsigned)blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

template <typename T, int DH, bool MASK, bool KV4> static hipError_t launch(const XAttnArgs& a, hipStream_t st) {
  constexpr int NS = sizeof(T) == 2 ? 1 : 3;
  if (a.rows <= 16) return launch_rt<T, DH, 1, NS, MASK, KV4>(a, st);
  if (a.rows <= 32) return launch_rt<T, DH, 2, NS, MASK, KV4>(a, st);
  if (a.rows <= 64) return launch_rt<T, DH, 4, NS, MASK, KV4>(a, st);
  return hipErrorInvalidValue;
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
