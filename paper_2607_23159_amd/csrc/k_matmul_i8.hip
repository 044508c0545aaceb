// Product of 8-bit rows and 8-bit weights with a scale for each row and output channel
// (cs_matmul_i8).  Sums are 32-bit integers and exact, so every kernel and tile shape gives
// bitwise the same results.
//
// The kernels are those of the other types: a 16-byte chunk holds 16 codes where it holds 8 bf16, and
// v_mfma_i32_16x16x64_i8 takes it in the cycles of v_mfma_f32_16x16x32_bf16, so a K slice of 128 bytes is
// 128 deep and the loads, LDS reads and products of a slice stay as they are.  32,760 x 13,824 x
// 5120 with the GELU: 1.77 to 1.89 ms (machines differ), 2.45 to 2.61 P operations/s at 1.93 GHz with the matrix pipe busy
// 64% of the cycles (bf16: 1.3 P); 12,480 x 1536 x 8960 140 to 155 us, 57% busy.
#include "gemm_kernel.hpp"
#include "gemm_tile.hpp"
#include "ops.hpp"

namespace cs {

constexpr int GROUP_M = 4;

// Few rows: the weights are all there is to read, once, so they go straight from memory to the
// operand registers.  A workgroup has 16 columns; its 8 waves take the K slices in turn, 4 each in
// flight, and add their sums up in LDS.  Rows past M repeat the last one, and bytes past the end of a
// row its last ones, which meet zeros of W.  Bound by latency: 1 x 1536 x 8960, 13.8 MB of weights from
// HBM, takes 6.0 us, of which 2.5 are those of an empty launch.  4 or 16 waves are within 10% of it, 32 columns a
// workgroup 40% slower.
template <class To>
__global__ __launch_bounds__(512) void k_matmul_few(const int8_t* __restrict__ a, long a_row,
                                                    const int8_t* __restrict__ w, int M, int N, int nk,
                                                    EpiI8<To> epi) {
  constexpr int U = 4, NW = 8, SLICE = W_BLOCK_ROWS * 128;   // SLICE: bytes from one slice to the next
  __shared__ i32x4 sums[NW][64];
  const int lane = threadIdx.x & 63, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16;
  const int8_t* wp = w + ((long)(n0 / W_BLOCK_ROWS) * nk * W_BLOCK_ROWS + n0 % W_BLOCK_ROWS + (lane & 15)) * 128;
  const int swz = gemm_swz(lane & 15), last = epi.a_row - 16;
  const int8_t* ap = a + min(lane & 15, M - 1) * a_row;
  i32x4 acc = {0, 0, 0, 0};
  for (int k0 = wave; k0 < nk; k0 += U * NW) {
    i32x4 wv[U][2], av[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kt = k0 + u * NW;
      if (kt >= nk) break;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        wv[u][s] = *reinterpret_cast<const i32x4*>(wp + (long)kt * SLICE + ((4 * s + quad) ^ swz) * 16);
        av[u][s] = *reinterpret_cast<const i32x4*>(ap + min(kt * 128 + s * 64 + quad * 16, last));
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u * NW >= nk) break;
#pragma unroll
      for (int s = 0; s < 2; ++s) acc = Mfma16<int8_t>::mma(wv[u][s], av[u][s], acc);
    }
  }
  sums[wave][lane] = acc;
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int i = 1; i < NW; ++i) acc += sums[i][lane];
  const int row = lane & 15, col0 = n0 + 4 * quad;
  if (row >= M || col0 >= N) return;
  const float sa = epi.scale_a[row];
  const f32x4 sw = epi.four(epi.scale_w, col0, N), b = epi.bias ? epi.four(epi.bias, col0, N) : f32x4{0.f, 0.f, 0.f, 0.f};
  float y[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = i8_value(acc[r], sa, sw[r], b[r]);
  epi.to(row, col0, y, epi.to.pre(row, col0));
}

template <class To> static void launch_few(const MatmulI8Args& a, int kp, const EpiI8<To>& epi, hipStream_t st) {
  hipLaunchKernelGGL(k_matmul_few<To>, dim3((unsigned)cdiv(a.d.n, 16)), dim3(512), 0, st, a.a, a.d.a_row, a.w.codes,
                     a.d.rows, a.d.n, kp / 128, epi);
}

template <int BM, int BN, int OCC, int PD, class Epi>
static hipError_t launch_w4(const MatmulI8Args& a, int kp, const Epi& epi, hipStream_t st) {
  const long tiles = (long)cdiv(a.d.rows, BM) * cdiv(a.d.n, BN);
  if (const hipError_t s = check_grid(tiles, 256); s != hipSuccess) return s;
  hipLaunchKernelGGL((k_gemm_w4<int8_t, BM, BN, OCC, GROUP_M, PD, Epi>), dim3((unsigned)tiles), dim3(256), 0, st, a.a,
                     a.d.a_row, a.w.codes, a.d.rows, a.d.n, kp, 0L, epi);
  return hipGetLastError();
}

template <int BM, int BN, int WGM, int WGN, int SL, int STAGES, int OCC, class Epi>
static hipError_t launch_ring(const MatmulI8Args& a, int kp, const Epi& epi, hipStream_t st, int parts = 1) {
  constexpr int THREADS = 64 * WGM * WGN;
  const long tiles = (long)cdiv(a.d.rows, BM) * cdiv(a.d.n, BN);
  if (const hipError_t s = check_grid(tiles * parts, THREADS); s != hipSuccess) return s;
  hipLaunchKernelGGL((k_gemm_ring<int8_t, BM, BN, WGM, WGN, SL, STAGES, OCC, GROUP_M, Epi>),
                     dim3((unsigned)tiles, (unsigned)parts), dim3(THREADS), 0, st, a.a, a.d.a_row, a.w.codes, a.d.rows, a.d.n,
                     kp, 0L, epi);
  return hipGetLastError();
}

template <class To> static hipError_t product(const MatmulI8Args& a, const To& to, hipStream_t st) {
  const EpiI8<To> epi = {a.a_scale, a.w.scales, a.bias, (int)round_up(a.d.k, 16), to};
  const int kp = (int)round_up(a.d.k, 128);
  constexpr bool RES = EpiIsResidual<To>::value;
  constexpr int PD = RES ? 8 : 2, PD2 = RES ? 4 : 2;   // as in bf16
  if (a.d.rows <= FEW_ROWS && a.d.n <= FEW_COLS) {
    launch_few(a, kp, epi, st);
    return hipGetLastError();
  }
  auto launch = [&](Bf16Tile tile) {
    switch (tile) {
      case W4_256x256: return launch_w4<256, 256, 1, PD>(a, kp, epi, st);
      case W4_224x256: return launch_w4<224, 256, 1, PD>(a, kp, epi, st);
      case W4_192x256: return launch_w4<192, 256, 1, PD>(a, kp, epi, st);
      case W4_160x256: return launch_w4<160, 256, 1, PD>(a, kp, epi, st);
      case W4_128x128: return launch_w4<128, 128, 2, PD2>(a, kp, epi, st);
      case W4_64x64: return launch_w4<64, 64, 3, 2>(a, kp, epi, st);
      case RING_128x128: return launch_ring<128, 128, 2, 4, 1, 4, 2>(a, kp, epi, st);
      case RING_64x128: return launch_ring<64, 128, 2, 4, 2, 3, 2>(a, kp, epi, st);
      case RING_64x64: return launch_ring<64, 64, 2, 4, 2, 4, 2>(a, kp, epi, st);
      case RING_32x64: return launch_ring<32, 64, 1, 4, 2, 3, 2>(a, kp, epi, st);
      default: return launch_ring<32, 32, 2, 2, 2, 4, 2>(a, kp, epi, st);
    }
  };
  const hipError_t s = launch(choose_tile_i8(a.d.rows, a.d.n, a.d.k, RES));
  // more tiles than a launch has: the largest are the fewest
  return s == hipErrorInvalidConfiguration ? launch(W4_256x256) : s;
}

// ------------------------------------------------------------- parts of K
// The parts' sums, scaled: four columns a thread.
template <class To>
__global__ __launch_bounds__(256) void k_matmul_join(const int* __restrict__ part, long ld, long stride, int parts, int M,
                                                     int N, EpiI8<To> epi) {
  const int cols = (N + 3) / 4, q = blockIdx.x * 256 + threadIdx.x, row = q / cols, col0 = 4 * (q - row * cols);
  if (row >= M) return;
  const int* p = part + (long)row * ld + col0;
  i32x4 v = *reinterpret_cast<const i32x4*>(p);
#pragma unroll 4
  for (int i = 1; i < parts; ++i) v += *reinterpret_cast<const i32x4*>(p + i * stride);
  const float sa = epi.scale_a[row];
  const f32x4 sw = epi.four(epi.scale_w, col0, N), b = epi.bias ? epi.four(epi.bias, col0, N) : f32x4{0.f, 0.f, 0.f, 0.f};
  float y[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) y[r] = i8_value(v[r], sa, sw[r], b[r]);
  epi.to(row, col0, y, epi.to.pre(row, col0));
}

static size_t part_bytes(const cs_matmul_i8_desc& d) { return (size_t)d.rows * round_up(d.n, 4) * sizeof(int); }

size_t matmul_i8_workspace(const cs_matmul_i8_desc& d) {
  const int parts = split_k_i8(d.rows, d.n, d.k).parts;
  return parts > 1 ? parts * part_bytes(d) : 0;
}

template <class To> static hipError_t product_of_parts(const MatmulI8Args& a, const To& to, int* part, hipStream_t st) {
  const SplitK s = split_k_i8(a.d.rows, a.d.n, a.d.k);
  if (s.parts == 1) return product(a, to, st);
  const long ld = round_up(a.d.n, 4), stride = a.d.rows * ld;
  const int kp = (int)round_up(a.d.k, 128), a_row = (int)round_up(a.d.k, 16);
  const EpiSums sums = {part, ld, stride, s.per, a_row};
  auto launch = [&] {
    switch (s.tile) {
      case RING_64x128: return launch_ring<64, 128, 2, 4, 2, 3, 2>(a, kp, sums, st, s.parts);
      case RING_64x64: return launch_ring<64, 64, 2, 4, 2, 4, 2>(a, kp, sums, st, s.parts);
      case RING_32x64: return launch_ring<32, 64, 1, 4, 2, 3, 2>(a, kp, sums, st, s.parts);
      default: return launch_ring<32, 32, 2, 2, 2, 4, 2>(a, kp, sums, st, s.parts);
    }
  };
  const hipError_t e = launch();
  if (e != hipSuccess) return e;
  const EpiI8<To> epi = {a.a_scale, a.w.scales, a.bias, a_row, to};
  hipLaunchKernelGGL(k_matmul_join<To>, dim3((unsigned)cdiv(a.d.rows * (ld / 4), 256)), dim3(256), 0, st, part, ld, stride,
                     s.parts, a.d.rows, a.d.n, epi);
  return hipGetLastError();
}

hipError_t matmul_i8(const MatmulI8Args& a, void* work, hipStream_t st) {
  int* part = (int*)work;
  if (a.d.out_dtype == CS_BF16)
    return a.d.act == CS_ACT_GELU ? product_of_parts(a, EpiMatmul<bf16, 1>{(bf16*)a.out, a.d.o_row, a.d.n}, part, st)
                                  : product_of_parts(a, EpiMatmul<bf16, 0>{(bf16*)a.out, a.d.o_row, a.d.n}, part, st);
  return a.d.act == CS_ACT_GELU ? product_of_parts(a, EpiMatmul<float, 1>{(float*)a.out, a.d.o_row, a.d.n}, part, st)
                                : product_of_parts(a, EpiMatmul<float, 0>{(float*)a.out, a.d.o_row, a.d.n}, part, st);
}

// ------------------------------------------------- the transformer's projections
static MatmulI8Args projection(const I8Rows& a, const I8Weight& w, int M, int N, int K, const float* bias) {
  MatmulI8Args m = {};
  m.a = a.codes;
  m.a_scale = a.scales;
  m.bias = bias;
  m.w = {const_cast<int8_t*>(w.codes), const_cast<float*>(w.scales), N, K};
  m.d.rows = M;
  m.d.n = N;
  m.d.k = K;
  m.d.a_row = K;   // K is a multiple of 64
  return m;
}

hipError_t gemm_store_i8(const I8Rows& a, const I8Weight& w, int M, int N, int K, const float* bias, int act,
                         bf16* out, hipStream_t st) {
  const MatmulI8Args m = projection(a, w, M, N, K, bias);
  return act == 1 ? product(m, EpiMatmul<bf16, 1>{out, N, N}, st) : product(m, EpiMatmul<bf16, 0>{out, N, N}, st);
}

hipError_t gemm_qkv_i8(const I8Rows& a, const I8Weight& w, int M, int d, const float* bias, int L, bf16* qk, bf16* vt,
                       long vt_ld, hipStream_t st) {
  return product(projection(a, w, M, 3 * d, d, bias), EpiQKV<bf16>{qk, vt, nullptr, d, L, vt_ld, (long)d * vt_ld}, st);
}

hipError_t gemm_residual_i8(const I8Rows& a, const I8Weight& w, int M, int N, int K, const float* bias,
                            const float* gate, float* z, bf16* y, hipStream_t st) {
  const MatmulI8Args m = projection(a, w, M, N, K, bias);
  if (y)
    return gate ? product(m, EpiResidualStore<1, bf16>{z, N, nullptr, gate, y}, st)
                : product(m, EpiResidualStore<0, bf16>{z, N, nullptr, nullptr, y}, st);
  return gate ? product(m, EpiResidual<1>{z, N, nullptr, gate}, st)
              : product(m, EpiResidual<0>{z, N, nullptr, nullptr}, st);
}

}  // namespace cs
