// Product of 8-bit rows and 8-bit weights with a scale for each row and output channel
// (cs_matmul_i8).  Sums are 32-bit integers and exact, so every kernel and tile shape gives
// bitwise the same results.
#include "gemm_kernel.hpp"
#include "ops.hpp"

namespace cs {

constexpr int GROUP_M = 4;

template <int BM, int BN, int WGM, int WGN, int SL, int STAGES, int OCC, class Epi>
static void launch_ring(const MatmulI8Args& a, int kp, const Epi& epi, hipStream_t st) {
  const unsigned tiles = (unsigned)((long)cdiv(a.d.rows, BM) * cdiv(a.d.n, BN));
  hipLaunchKernelGGL((k_gemm_ring<int8_t, BM, BN, WGM, WGN, SL, STAGES, OCC, GROUP_M, Epi>), dim3(tiles),
                     dim3(64 * WGM * WGN), 0, st, a.a, a.d.a_row, a.w.codes, a.d.rows, a.d.n, kp, 0L, epi);
}

template <class To> static hipError_t product(const MatmulI8Args& a, const To& to, hipStream_t st) {
  const EpiI8<To> epi = {a.a_scale, a.w.scales, a.bias, (int)round_up(a.d.k, 16), to};
  const int kp = (int)round_up(a.d.k, 128);
  launch_ring<64, 64, 2, 4, 2, 4, 2>(a, kp, epi, st);
  return hipGetLastError();
}

size_t matmul_i8_workspace(const cs_matmul_i8_desc&) { return 0; }

hipError_t matmul_i8(const MatmulI8Args& a, void*, hipStream_t st) {
  if (a.d.out_dtype == CS_BF16)
    return a.d.act == CS_ACT_GELU ? product(a, EpiMatmul<bf16, 1>{(bf16*)a.out, a.d.o_row, a.d.n}, st)
                                  : product(a, EpiMatmul<bf16, 0>{(bf16*)a.out, a.d.o_row, a.d.n}, st);
  return a.d.act == CS_ACT_GELU ? product(a, EpiMatmul<float, 1>{(float*)a.out, a.d.o_row, a.d.n}, st)
                                : product(a, EpiMatmul<float, 0>{(float*)a.out, a.d.o_row, a.d.n}, st);
}

}  // namespace cs
