// Rows to 8-bit codes with a scale each, and back (cs_i8_quantise, cs_i8_dequantise), and the
// layout of 8-bit weights (cs_i8_weight_pack).  Bound by memory: 32,760 x 8960 in bf16 take 151
// us (5.8 TB/s) and 144 back (6.1); 32,760 x 5120 77 (6.6) and 72 (7.0).
#include "gemm_kernel.hpp"
#include "ops.hpp"
#include "row_tile.hpp"

namespace cs {

template <typename X, int U, int WPR, int NV, bool TAIL, bool FAR>
__global__ __launch_bounds__(WPR == 16 ? 1024 : 256) void k_i8_quantise(I8RowsArgs a) {
  __shared__ uint32_t lds[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long row = WPR == 1 ? (long)blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= a.d.rows) return;
  const int dim = a.d.dim, t = WPR == 1 ? lane : (int)threadIdx.x;
  const X* x = (const X*)a.x + row * a.d.x_row;
  typename Chunk<X, U>::vec raw[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = U * (64 * WPR * i + t);
    raw[i] = load_chunk<X, U, TAIL, FAR>(x + c, dim - c);
  }
  std::conditional_t<sizeof(X) == 2, u16x2, uint32_t> m = {};
#pragma unroll
  for (int i = 0; i < NV; ++i) max_bits(m, raw[i]);
  const I8Scale s(row_max<WPR>(fp32_bits(m), lds, wave));
  if (t == 0) a.scales[row] = s.scale;
  store_codes<U, NV, WPR, TAIL, sizeof(X) == 2>(s, a.codes + row * a.d.q_row, dim, t,
                                                [&](int i, int e) { return to_f(raw[i][e]); });
}

// WPR: waves of a row (1 or 4).
template <typename X, int U, int WPR, bool TAIL, bool FAR>
__global__ __launch_bounds__(256) void k_i8_dequantise(I8RowsArgs a) {
  const int t = WPR == 1 ? threadIdx.x & 63 : threadIdx.x;
  const long row = WPR == 1 ? (long)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.d.rows) return;
  const float scale = a.scales[row];
  const int8_t* q = a.codes + row * a.d.q_row;
  X* x = (X*)a.x_out + row * a.d.x_row;
  for (int c = U * t; c < a.d.dim; c += 64 * WPR * U) {
    const auto v = load_chunk<int8_t, U, TAIL>(q + c, a.d.dim - c);
    float y[U];
#pragma unroll
    for (int e = 0; e < U; ++e) y[e] = scale * (float)v[e];
    store_chunk<X, U, TAIL, FAR>(x + c, a.d.dim - c, y);
  }
}

template <typename X> static hipError_t quantise(const I8RowsArgs& a, hipStream_t st) {
  constexpr int U = sizeof(X) == 2 ? 8 : 4;
  const bool far = past_caches((double)a.d.rows * a.d.dim * (sizeof(X) + 1));
  // A workgroup of 16 waves to a row, one shape for all lengths.  In fp32 its 16 chunks spill: 8,000 x
  // 16,385 take 1221 us, x 16,384 (4 waves) 110; in bf16 8,000 x 20,000 231.
  if (a.d.dim > 16384) {
    if (const hipError_t s = check_grid(a.d.rows, 1024); s != hipSuccess) return s;
    const auto kernel = far ? k_i8_quantise<X, U, 16, 64 / U, true, true> : k_i8_quantise<X, U, 16, 64 / U, true, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)a.d.rows), dim3(1024), 0, st, a);
    return hipGetLastError();
  }
  return with_row_shape<U>(a.d.dim, [&](auto shape) {
    typedef decltype(shape) S;
    const long grid = S::WPR == 1 ? ((long)a.d.rows + 3) / 4 : a.d.rows;
    if (const hipError_t s = check_grid(grid, 256); s != hipSuccess) return s;
    const auto kernel = far ? k_i8_quantise<X, U, S::WPR, S::NV, S::TAIL, true>
                            : k_i8_quantise<X, U, S::WPR, S::NV, S::TAIL, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t i8_quantise(const I8RowsArgs& a, hipStream_t st) {
  return a.d.dtype == CS_BF16 ? quantise<bf16>(a, st) : quantise<float>(a, st);
}

template <typename X> static hipError_t dequantise(const I8RowsArgs& a, hipStream_t st) {
  constexpr int U = sizeof(X) == 2 ? 8 : 4;
  const bool tail = a.d.dim % U != 0, wide = a.d.dim > 2048;
  const bool far = past_caches((double)a.d.rows * a.d.dim * (sizeof(X) + 1));
  auto pick = [&](auto t, auto f) {
    constexpr bool T = decltype(t)::value, F = decltype(f)::value;
    return wide ? k_i8_dequantise<X, U, 4, T, F> : k_i8_dequantise<X, U, 1, T, F>;
  };
  typedef std::true_type Y;
  typedef std::false_type N;
  const auto kernel = tail ? (far ? pick(Y{}, Y{}) : pick(Y{}, N{})) : (far ? pick(N{}, Y{}) : pick(N{}, N{}));
  const long grid = wide ? a.d.rows : ((long)a.d.rows + 3) / 4;
  if (const hipError_t s = check_grid(grid, 256); s != hipSuccess) return s;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t i8_dequantise(const I8RowsArgs& a, hipStream_t st) {
  return a.d.dtype == CS_BF16 ? dequantise<bf16>(a, st) : dequantise<float>(a, st);
}

// -------------------------------------------------------------- 8-bit weights
// The layout of gemm_tile_weight with 128 codes to a row of a block; rows past n and columns
// past k are zero.  A wave per row of the padded matrix.  W int8_t: codes and scales given.
template <typename W>
__global__ __launch_bounds__(256) void k_i8_weight(const W* __restrict__ w, long w_row, const float* __restrict__ given,
                                                   int n, int k, int rows, int8_t* __restrict__ codes,
                                                   float* __restrict__ scales) {
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (row >= rows) return;
  const bool real = row < n;
  const W* src = w + (real ? row * w_row : 0);
  const int nk = (k + 127) / 128;
  int8_t* dst = codes + ((long)(row / W_BLOCK_ROWS) * nk * W_BLOCK_ROWS + row % W_BLOCK_ROWS) * 128;
  uint32_t m = 0;
  if constexpr (sizeof(W) > 1) {
    if (real)
      for (int c = lane; c < k; c += 64) m = max(m, abs_bits(to_f(src[c])));
    m = row_max<1>(m, nullptr, 0);
  }
  const I8Scale s(m);
  if (real && lane == 0) {
    if constexpr (sizeof(W) > 1) scales[row] = s.scale;
    else scales[row] = given[row];
  }
  for (int q = lane; q < nk * 8; q += 64) {
    const int kt = q >> 3, chunk = q & 7;
    union { int8_t b[16]; uint4 v; } o;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int c = kt * 128 + chunk * 16 + e;
      o.b[e] = 0;
      if (real && c < k) {
        if constexpr (sizeof(W) > 1) o.b[e] = (int8_t)(int)s.code(to_f(src[c]));
        else o.b[e] = src[c];
      }
    }
    *reinterpret_cast<uint4*>(dst + (long)kt * W_BLOCK_ROWS * 128 + (chunk ^ gemm_swz(row)) * 16) = o.v;
  }
}

long i8_weight_bytes(int n, int k) { return round_up(n, W_BLOCK_ROWS) * round_up(k, 128); }

hipError_t i8_weight_pack(const cs_i8_weight& o, int dtype, const void* w, long w_row, const float* given,
                          hipStream_t st) {
  const int rows = (int)round_up(o.n, W_BLOCK_ROWS);
  const dim3 grid((unsigned)(rows / 4)), block(256);
  if (dtype == CS_BF16)
    hipLaunchKernelGGL(k_i8_weight<bf16>, grid, block, 0, st, (const bf16*)w, w_row, given, o.n, o.k, rows, o.codes, o.scales);
  else if (dtype == CS_FP32)
    hipLaunchKernelGGL(k_i8_weight<float>, grid, block, 0, st, (const float*)w, w_row, given, o.n, o.k, rows, o.codes, o.scales);
  else
    hipLaunchKernelGGL(k_i8_weight<int8_t>, grid, block, 0, st, (const int8_t*)w, w_row, given, o.n, o.k, rows, o.codes, o.scales);
  return hipGetLastError();
}

}  // namespace cs
