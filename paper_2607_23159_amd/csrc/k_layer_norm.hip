// Layer norm by itself, forward and backward (cs_layer_norm, cs_layer_norm_backward), on
// rows held in registers (row_tile.hpp).  Both are bound by memory.
#include "ops.hpp"
#include "row_tile.hpp"

#include <algorithm>
#include <type_traits>

namespace cs {

// ------------------------------------------------------------------ forward
//   y = (x - mean) rstd gain + bias,  gain = weight or 1 + weight,
//   mean and variance from the row in registers, the variance of the centred values.
// Y int8_t: the result, in fp32, goes on to codes and the row's scale.
// One row to a wave or workgroup, its gains and biases asked for with it: 65,520 x 1536, fp32 to
// bf16, takes 103 us, 5.9 TB/s (110 with them asked for after the sums, from the first cache).  A loop
// over rows with the gains in registers and the next row on its way keeps fewer rows in flight: 120.
// Rows of 48 values a lane and more take theirs after the sums: registers for them would leave one or two
// waves a SIMD.  16,000 x 13,824: fp32 to fp32 364 -> 306 us, to codes 366 -> 235, bf16 to bf16 187 -> 169;
// 16,000 x 13,825 in bf16 298 -> 214.  fp32 rows to codes at lengths that end inside a chunk keep a wave a SIMD
// either way and ask early: 627 us against 660.
template <typename X, typename Y, int U, int WPR, int NV, bool TAIL, bool FAR>
__global__ __launch_bounds__(256) void k_layer_norm_op(LayerNormArgs a) {
  __shared__ float lds[2][4];
  __shared__ uint32_t lds_max[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long row = WPR == 1 ? (long)blockIdx.x * 4 + wave : blockIdx.x;
  if (row >= (long)a.d.groups * a.d.rows) return;   // whole waves, and whole workgroups at WPR 4
  const int dim = a.d.dim, t = WPR == 1 ? lane : (int)threadIdx.x;
  const X* x = (const X*)a.x + row * a.d.x_row;
  typename Chunk<X, U>::vec raw[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = U * (64 * WPR * i + t);
    raw[i] = load_chunk<X, U, TAIL, FAR>(x + c, dim - c);
  }
  const int group = (int)((uint32_t)row / (uint32_t)a.d.rows);   // rows in all are below 2^30
  const float* w = a.weight ? a.weight + group * a.d.w_group : nullptr;
  const float* b = a.bias ? a.bias + group * a.d.b_group : nullptr;
  const float one = a.d.unit_offset ? 1.0f : 0.0f;
  f32x4 wv[NV][U / 4], bv[NV][U / 4];
  auto params = [&](int i) {   // of chunk i
#pragma unroll
    for (int h = 0; h < U / 4; ++h) {
      const int c = U * (64 * WPR * i + t) + 4 * h;
      wv[i][h] = bv[i][h] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (w) wv[i][h] = load_chunk<float, 4, TAIL>(w + c, dim - c);
      if (b) bv[i][h] = load_chunk<float, 4, TAIL>(b + c, dim - c);
    }
  };
  constexpr bool LATE = U * NV >= 48 && !(TAIL && sizeof(X) == 4 && std::is_same<Y, int8_t>::value);
  if constexpr (!LATE) {
#pragma unroll
    for (int i = 0; i < NV; ++i) params(i);
  }
  float s = 0.0f, q = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < U; ++e) s += to_f(raw[i][e]);
  const float mean = row_sum<WPR>(s, lds[0], wave) / (float)dim;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int left = dim - U * (64 * WPR * i + t);
#pragma unroll
    for (int e = 0; e < U; ++e) {
      const float z = to_f(raw[i][e]) - mean;
      q += (TAIL ? e < left : left > 0) ? z * z : 0.0f;
    }
  }
  const float rstd = 1.0f / sqrtf(row_sum<WPR>(q, lds[1], wave) / (float)dim + a.d.eps);
  if (t == 0) {
    if (a.mean) a.mean[row] = mean;
    if (a.rstd) a.rstd[row] = rstd;
  }
  // the result of chunk i
  auto result = [&](int i, float* y) {
    if constexpr (LATE) params(i);
#pragma unroll
    for (int e = 0; e < U; ++e) {
      const float n = (to_f(raw[i][e]) - mean) * rstd;
      y[e] = fmaf(n, w ? one + wv[i][e / 4][e % 4] : 1.0f, bv[i][e / 4][e % 4]);
    }
  };
  if constexpr (std::is_same<Y, int8_t>::value) {
    float y[NV][U];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int left = dim - U * (64 * WPR * i + t);
      result(i, y[i]);
#pragma unroll
      for (int e = 0; e < U; ++e) m = max(m, (TAIL ? e < left : left > 0) ? abs_bits(y[i][e]) : 0u);
    }
    const I8Scale s8(row_max<WPR>(m, lds_max, wave));
    if (t == 0) a.y_scale[row] = s8.scale;
    store_codes<U, NV, WPR, TAIL, false>(s8, (int8_t*)a.y + row * a.d.y_row, dim, t,
                                         [&](int i, int e) { return y[i][e]; });
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = U * (64 * WPR * i + t);
      float y[U];
      result(i, y);
      store_chunk<Y, U, TAIL, FAR>((Y*)a.y + row * a.d.y_row + c, dim - c, y);
    }
  }
}

template <typename X, typename Y>
static hipError_t forward(const LayerNormArgs& a, hipStream_t st) {
  const long total = (long)a.d.groups * a.d.rows;
  constexpr int U = sizeof(X) == 2 ? 8 : 4;   // x alone decides: a row's sums do not depend on y's type
  return with_row_shape<U>(a.d.dim, [&](auto shape) {
    typedef decltype(shape) S;
    const long grid = S::WPR == 1 ? (total + 3) / 4 : total;
    if (const hipError_t s = check_grid(grid, 256); s != hipSuccess) return s;
    const bool far = past_caches((double)total * a.d.dim * (sizeof(X) + sizeof(Y)));
    const auto kernel = far ? k_layer_norm_op<X, Y, U, S::WPR, S::NV, S::TAIL, true>
                            : k_layer_norm_op<X, Y, U, S::WPR, S::NV, S::TAIL, false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t layer_norm(const LayerNormArgs& a, hipStream_t st) {
  if (a.d.x_dtype == CS_BF16)
    return a.d.y_dtype == CS_BF16   ? forward<bf16, bf16>(a, st)
           : a.d.y_dtype == CS_FP32 ? forward<bf16, float>(a, st)
                                    : forward<bf16, int8_t>(a, st);
  return a.d.y_dtype == CS_BF16   ? forward<float, bf16>(a, st)
         : a.d.y_dtype == CS_FP32 ? forward<float, float>(a, st)
                                  : forward<float, int8_t>(a, st);
}

// ----------------------------------------------------------------- backward
// With n = (x - mean) rstd and g = dy gain:
//   dx = rstd (g - mean(g) - n mean(g n)),  dw = sum over rows of dy n,  db = sum of dy.
// A workgroup takes ln_part_rows of a group's rows, with the gains and its lanes' sums dw and db in
// registers and the next row on its way while one is reduced; its sums go to the workspace,
// [group][part][2][dim], and a second launch adds a group's parts up in order.  12,480 x 1536 with fp32
// x and bf16 dy take 33 us (5.8 TB/s) and 4.2 for the parts, 32,760 x 5120 in bf16 197 (5.1
// TB/s) and 5.0.
int ln_part_rows(int rows) {
  // About 512 parts of a long group, so that one alone fills the card, 16 rows at least: what is
  // written and read of the sums, 16 bytes a channel and part, is then a twelfth of the rows' bytes in fp32, a
  // sixth in bf16, half as much again where dx is not wanted.  Rows
  // of the group alone decide, so that its gradients do not depend on other groups.  Up to 32 rows are
  // one part, whose sums are the gradient: the second launch costs more than 16 rows do.  256 rows at most:
  // a part's sums are fp32, so that more would lose digits (at 8 M rows, in parts of 16,384, 1024 half
  // steps of a sum of equal values); past 131,072 rows there are more parts instead.
  if (rows <= 32) return 32;
  return std::clamp((cdiv(rows, 512) + 3) / 4 * 4, 16, 256);
}
static int ln_parts(int rows) { return cdiv(rows, ln_part_rows(rows)); }

size_t layer_norm_backward_workspace(const cs_layer_norm_grad_desc& d) {
  if (ln_parts(d.rows) == 1) return 0;
  return (size_t)d.groups * ln_parts(d.rows) * 2 * round_up(d.dim, 4) * sizeof(float);
}

template <typename X, typename Y, int U, int WPR, int NV, bool TAIL, bool FAR>
__global__ __launch_bounds__(256) void k_layer_norm_grad(LayerNormGradArgs a, int parts, int part_rows) {
  constexpr int STEP = WPR == 1 ? 4 : 1;               // rows of the workgroup's waves
  __shared__ float2 lds[2][4];
  __shared__ float sums[WPR == 1 ? 4 : 1][WPR == 1 ? 64 * NV * U : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int group = blockIdx.x / parts, part = blockIdx.x - group * parts;
  const int dim = a.d.dim, t = WPR == 1 ? lane : (int)threadIdx.x;
  const int first = part * part_rows + (WPR == 1 ? wave : 0), last = min((part + 1) * part_rows, a.d.rows);
  const float inv = 1.0f / (float)dim;
  float gain[NV][U];
  {
    const float one = a.d.unit_offset ? 1.0f : 0.0f;
    const float* w = a.weight ? a.weight + group * a.d.w_group : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int h = 0; h < U / 4; ++h) {
        const int c = U * (64 * WPR * i + t) + 4 * h;
        const f32x4 v = w ? load_chunk<float, 4, TAIL>(w + c, dim - c) : f32x4{};
#pragma unroll
        for (int e = 0; e < 4; ++e) gain[i][4 * h + e] = w ? one + v[e] : 1.0f;
      }
  }
  struct Row {
    typename Chunk<X, U>::vec x[NV];
    typename Chunk<Y, U>::vec dy[NV];
    float mean, rstd;
  };
  auto load = [&](int r, Row& o) {
    const long row = (long)group * a.d.rows + r;
    const X* x = (const X*)a.x + row * a.d.x_row;
    const Y* dy = (const Y*)a.dy + row * a.d.dy_row;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = U * (64 * WPR * i + t);
      o.x[i] = load_chunk<X, U, TAIL, FAR>(x + c, dim - c);
      o.dy[i] = load_chunk<Y, U, TAIL, FAR>(dy + c, dim - c);
    }
    o.mean = a.mean[row];
    o.rstd = a.rstd[row];
  };
  float dw[NV][U] = {}, db[NV][U] = {};
  Row next;
  if (first < last) load(first, next);
  int odd = 0;
  for (int r = first; r < last; r += STEP, odd ^= 1) {
    const Row cur = next;
    if (r + STEP < last) load(r + STEP, next);   // on its way while this row is reduced
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int left = dim - U * (64 * WPR * i + t);
      if (left <= 0) continue;
#pragma unroll
      for (int e = 0; e < U; ++e) {
        if (TAIL && e >= left) continue;   // dy is zero there, but n need not be finite
        const float d = to_f(cur.dy[i][e]), n = (to_f(cur.x[i][e]) - cur.mean) * cur.rstd, g = d * gain[i][e];
        dw[i][e] = fmaf(d, n, dw[i][e]);
        db[i][e] += d;
        s1 += g;
        s2 = fmaf(g, n, s2);
      }
    }
    const float2 m = row_sums<WPR>(s1, s2, lds[odd], wave);
    if (!a.dx) continue;
    const float m1 = m.x * inv, m2 = m.y * inv;
    X* dx = (X*)a.dx + ((long)group * a.d.rows + r) * a.d.dx_row;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = U * (64 * WPR * i + t);
      float o[U];
#pragma unroll
      for (int e = 0; e < U; ++e) {
        const float n = (to_f(cur.x[i][e]) - cur.mean) * cur.rstd;
        o[e] = cur.rstd * (fmaf(to_f(cur.dy[i][e]), gain[i][e], -m1) - n * m2);
      }
      store_chunk<X, U, TAIL, FAR>(dx + c, dim - c, o);
    }
  }
  if (!a.dweight && !a.dbias) return;
  const long ld = (dim + 3) & ~3;
  float* sum[2] = {a.dweight + group * a.d.dw_group, a.dbias + group * a.d.db_group};
  if (parts > 1) {
    sum[0] = a.part + ((long)group * parts + part) * 2 * ld;
    sum[1] = sum[0] + ld;
  }
  const bool wanted[2] = {parts > 1 || a.dweight, parts > 1 || a.dbias};
  // whole chunks to the workspace, whose rows are padded to 4
  const int end = parts > 1 ? (int)ld : dim;
  auto store = [&](float* p, int c, const float* v) {
#pragma unroll
    for (int h = 0; h < U / 4; ++h) store_chunk<float, 4, TAIL>(p + c + 4 * h, end - c - 4 * h, v + 4 * h);
  };
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (WPR == 1) {
      // the four waves' rows, added in order; element e of chunk i of a lane lies at 64 (U i + e) + lane
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < U; ++e) sums[wave][64 * (U * i + e) + lane] = k ? db[i][e] : dw[i][e];
      __syncthreads();
      for (int i = wave; i < NV; i += 4) {
        float v[U];
#pragma unroll
        for (int e = 0; e < U; ++e) {
          const int q = 64 * (U * i + e) + lane;
          v[e] = ((sums[0][q] + sums[1][q]) + sums[2][q]) + sums[3][q];
        }
        if (wanted[k]) store(sum[k], U * (64 * i + lane), v);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (wanted[k]) store(sum[k], U * (64 * WPR * i + t), k ? db[i] : dw[i]);
    }
  }
}

// The parts' sums, a channel a lane and a sixteenth of the parts a wave, in 64 bits: 512 or
// more numbers that partly cancel, and the launch waits for memory anyway.  With four waves, a load
// behind the other, 512 parts of 5120 channels took 33 us.
__global__ __launch_bounds__(1024) void k_layer_norm_grad_sum(LayerNormGradArgs a, int parts) {
  __shared__ double sums[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int cols = (a.d.dim + 63) / 64, group = blockIdx.x / cols, k = blockIdx.y;
  const int c = (blockIdx.x - group * cols) * 64 + lane;
  const long ld = (a.d.dim + 3) & ~3;
  const float* p = a.part + ((long)group * parts * 2 + k) * ld + c;
  const int per = (parts + 15) / 16, first = wave * per, last = min(first + per, parts);
  double s = 0.0;
  if (c < a.d.dim) {
#pragma unroll 8
    for (int i = first; i < last; ++i) s += p[(long)i * 2 * ld];
  }
  sums[wave][lane] = s;
  __syncthreads();
  float* out = k ? a.dbias : a.dweight;
  if (wave != 0 || c >= a.d.dim || !out) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += sums[i][lane];
  out[group * (k ? a.d.db_group : a.d.dw_group) + c] = (float)s;
}

template <typename X, typename Y>
static hipError_t backward(const LayerNormGradArgs& a, hipStream_t st) {
  const int parts = ln_parts(a.d.rows), part_rows = ln_part_rows(a.d.rows);
  const long blocks = (long)a.d.groups * parts, sums = (long)a.d.groups * cdiv(a.d.dim, 64);
  const bool join = parts != 1 && (a.dweight || a.dbias);   // parts 0: no rows, whose sums are zeros
  if (const hipError_t s = check_grid(blocks, 256); s != hipSuccess) return s;
  if (const hipError_t s = join ? check_grid(sums, 1024) : hipSuccess; s != hipSuccess) return s;
  if (a.d.rows > 0) {
    constexpr int U = sizeof(X) == 2 && sizeof(Y) == 2 ? 8 : 4;
    const hipError_t s = with_row_shape<U>(a.d.dim, [&](auto shape) {
      typedef decltype(shape) S;
      const bool far = past_caches((double)a.d.groups * a.d.rows * a.d.dim * (2 * sizeof(X) + sizeof(Y)));
      const auto kernel = far ? k_layer_norm_grad<X, Y, U, S::WPR, S::NV, S::TAIL, true>
                              : k_layer_norm_grad<X, Y, U, S::WPR, S::NV, S::TAIL, false>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, a, parts, part_rows);
      return hipGetLastError();
    });
    if (s != hipSuccess) return s;
  }
  if (!join) return hipSuccess;
  hipLaunchKernelGGL(k_layer_norm_grad_sum, dim3((unsigned)sums, 2), dim3(1024), 0, st, a,
                     parts);
  return hipGetLastError();
}

hipError_t layer_norm_backward(const LayerNormGradArgs& a, hipStream_t st) {
  if (a.d.x_dtype == CS_BF16)
    return a.d.y_dtype == CS_BF16 ? backward<bf16, bf16>(a, st) : backward<bf16, float>(a, st);
  return a.d.y_dtype == CS_BF16 ? backward<float, bf16>(a, st) : backward<float, float>(a, st);
}

}  // namespace cs
