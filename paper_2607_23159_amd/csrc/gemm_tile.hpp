// Choice of the GEMM tile in bf16 and in 8 bits.  Plain host code, without HIP, so that the
// tests can ask which tiles their shapes reach.
#pragma once

namespace cs {

enum Bf16Tile {
  W4_256x256, W4_224x256, W4_192x256, W4_160x256, W4_128x128, W4_64x64,
  RING_128x128, RING_64x128, RING_64x64, RING_32x64, RING_32x32, N_TILES
};

// Time of a launch per tile shape, in us:
//   fixed + rounds * (K/64 * full + epi) + K/64 * (lone + (full - lone) * r) + epi * (1 + r) / 2
// where a round fills `slots` workgroups on each of the 256 CUs of a whole device
// (another count changes the speed of the choice, not a result), r is the
// filled part of the last round (left out when 0), `lone` and `full` are the
// time per K slice of 64 of a tile alone on its CU and of a full chip, and epi
// grows by epi_res for residual updates.  The constants are a least-squares fit
// to 966 measured shapes (32 to 65,520 rows; N and K of projections at widths
// 128 to 5120 and of the heads; bf16 stores and residual updates), each launch
// on another copy of the weights out of 900 MB: in a model a layer's weights
// come from HBM, which shifts the choice towards shapes with more loads in
// flight.  They were then adjusted for the choice rather than for the times:
// against the best tile of each of these shapes (none was held out) it costs 1.0%
// on average below 1,024 rows or so (at most 20%, at launches of 20 us) and 0.6%
// above, where 256 x 256 tiles for everything took 3.2 times and 12% longer on
// average.  A 128 x 256 tile is not among them, though at width 5120 it measured 4
// to 8% faster than the tile chosen (1024 x 5120 x 13824 190 against 205 us, 3120 x
// 5120 x 5120 152 against 160).  The row counts between 128 and 256 are for the
// last round: 12,480 x 1536 x 8960 takes 384 us with 256 rows (294 workgroups on
// 256 CUs), 315 with 192 and 297 with 160 (468, two nearly full rounds), 12,480 x
// 4608 x 1536 154 us with 256 and 144 with 224.
struct TileCost { int bm, bn, slots; double lone, full, fixed, epi, epi_res; };
static constexpr TileCost TILE_COST[N_TILES] = {
    {256, 256, 1, 1.022, 1.378, 3.20, 6.88, 16.20},
    {224, 256, 1, 0.820, 1.222, 1.71, 6.29, 14.71},
    {192, 256, 1, 0.785, 1.107, 3.09, 5.48, 11.52},
    {160, 256, 1, 0.754, 0.977, 1.74, 3.78, 9.75},
    {128, 128, 2, 0.472, 0.930, 2.00, 2.62, 5.00},
    {64, 64, 3, 0.246, 0.646, 2.07, 1.14, 0.88},
    {128, 128, 1, 0.469, 0.457, 1.29, 4.23, 2.50},
    {64, 128, 1, 0.355, 0.368, 1.56, 2.16, 0.92},
    {64, 64, 1, 0.198, 0.218, 1.79, 1.51, 0.41},
    {32, 64, 2, 0.164, 0.276, 1.86, 1.05, 0.25},
    {32, 32, 2, 0.159, 0.245, 1.76, 0.76, 0.00},
};

// The same for 8-bit products, K/128 slices of as many bytes (and cycles) each: a fit to 277
// measured shapes (1 to 65,520 rows; N and K of projections at widths 256 to 5120, and odd ones),
// weights from HBM.  Against the best tile of each it costs 0.9% on average, 13% at most.  12,480 x
// 1536 x 8960 takes 191 us with 256 x 256 tiles, 154 with 160 x 256; 1560 x 4608 x 1536 25.7 and
// 18.5; 32,760 x 13,824 x 5120 1790 us with 256 x 256 and 2124 with 128 x 128, on one machine (others
// take 1770 to 1890 with the former).
// Residual updates are taken to add what they add in bf16.
static constexpr TileCost TILE_COST_I8[N_TILES] = {
    {256, 256, 1, 0.912, 1.320, 5.06, 11.57, 16.20},
    {224, 256, 1, 0.847, 1.160, 4.70, 10.64, 14.71},
    {192, 256, 1, 0.820, 1.069, 4.55, 8.98, 11.52},
    {160, 256, 1, 0.759, 0.956, 3.99, 7.31, 9.75},
    {128, 128, 2, 0.488, 0.996, 2.30, 4.52, 5.00},
    {64, 64, 3, 0.401, 0.608, 2.05, 1.34, 0.88},
    {128, 128, 1, 0.436, 0.509, 2.37, 4.34, 2.50},
    {64, 128, 1, 0.370, 0.426, 2.18, 2.39, 0.92},
    {64, 64, 1, 0.199, 0.260, 2.12, 1.70, 0.41},
    {32, 64, 2, 0.223, 0.305, 2.13, 1.25, 0.25},
    {32, 32, 2, 0.117, 0.193, 2.28, 1.06, 0.00},
};

// The loop is unrolled so that every division is by a constant (0.07 us a launch
// instead of 0.12).
template <const TileCost (&COST)[N_TILES], int FIRST = 0>
static Bf16Tile cheapest_tile(long M, long N, double nk, long batch, bool residual, double* time = nullptr) {
  auto cost = [&](int i) {
    const TileCost& c = COST[i];
    const long tiles = (M + c.bm - 1) / c.bm * ((N + c.bn - 1) / c.bn) * batch, round = 256L * c.slots;
    const double epi = c.epi + (residual ? c.epi_res : 0.0), r = (double)(tiles % round) / (double)round;
    double t = c.fixed + (double)(tiles / round) * (nk * c.full + epi);
    if (r > 0) t += nk * (c.lone + (c.full - c.lone) * r) + epi * 0.5 * (1.0 + r);
    return t;
  };
  int best = FIRST;
  double best_t = cost(FIRST);
#pragma clang loop unroll(full)
  for (int i = FIRST + 1; i < N_TILES; ++i) {
    const double t = cost(i);
    if (t < best_t) { best = i; best_t = t; }
  }
  if (time) *time = best_t;
  return (Bf16Tile)best;
}

static Bf16Tile choose_tile(long M, long N, long K, long batch, bool residual) {
  return cheapest_tile<TILE_COST>(M, N, (double)(K / 64), batch, residual);
}

static inline Bf16Tile choose_tile_i8(long M, long N, long K, bool residual) {
  return cheapest_tile<TILE_COST_I8>(M, N, (double)((K + 127) / 128), 1, residual);
}

// Up to 16 rows of up to FEW_COLS outputs are k_matmul_few's.  1 x 1536 x 8960: 6.0 us against
// 11.0 with the best tile, 16 rows 8.3 against 11.2; 16 x 1536 x 1536 4.0 against 4.3.  Past them one
// row is as fast either way (1 x 13,824 x 5120: 16.1 us both, weights from HBM), and for more the
// rows, which every workgroup reads past LDS, cost more than the tiles' latency (16 x 13,824 x 5120
// 21.3 against 16.5).
constexpr int FEW_ROWS = 16, FEW_COLS = 4096;

// Parts of K for 8-bit products: their sums in one launch, joined by a second.  For few rows and a long
// K, where one launch of small tiles is a chain of slices on a part of the chip.  64 x 5120 x 13,824
// takes 20.5 us in 3 parts against 29.1, 32 x 512 x 8960 7.0 in 6 against 11.2, 128 x 5120 x
// 13,824 25.9 in 3 against 34.6.  The parts' time is that of as many tiles with their share of K, 2.5 us and the
// sums at 8 bytes each and way: over 99 measured shapes (8 to 700 rows, k 1536 to 13,824) the choice costs
// 2.3% against the best; the 21 shapes that it cuts are 21% faster than in one launch (0.9% slower at worst).
// A tenth has to be had: the second launch is the host's time too.
struct SplitK { int parts, per; Bf16Tile tile; };   // per: slices of a part

static inline SplitK split_k_i8(long M, long N, long K) {
  const long nk = (K + 127) / 128;
  SplitK best = {1, (int)nk, RING_32x32};
  if (nk < 48 || M > 1024 || N > 65536 || (M <= FEW_ROWS && N <= FEW_COLS)) return best;
  double least;
  cheapest_tile<TILE_COST_I8>(M, N, (double)nk, 1, false, &least);
  least *= 0.9;
  static constexpr int TRIES[] = {2, 3, 4, 6};
  for (int s : TRIES) {
    const long per = (nk + s - 1) / s, parts = (nk + per - 1) / per;
    double t;
    const Bf16Tile tile = cheapest_tile<TILE_COST_I8, RING_64x128>(M, N, (double)per, parts, false, &t);
    t += 2.5 + (double)(parts * M * N) * 1e-6;
    if (t < least) {
      least = t;
      best = {(int)parts, (int)per, tile};
    }
  }
  return best;
}

}  // namespace cs
