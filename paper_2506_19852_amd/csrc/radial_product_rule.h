// Which tiles an 8-bit product takes, which workgroup takes which, and where a stage's codes lie in LDS: evaluated on the host, too.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace radial {

// Tiles of a product.  What a launch takes is put together from the time of a stage (of each part) and of what a tile does besides, in us, as measured
// with the chip full of that tile, or with one on each compute unit where two fit (5120 x 5120, 100 to 14 040 rows, and others): large tiles move the
// fewest codes per product, but a launch of a few of them leaves compute units idle, and a workgroup alone on its unit spends more than half of a small
// tile's stage waiting, which parts of the groups at the same time make up for.  With few groups, where the start and the end of a tile are most of it, the
// estimate is too low: 1237 x 1961 x 1000, eight groups, 8.0 us of 11.4 to 12.2.
struct TileForm {
  int32_t rows, columns, at_once, split;
  float stage_full, stage_one, besides;
};
constexpr TileForm kTileForms[] = {
    {256, 256, 1, 1, 1.66f, 1.66f, 6.f}, {192, 256, 1, 1, 1.33f, 1.33f, 5.f}, {128, 128, 2, 1, 1.28f, 0.80f, 3.f}, {128, 128, 1, 2, 1.25f, 1.25f, 3.f},
    {64, 128, 2, 1, 0.74f, 0.55f, 2.5f}, {64, 128, 1, 2, 0.80f, 0.80f, 2.5f}, {64, 64, 2, 2, 0.90f, 0.62f, 2.f},   {64, 64, 1, 4, 1.10f, 1.10f, 2.f},
};
constexpr int kTileFormCount = sizeof(kTileForms) / sizeof(kTileForms[0]);
constexpr int64_t kComputeUnits = 256;

inline double tile_time(const TileForm& f, int32_t M, int32_t N, int32_t groups) {
  const int64_t tiles = (((int64_t)M + f.rows - 1) / f.rows) * (((int64_t)N + f.columns - 1) / f.columns);
  const int64_t round = kComputeUnits * f.at_once, full = tiles / round, rest = tiles % round;
  const double stages = (groups + f.split - 1) / f.split;
  const double last = rest == 0 ? 0.0 : rest <= kComputeUnits ? stages * f.stage_one + f.besides : stages * f.stage_full + f.besides;
  return full * (stages * f.stage_full + f.besides) + last;
}

inline int choose_tiles(int32_t M, int32_t N, int32_t groups, double* time, const TileForm* forms = kTileForms, int count = kTileFormCount) {
  int best = 0;
  for (int i = 0; i < count; ++i) {
    const double t = tile_time(forms[i], M, N, groups);
    if (i == 0 || t < *time) {
      best = i;
      *time = t;
    }
  }
  return best;
}

// The forms of a product: one for all rows, or where whole rounds of large tiles leave a small part of a round over, one for the rows of the whole rounds and
// another, in a launch of its own, for the rest.  (5120 x 5120 x 14 040: 400 tiles of 256 x 256 are two rounds; 240 of them, and 220 of 192 x 256,
// one round each.)
struct ProductPlan {
  int32_t rows, form, rest;  // rows in `form`, those behind them in `rest`
};
inline ProductPlan plan_product(int32_t M, int32_t N, int32_t groups, const TileForm* forms = kTileForms, int count = kTileFormCount) {
  constexpr double kLaunch = 8.0, kWorth = 0.95;  // us of another launch and its start; what the estimate has to promise
  double least = 0;
  ProductPlan plan = {M, choose_tiles(M, N, groups, &least, forms, count), 0};
  least *= kWorth;
  for (int form = 0; form < 2; ++form) {
    const TileForm& f = forms[form];
    const int64_t of_row = ((int64_t)N + f.columns - 1) / f.columns, tiles = ((int64_t)M + f.rows - 1) / f.rows * of_row;
    const int64_t rows = tiles / kComputeUnits * kComputeUnits / of_row * f.rows;
    if (rows < f.rows || rows >= M) continue;
    double rest_time = 0;
    const int rest = choose_tiles((int32_t)(M - rows), N, groups, &rest_time, forms, count);
    const double time = tile_time(f, (int32_t)rows, N, groups) + rest_time + kLaunch;
    if (time < least) {
      least = time;
      plan = {(int32_t)rows, form, rest};
    }
  }
  return plan;
}

// Few rows or few results: pieces of 16 x 16, whose eight waves share the groups and read them straight from memory, as long as each piece has a compute
// unit of its own.  (256 x 128 x 20 519, 128 pieces: 21 us, in tiles 33; 512 x 128 x 20 480, 256: 21, 41; 128 x 128 x 2048: 4.6, 7.4; with 264 pieces 14.1
// either way; 403 x 384 x 7296, 624: 22, 15; 1024 x 1024 x 2048: 32, 8.)
inline int64_t pieces_of(int32_t n) { return ((int64_t)n + 15) / 16; }
inline bool takes_pieces(int32_t M, int32_t N) { return M <= 16 || pieces_of(M) * pieces_of(N) <= kComputeUnits; }

// Tile of a workgroup.  XCD x of 8 (workgroup id mod 8) gets a run of neighbouring tiles, in bands of kBand rows of tiles, column by column: of the 32 that
// it works on at a time 8 share a column with kBand 8 (8 x 4) and 6 with 6, and their codes are fetched into its L2 once.
template <uint32_t kBand = 8>
__host__ __device__ __forceinline__ void tile_of(uint32_t id, int32_t tiles_m, int32_t tiles_n, int32_t& m, int32_t& n) {
  constexpr uint32_t kXcds = 8;
  const uint32_t tiles = (uint32_t)tiles_m * tiles_n, each = tiles / kXcds, more = tiles % kXcds;
  const uint32_t xcd = id % kXcds, at = xcd * each + (xcd < more ? xcd : more) + id / kXcds;
  const uint32_t band = at / (kBand * tiles_n), in_band = at - band * kBand * tiles_n;
  const uint32_t left = (uint32_t)tiles_m - band * kBand, rows = left < kBand ? left : kBand;
  m = band * kBand + in_band % rows;
  n = in_band / rows;
}

// Where piece p (16 bytes) of row r of an operand lies: two rows to a line of 256 bytes, pieces exchanged within it so that the 16 lanes that read one piece
// of 16 rows meet 16 different banks of 16 bytes: of A 16 neighbouring rows, of B rows 16 i + 4 t + j, i and j below 4.  The exchange is the
// same for all fragments of a lane, so that they are at constant distances from one another.
template <bool kB>
__host__ __device__ __forceinline__ int exchange_of(int line) { return kB ? (line & 1) | (line >> 3 & 3) << 1 : line & 7; }
template <bool kB>
__host__ __device__ __forceinline__ int code_piece(int r, int p) {
  const int line = r >> 1, slot = (r & 1) * 8 + p;
  return (line << 8) + ((slot ^ exchange_of<kB>(line)) << 4);
}

}  // namespace radial
