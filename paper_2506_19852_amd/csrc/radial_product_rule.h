// Which tiles an 8-bit product takes, which workgroup takes which, and where a stage's codes lie in LDS: evaluated on the host, too.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace radial {

// Tiles of a product.  What a launch takes is put together from the time of a stage (of each part) and of what a tile does besides, in us, as measured
// with the chip full of that tile, or with one on each compute unit where two fit (5120 x 5120, 100 to 14 040 rows, and others): large tiles move the
// fewest codes per product, but a launch of a few of them leaves compute units idle, and a workgroup alone on its unit spends more than half of a small
// tile's stage waiting, which parts of the groups at the same time make up for.
struct TileForm {
  int32_t rows, columns, at_once, split;
  float stage_full, stage_one, besides;
};
constexpr TileForm kTileForms[] = {
    {256, 256, 1, 1, 1.66f, 1.66f, 6.f}, {192, 256, 1, 1, 1.33f, 1.33f, 5.f}, {128, 128, 2, 1, 1.28f, 0.80f, 3.f}, {128, 128, 1, 2, 1.25f, 1.25f, 3.f},
    {64, 128, 2, 1, 0.74f, 0.55f, 2.5f}, {64, 128, 1, 2, 0.80f, 0.80f, 2.5f}, {64, 64, 2, 2, 0.90f, 0.62f, 2.f},   {64, 64, 1, 4, 1.10f, 1.10f, 2.f},
};
inline int choose_tiles(int32_t M, int32_t N, int32_t groups) {
  constexpr int64_t kUnits = 256;
  int best = 0;
  double least = 0;
  for (int i = 0; i < (int)(sizeof(kTileForms) / sizeof(kTileForms[0])); ++i) {
    const TileForm& f = kTileForms[i];
    const int64_t tiles = (((int64_t)M + f.rows - 1) / f.rows) * (((int64_t)N + f.columns - 1) / f.columns);
    const int64_t round = kUnits * f.at_once, full = tiles / round, rest = tiles % round;
    const double stages = (groups + f.split - 1) / f.split;
    const double last = rest == 0 ? 0.0 : rest <= kUnits ? stages * f.stage_one + f.besides : stages * f.stage_full + f.besides;
    const double time = full * (stages * f.stage_full + f.besides) + last;
    if (i == 0 || time < least) {
      best = i;
      least = time;
    }
  }
  return best;
}

// Tile of a workgroup.  XCD x of 8 (workgroup id mod 8) gets a run of neighbouring tiles, in bands of 8 rows of tiles, column by column: the 32 that
// it works on at a time are 8 x 4, whose codes it fetches into its L2 once.
__host__ __device__ __forceinline__ void tile_of(uint32_t id, int32_t tiles_m, int32_t tiles_n, int32_t& m, int32_t& n) {
  constexpr uint32_t kXcds = 8, kBand = 8;
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
