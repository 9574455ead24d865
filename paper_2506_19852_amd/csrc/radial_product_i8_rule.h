// Which tiles a product of 8-bit integers takes: evaluated on the host, too.
#pragma once

#include "radial_product_rule.h"

namespace radial {

// Tiles as in radial_product_rule.h, with times measured for whole numbers, which need no scaling between the matrix instructions: stages at K 256 to 5120 with one tile on each
// compute unit and with the chip full several times over.  What a tile does besides, mostly writing its results, includes the launch of 3 to 4 us.  Few tiles take forms of many
// waves, or of parts of the groups, and rings of three stages: one tile of 128 x 128 takes 0.48 us a stage on eight waves, 0.70 on four with two stages.
constexpr TileForm kTileFormsI8[] = {
    {256, 256, 1, 1, 1.40f, 1.40f, 8.5f}, {192, 256, 1, 1, 1.13f, 1.13f, 7.f},  {128, 128, 2, 1, 0.84f, 0.70f, 5.f}, {128, 128, 1, 1, 0.48f, 0.48f, 5.2f},
    {96, 128, 1, 1, 0.41f, 0.41f, 4.8f},  {64, 128, 2, 1, 0.57f, 0.33f, 4.3f}, {64, 64, 3, 1, 0.53f, 0.25f, 3.7f},   {64, 64, 1, 2, 0.36f, 0.36f, 4.f},
    {32, 64, 2, 2, 0.46f, 0.244f, 3.7f},  {32, 64, 1, 4, 0.42f, 0.42f, 4.f},
};
constexpr int kTileFormCountI8 = sizeof(kTileFormsI8) / sizeof(kTileFormsI8[0]);
inline ProductPlan plan_product_i8(int32_t M, int32_t N, int32_t groups) { return plan_product(M, N, groups, kTileFormsI8, kTileFormCountI8); }

// Rows of tiles of a band: 6, so that the 32 tiles of 256 x 256 that an XCD works on at a time are 6 x 5.  A band's rows of A are read from beyond the XCD's L2 once for each five
// columns of tiles, which counts where A does not fit the last-level cache: 32 760 x 5120 x 5120 663 us, 689 with bands of 8 (eight by four), 32 760 x 8192 x 2560 581 (645),
// 32 760 x 15 360 x 5120 2038 (2100), smaller ones alike; bands of 4, 5 and 7 between 655 and 666, 591 and 603, 1959 and 2086.
constexpr uint32_t kBandI8 = 6;

// Up to 4 rows, or few results: pieces of 16 x 16.  (1 x 5120 x 5120 7.7 us, in tiles of 32 x 64 8.2; 8 rows 9.3, 8.2; 16 rows 10.9, 8.1.  1 x 8192 x 2048 4.5, 5.5;
// 32 x 2048 x 8192, 256 pieces: 9.5, 10.4; 32 x 1024 x 1024, 128: 3.7, 4.5.)
inline bool takes_pieces_i8(int32_t M, int32_t N) { return M <= 4 || pieces_of(M) * pieces_of(N) <= kComputeUnits; }

}  // namespace radial
