// Which tile a product of 8-bit integers is cut into.  Plain C++: the host decides, a CPU test asks it.
#pragma once
#include <stdint.h>

// A launch takes about as long as the compute unit with the most tiles needs for their operands, rows of X and of W alike:
// rounds of tiles times (BM + BN).  Measured at inner = 4096 and 4096 columns (us): 1.2 + 0.065 rounds (BM + BN), within
// 10 % from 63 to 512 rows, for the tiles whose cost is BM + BN; the larger ones, which the matrix instructions bind, cost what
// they measure in this unit.  (With few rows and many columns the weights' way from memory comes on top for all alike:
// 90 MB of weights take 15 us with one row, 20 with 63.)
// Tiles of 32 rows, with the widths that let one round hold a common matrix, matter from 17 to 32 rows (32 x 22016 x 4096 18.5 -> 16.9 us,
// 32 x 27648 x 5120 27.4 -> 25.1) and where two of them fit better than one of 64 (63 x 5120 x 13824 from memory 25.7 -> 23.9).
// Up to 16 rows it is the weights alone, and several workgroups a compute unit take them in best: no taller tiles (one row x 22016 x
// 4096 15.0 us in tiles of 16 x 48, 16.0 in tiles of 32 x 96).
struct QuantTile {
    int bm, bn, cost;   // rows, columns, cost of a round of one tile per compute unit
};
constexpr QuantTile QUANT_TILES[] = {{16, 16, 32},   {16, 32, 50},   {16, 48, 70},   {32, 16, 48},   {32, 32, 64},   {32, 48, 80},   {32, 64, 96},
                                     {32, 96, 128},  {32, 112, 144}, {32, 128, 160}, {64, 32, 96},   {64, 48, 112},  {64, 64, 128},  {64, 96, 160},
                                     {64, 112, 176}, {64, 128, 192}, {96, 96, 192},  {128, 64, 192}, {128, 96, 250}, {96, 128, 288},
                                     {128, 112, 330}, {128, 128, 350}, {128, 256, 500}, {256, 256, 700}};
constexpr int N_QUANT_TILES = sizeof(QUANT_TILES) / sizeof(QUANT_TILES[0]);
inline int quant_tile_choice(int rows, int cols, int n_cus) {
    int best = 0;
    int64_t least = INT64_MAX;
    for (int i = 0; i < N_QUANT_TILES; ++i) {
        const QuantTile& c = QUANT_TILES[i];
        if (rows <= 16 && c.bm > 16) break;
        const int64_t tiles = ((int64_t{rows} + c.bm - 1) / c.bm) * ((int64_t{cols} + c.bn - 1) / c.bn);
        const int64_t cost = (tiles + n_cus - 1) / n_cus * c.cost;
        if (cost <= least) {   // of equals the larger tile: fewer bytes
            least = cost;
            best = i;
        }
    }
    return best;
}
