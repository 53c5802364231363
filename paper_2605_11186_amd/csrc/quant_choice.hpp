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
                                     {128, 112, 330}, {128, 128, 350}, {128, 192, 420}, {128, 256, 500},
                                     {256, 192, 600}, {256, 256, 700}};
constexpr int N_QUANT_TILES = sizeof(QUANT_TILES) / sizeof(QUANT_TILES[0]);
constexpr int N_QUANT_SPLIT_TILES = N_QUANT_TILES - 4;   // those whose kernel can take a piece of the inner length
inline int quant_tile_choice(int rows, int cols, int n_cus, int pieces = 1, int64_t* cost_out = nullptr) {
    int best = 0;
    int64_t least = INT64_MAX;
    for (int i = 0; i < (pieces > 1 ? N_QUANT_SPLIT_TILES : N_QUANT_TILES); ++i) {
        const QuantTile& c = QUANT_TILES[i];
        if (rows <= 16 && c.bm > 16) break;
        const int64_t tiles = ((int64_t{rows} + c.bm - 1) / c.bm) * ((int64_t{cols} + c.bn - 1) / c.bn) * pieces;
        const int64_t cost = (tiles + n_cus - 1) / n_cus * c.cost;
        if (cost <= least) {   // of equals the larger tile: fewer bytes
            least = cost;
            best = i;
        }
    }
    if (cost_out) *cost_out = least;
    return best;
}

// Many rows: tiles that fill a round of compute units and a few more leave the chip idle for most of the next one.  Then the first
// columns, whole rounds of one of the four largest tiles, are one launch and the others another, in the tiles that suit them best.
// 700 x 22016 x 4096 90 us as 258 tiles of 256 x 256, 66.5 as 255 of them and 256 columns in tiles of 32 x 32; 1500 x 12288 x 4096 88 and
// 73.  What the second launch costs, a start and, at any inner length, some operands that nothing hides, decides where little is
// gained: of 127 sizes with two launches by the tiles and the start alone the 40 that go out in one took 7 % more to 6 % less time in two, 1 %
// more on average (1500 x 4096 x 11008 68 us, 71 in two; 300 x 22016 x 4096 44.5 and 46), the other 87 take 13 % more to 27 % less, 6 % less
// on average; what loses still is of short inner lengths (1200 x 15360 x 1024 27.6, 31 in two).
// The tiles of 192 columns fill the chip where those of 256 do not: 256 x 22016 x 4096 43.6 -> 37.0, 300 x 15360 x 5120 43.5 -> 35.5.
struct QuantPlan {
    int tile, cols;     // of the first launch; cols: all of them, or the first ones, a multiple of 64
    int rest_tile;      // of the second, if there is one
};
constexpr int LAUNCH_COST = 40;   // of the second launch, at inner = 4096
constexpr int SECOND_COST = 50;   // and at any inner length
inline QuantPlan quant_plan(int rows, int cols, int inner, int n_cus) {
    int64_t least;
    QuantPlan best{quant_tile_choice(rows, cols, n_cus, 1, &least), cols, 0};
    if (rows <= 128) return best;
    least *= inner;
    for (int i = N_QUANT_SPLIT_TILES; i < N_QUANT_TILES; ++i) {
        const QuantTile& c = QUANT_TILES[i];
        const int64_t m_tiles = (int64_t{rows} + c.bm - 1) / c.bm, n_tiles = (int64_t{cols} + c.bn - 1) / c.bn;
        const int64_t rounds = m_tiles * n_tiles / n_cus, n_main = rounds * n_cus / m_tiles;
        if (n_main < 1 || n_main == n_tiles) continue;
        const int main_cols = static_cast<int>(n_main) * c.bn;
        int64_t rest;
        const int rest_tile = quant_tile_choice(rows, cols - main_cols, n_cus, 1, &rest);
        const int64_t cost = ((m_tiles * n_main + n_cus - 1) / n_cus * c.cost + rest + SECOND_COST) * inner + int64_t{LAUNCH_COST} * 4096;
        if (cost < least) {
            least = cost;
            best = {i, main_cols, rest_tile};
        }
    }
    return best;
}

// Pieces of the inner length, each a product of its own, that the consumer adds up: where few columns make small tiles, larger
// ones of a piece each read less (63 x 4096 x 11008 from memory 16.0 us in tiles of 32 x 32, 13.7 in two pieces of 64 x 32; 63 x 5120
// x 13824 24.7 and in three of 64 x 64 17.2).  Every piece more is rows of float32 written and read and counts PIECE_COST at inner =
// 4096.  Layers in 8 bits, us, one piece | cost 8 | 16 | 24: 7B-shaped, 63 nodes 93.7 | 92.6 | 92.6 | 92.8, 128 nodes 121.3 | 121.3 |
// 119.4 | 119.4; 13B-shaped 123.7 | 116.6 | 116.7 | 116.6 and 166.6 | 161.0 | 161.0 | 159.2.
struct QuantCut {
    int tile, pieces;
};
constexpr int PIECE_COST = 24;
inline QuantCut quant_cut_choice(int rows, int cols, int inner, int n_cus, int max_pieces) {
    QuantCut best{0, 1};
    int64_t least = INT64_MAX;
    for (int p = 1; p <= (rows > 16 ? max_pieces : 1); ++p) {
        int64_t cost;
        const int tile = quant_tile_choice(rows, cols, n_cus, p, &cost);
        cost = cost * inner / p + int64_t{PIECE_COST} * 4096 * (p - 1);
        if (cost < least) {
            least = cost;
            best = {tile, p};
        }
    }
    return best;
}
