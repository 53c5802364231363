"""Which tile a product of 8-bit integers is cut into (host code, no GPU)."""
import ctypes
import re

import pytest

import host_shim
from test_gpu_quant import CUT_SIZES, ONCE_SIZES, TILE_SIZES
from test_gpu_quant_layers import PIECES

SHIM = """
#include "quant_choice.hpp"
extern "C" {
int n_tiles() { return N_QUANT_TILES; }
int tile(int i, int what) { return what == 0 ? QUANT_TILES[i].bm : what == 1 ? QUANT_TILES[i].bn : QUANT_TILES[i].cost; }
int choice(int rows, int cols, int n_cus) { return quant_tile_choice(rows, cols, n_cus); }
int plan(int rows, int cols, int inner, int n_cus, int what) {
    const QuantPlan p = quant_plan(rows, cols, inner, n_cus);
    return what == 0 ? p.tile : what == 1 ? p.cols : p.rest_tile;
}
int pieces(int rows, int cols, int inner, int n_cus, int most) { return quant_cut_choice(rows, cols, inner, n_cus, most).pieces; }
int cut_tile(int rows, int cols, int inner, int n_cus, int most) { return quant_cut_choice(rows, cols, inner, n_cus, most).tile; }
}
"""


@pytest.fixture(scope="module")
def rule():
    return host_shim.build(SHIM)


def tile(rule, rows, cols, n_cus=256):
    i = rule.choice(rows, cols, n_cus)
    return rule.tile(i, 0), rule.tile(i, 1)


def test_every_tile_has_its_gpu_case(rule):
    assert sorted(TILE_SIZES) == sorted((rule.tile(i, 0), rule.tile(i, 1)) for i in range(rule.n_tiles()))
    for want, (rows, cols) in TILE_SIZES.items():
        assert tile(rule, rows, cols) == want
        assert rows % want[0] and cols % want[1]   # no size is a whole number of tiles


def test_sizes_whose_weights_pass_the_caches(rule):
    """The sizes of that GPU test: one row tile, more than a third of 256 MB of weights."""
    for want, (rows, cols, inner) in ONCE_SIZES.items():
        assert tile(rule, rows, cols) == want, (rows, cols, tile(rule, rows, cols))
        assert rows <= want[0] and cols * inner >= (256 << 20) // 3
    assert sorted(ONCE_SIZES) == sorted(t for t in TILE_SIZES if t[0] <= 128 and t[1] < 192)


def plan(rule, rows, cols, inner, n_cus=256):
    """The first launch's tile and columns, the second's tile."""
    return rule.plan(rows, cols, inner, n_cus, 0), rule.plan(rows, cols, inner, n_cus, 1), rule.plan(rows, cols, inner, n_cus, 2)


def test_several_tiles_a_workgroup(rule):
    """The sizes of the GPU test of that name: one launch, and but for the last more of the largest tiles than compute units."""
    for rows, cols, inner, want in ((4001, 4177, 333, (256, 192)), (3800, 8200, 1290, (256, 256)), (300, 43501, 333, (128, 256)),
                                    (513, 33000, 600, (256, 256)), (999, 24504, 333, (256, 192)), (500, 12200, 333, (128, 192))):
        t, first, _ = plan(rule, rows, cols, inner)
        assert (rule.tile(t, 0), rule.tile(t, 1)) == want and first == cols
        assert -(-rows // want[0]) * -(-cols // want[1]) > 256 or cols == 12200


def test_two_launches(rule):
    """The first columns fill whole rounds of compute units, the others come after; never dearer than one launch."""
    for rows, cols, inner in CUT_SIZES:
        assert plan(rule, rows, cols, inner)[1] < cols
    for rows in (1, 63, 128, 129, 300, 700, 1500, 4096, 2 ** 21):
        for cols in (1, 255, 4096, 12288, 22016, 100003, 2 ** 21):
            for inner in (16, 333, 4096, 131071):
                for n_cus in (1, 80, 256):
                    t, first, rest = plan(rule, rows, cols, inner, n_cus)
                    if first == cols:
                        assert t == rule.choice(rows, cols, n_cus)
                        continue
                    bm, bn = rule.tile(t, 0), rule.tile(t, 1)
                    assert rows > 128 and t >= rule.n_tiles() - 4 and 0 < first < cols and first % bn == 0
                    assert rest == rule.choice(rows, cols - first, n_cus)

                    def cost(i, n):
                        tiles = -(-rows // rule.tile(i, 0)) * -(-n // rule.tile(i, 1))
                        return -(-tiles // n_cus) * rule.tile(i, 2)

                    one = rule.choice(rows, cols, n_cus)
                    assert (cost(t, first) + cost(rest, cols - first)) * inner < cost(one, cols) * inner


def test_kernels_stand_in_the_order_of_the_tiles(rule):
    """launch_quant_linear's list: <row blocks, column blocks, ...> of 16, then the four of the other kernel."""
    text = (host_shim.CSRC / "quant_linear.hip").read_text()
    built = [(16 * int(m), 16 * int(n)) for m, n in re.findall(r"launch_split<(\d), (\d), \d, \d, \d>[,\s]", text)]
    tiles = [(rule.tile(i, 0), rule.tile(i, 1)) for i in range(rule.n_tiles())]
    assert built + [(128, 192), (128, 256), (256, 192), (256, 256)] == tiles


def test_the_choice_costs_least(rule):
    """Of all tiles; up to 16 rows, of those of 16 rows, which come first."""
    for rows in (1, 16, 17, 63, 64, 65, 128, 129, 500, 1024, 4096, 100000, 2 ** 21):
        for cols in (1, 16, 100, 4096, 5120, 22016, 32000, 2 ** 21):
            for n_cus in (1, 80, 256):
                costs = [-(-(-(-rows // rule.tile(i, 0)) * -(-cols // rule.tile(i, 1))) // n_cus) * rule.tile(i, 2)
                         for i in range(rule.n_tiles()) if rows > 16 or rule.tile(i, 0) == 16]
                assert costs[rule.choice(rows, cols, n_cus)] == min(costs)


def test_pieces_of_the_inner_length(rule):
    """One piece: the tile of the whole product.  More: a tile of the kernel that can take pieces, and not for up to 16 rows."""
    for hidden, ffn, nodes, want in PIECES:
        assert (rule.pieces(nodes, hidden, hidden, 256, 3), rule.pieces(nodes, hidden, ffn, 256, 3)) == want, (hidden, nodes)
    for rows in (1, 16, 17, 63, 128):
        for cols in (64, 512, 4096, 8192):
            for inner in (16, 64, 4096, 65536):
                assert rule.cut_tile(rows, cols, inner, 256, 1) == rule.choice(rows, cols, 256)
                p = rule.pieces(rows, cols, inner, 256, 3)
                assert p in (1, 2, 3) and (rows > 16 or p == 1) and (p == 1 or inner >= 128 * p)
                assert p == 1 or rule.cut_tile(rows, cols, inner, 256, 3) < rule.n_tiles() - 4
