"""GPU parity of the operators in 8-bit integers against their definitions in 64 bits.

Rows in 8 bits: with v the exact row and d the relative error of the kernel's float32 v, the kernel rounds
v (1 + d) * fl(127 / top), top = max|v| (1 + d), to a whole number in one rounding, so
|q - 127 v / max|v|| <= 1/2 + 127 (2 d + 2^-23), and its scale is max|v| / 127 to within (d + 2^-24) of it.
  d = 0 for plain rows;
  norm: at most 64 multiply-adds a thread, 6 + 16 additions across threads, halved by the square root, and 8 more
  roundings: (86 / 2 + 8) 2^-24 < 2^-18;
  SwiGLU: exp(-g) by the hardware's exp2, off by 2 |g| 2^-24 for the rounded product with log2(e) and 2 more, and 5
  roundings behind it: with |g| <= 20 less than (40 + 2 + 5) 2^-24 < 2^-18.
Product: the sums are exact; their conversion and two products in float32 give 3 roundings of 2^-24, bf16 one of 2^-8.
"""
import numpy as np
import pytest
import torch

import paper_2605_11186_amd as cats

pytestmark = pytest.mark.gpu

D = 2.0 ** -18
EPS = 1e-6


def padded(rows, cols, dtype, ld=None, offset=0, fill=None):
    """A [rows][cols] view with rows `ld` elements apart, `offset` elements into its memory."""
    ld = (cols + 15) // 16 * 16 if ld is None else ld
    flat = torch.empty(offset + rows * ld + 16, dtype=dtype, device="cuda")
    flat.fill_(0 if fill is None else fill)
    return flat.as_strided((rows, cols), (ld, 1), offset), flat


def rng_of(*key):
    return np.random.default_rng(key)


def normal(rng, rows, cols, dtype=torch.float32, **place):
    view, _ = padded(rows, cols, dtype, **place)
    view.copy_(torch.from_numpy(rng.standard_normal((rows, cols)).astype(np.float32)).cuda().to(dtype))
    return view


def f64(t):
    return t.detach().cpu().double().numpy()


def check_rows(v, q, scale, d):
    """v: exact rows (numpy float64)."""
    top = np.maximum(np.abs(v).max(1), 127 * 2.0 ** -126)
    q, scale = f64(q), f64(scale)
    assert np.abs(q).max() <= 127
    assert (np.abs(scale - top / 127) <= (d + 2.0 ** -24) * top / 127 * (1 + 1e-6)).all()
    off = np.abs(q - v * 127 / top[:, None])
    assert off.max() <= 0.5 + 127 * (2 * d + 2.0 ** -23), off.max()


def silu_mul(gu, cols):
    g, u = gu[:, :cols], gu[:, cols:]
    return g / (1 + np.exp(-g)) * u


def norm_of(x, gain):
    return x / np.sqrt((x * x).mean(1, keepdims=True) + EPS) * gain


# every number of threads and pieces a row is cut into, both sides of each border, rows of one value
SIZES = [(1, 1), (3, 7), (5, 8), (2, 64), (9, 500), (4, 512), (3, 520), (1, 2047), (2, 2048), (300, 2056), (700, 4096),
         (1, 4096), (300, 4097), (5, 6144), (3, 6152), (270, 8192), (3, 8192), (2, 8200), (3, 12288), (2, 12296), (2, 16384), (2, 20001),
         (1, 65536)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantize_rows(rows, cols, dtype):
    src = normal(rng_of(1, rows, cols), rows, cols, dtype)
    q, _ = padded(rows, cols, torch.int8)
    scale = torch.empty(rows, device="cuda")
    cats.cats_quantize_rows(src, q, scale)
    check_rows(f64(src), q, scale, 0.0)


@pytest.mark.parametrize("delta_type", [None, torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_rmsnorm_quantize(rows, cols, delta_type):
    rng = rng_of(2, rows, cols)
    x = normal(rng, rows, cols)
    delta = None if delta_type is None else normal(rng, rows, cols, delta_type)
    gain = torch.from_numpy(1 + 0.02 * rng.standard_normal(cols)).cuda().to(torch.bfloat16)
    before = x.clone()
    q, _ = padded(rows, cols, torch.int8)
    scale = torch.empty(rows, device="cuda")
    x_out = None if delta is None else torch.empty(rows, cols, device="cuda")
    cats.cats_rmsnorm_quantize(x, gain, EPS, q, scale, delta=delta, x_out=x_out)
    assert torch.equal(x, before)
    if delta is not None:
        assert torch.equal(x_out, x + delta.float())   # one addition, rounded once
    check_rows(norm_of(f64(x if delta is None else x_out), f64(gain)), q, scale, D)
    if delta is not None:   # in place: the same bits
        q2, scale2 = torch.empty_like(q), torch.empty_like(scale)
        cats.cats_rmsnorm_quantize(x, gain, EPS, q2, scale2, delta=delta)
        assert torch.equal(x, x_out) and torch.equal(q2, q) and torch.equal(scale2, scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_swiglu_quantize(rows, cols, dtype):
    gate_up = normal(rng_of(3, rows, cols), rows, 2 * cols, dtype)
    gate_up *= 3.5   # gates up to about 17: both ends of the sigmoid
    gate_up.clamp_(-20, 20)
    q, _ = padded(rows, cols, torch.int8)
    scale = torch.empty(rows, device="cuda")
    cats.cats_swiglu_quantize(gate_up, q, scale)
    check_rows(silu_mul(f64(gate_up), cols), q, scale, D)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols,ld,offset,q_ld,q_offset", [(64, 65, 0, 64, 0), (64, 64, 1, 72, 0), (128, 136, 8, 129, 0),
                                                          (1000, 1001, 3, 1003, 5), (2056, 2064, 0, 2056, 4)])
def test_any_alignment_and_nothing_beside_the_rows(cols, ld, offset, q_ld, q_offset, dtype):
    rows = 6
    rng = rng_of(4, cols, ld)
    src = normal(rng, rows, cols, dtype, ld=ld, offset=offset)
    q, q_flat = padded(rows, cols, torch.int8, ld=q_ld, offset=q_offset, fill=77)
    scale_flat = torch.full((rows + 8,), 5.0, device="cuda")
    scale = scale_flat[1:rows + 1]
    cats.cats_quantize_rows(src, q, scale)
    check_rows(f64(src), q, scale, 0.0)
    assert scale_flat[0] == 5 and (scale_flat[rows + 1:] == 5).all()
    q.fill_(77)   # the rows themselves: all else must still be what it was
    assert (q_flat == 77).all()

    x = normal(rng, rows, cols, ld=ld, offset=offset)
    delta = normal(rng, rows, cols, dtype, ld=ld, offset=offset + 1)
    gain = torch.ones(cols + 3, device="cuda").to(torch.bfloat16)[3:]
    x_out, x_flat = padded(rows, cols, torch.float32, ld=ld, offset=offset, fill=-3)
    cats.cats_rmsnorm_quantize(x, gain, EPS, q, scale, delta=delta, x_out=x_out)
    assert torch.equal(x_out, x + delta.float())
    check_rows(norm_of(f64(x_out), f64(gain)), q, scale, D)
    x_out.fill_(-3)
    q.fill_(77)
    assert (x_flat == -3).all() and (q_flat == 77).all()

    gate_up = normal(rng, rows, 2 * cols, dtype, ld=2 * ld, offset=offset)
    cats.cats_swiglu_quantize(gate_up, q, scale)
    check_rows(silu_mul(f64(gate_up), cols), q, scale, D)
    q.fill_(77)
    assert (q_flat == 77).all()


def test_whole_numbers_and_ties_to_even():
    """Rows whose largest value is 127: the quotient is the value itself, halves are exact ties."""
    row = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5, -126.5, -127.0, 3.25, -0.0], device="cuda")[None]
    for src in (row, torch.cat([row, torch.zeros(1, 4, device="cuda")], 1)):   # one by one, and whole pieces
        q, scale = torch.empty(src.shape, dtype=torch.int8, device="cuda"), torch.empty(1, device="cuda")
        cats.cats_quantize_rows(src, q, scale)
        assert scale.item() == 1.0
        assert q[0, :12].tolist() == [127, 0, 2, 2, 0, -2, -2, 126, -126, -127, 3, 0]


def test_ties_among_bf16_values():
    """127 v / max|v| of bf16 values is a tie or next to none: |2 * 127 v - k max|v||, k odd, is a whole multiple of the values' last
    bits, so the quotient is a tie or at least 2^-16 / 2 from one relative to it, and float64 tells which."""
    src = normal(rng_of(12), 400, 2048, torch.bfloat16)
    src[100:200] *= 1e30
    src[200:300] *= 1e-30
    q, scale = torch.empty(400, 2048, dtype=torch.int8, device="cuda"), torch.empty(400, device="cuda")
    cats.cats_quantize_rows(src, q, scale)
    v = f64(src)
    y = v * 127 / np.abs(v).max(1, keepdims=True)
    assert (np.abs(y) % 1 == 0.5).sum() > 100   # there are some
    assert np.array_equal(f64(q), np.rint(y))


@pytest.mark.parametrize("cols", [5, 64, 4096, 9000])
def test_rows_of_zeros_tiny_huge_and_not_numbers(cols):
    rng = rng_of(5, cols)
    base = normal(rng, 9, cols)
    base[0] = 0
    base[1] *= 1e-42           # below the smallest scale
    base[2] *= 1e37            # near the end of the range
    base[3, cols // 2] = float("inf")
    base[4, 0] = float("-inf")
    base[5, cols - 1] = float("nan")
    base[6, 0], base[6, cols - 1] = float("nan"), float("inf")
    q, scale = torch.full((9, cols), 77, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    cats.cats_quantize_rows(base, q, scale)
    fine = [0, 1, 2, 7, 8]
    check_rows(f64(base[fine]), q[fine], scale[fine], 0.0)
    assert scale[0].item() == 2.0 ** -126 and not q[0].any()
    assert torch.isnan(scale[3:7]).all() and not q[3:7].any()
    # a product keeps it to those rows
    w = torch.ones(16, cols, dtype=torch.int8, device="cuda")
    qp, _ = padded(9, cols, torch.int8)
    qp.copy_(q)
    y = torch.empty(9, 16, device="cuda")
    cats.cats_quantized_linear(qp, scale, cats.cats_pack_quantized_matrix(w), torch.ones(16, device="cuda"), y)
    assert torch.isnan(y[3:7]).all()
    # row 2's sum, some sqrt(9000) * 1e37 = 9.5e38 for the longest rows, is itself beyond float32 (3.4e38): infinity is right there
    want = f64(q).sum(1) * f64(scale)
    assert np.array_equal(np.isfinite(f64(y[fine])), np.repeat(np.abs(want[fine])[:, None] < 3.4e38, 16, 1))
    # the norm: squares beyond float32 count as not a number, everything else as above
    gain = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    cats.cats_rmsnorm_quantize(base, gain, EPS, q, scale)
    fine = [0, 1, 7, 8]
    check_rows(norm_of(f64(base[fine]), 1.0), q[fine], scale[fine], D)
    assert torch.isnan(scale[2:7]).all() and not q[2:7].any()
    # SwiGLU: an infinite gate or factor makes its row not a number; a gate far below zero closes
    gu = torch.cat([base, base], 1).contiguous()
    gu[2] = 1.0
    gu[7, 0] = -200.0
    cats.cats_swiglu_quantize(gu, q, scale)
    fine = [0, 1, 2, 7, 8]
    with np.errstate(over="ignore"):
        check_rows(silu_mul(f64(gu[fine]), cols), q[fine], scale[fine], D)
    assert torch.isnan(scale[3:7]).all() and not q[3:7].any()


# ---------------------------------------------------------------- product
def whole_numbers(rng, rows, cols, lo=-128, ld=None):
    view, _ = padded(rows, cols, torch.int8, ld=ld, fill=99)   # what lies between the rows must not count
    view.copy_(torch.from_numpy(rng.integers(lo, 128, (rows, cols), dtype=np.int8)).cuda())
    return view


def check_linear(x, sx, w, sw, y):
    acc = f64(x.double() @ w.double().t().contiguous())   # whole numbers below 2^53: exact
    want = acc * f64(sx)[:, None] * f64(sw)[None, :]
    got = f64(y)
    tol = 3.01 * 2.0 ** -24 + (2.0 ** -8 if y.dtype == torch.bfloat16 else 0)
    assert (np.abs(got - want) <= np.abs(want) * tol).all(), np.abs(got - want).max()


def run_linear(rows, cols, inner, dtype, x_ld=None, y_ld=None, seed=0):
    rng = rng_of(6, rows, cols, inner, seed)
    x, w = whole_numbers(rng, rows, inner, ld=x_ld), whole_numbers(rng, cols, inner)
    sx = torch.from_numpy(rng.uniform(0.01, 0.02, rows).astype(np.float32)).cuda()
    sw = torch.from_numpy(rng.uniform(1e-4, 1e-3, cols).astype(np.float32)).cuda()
    y, flat = padded(rows, cols, dtype, ld=cols if y_ld is None else y_ld, offset=16, fill=-7)
    cats.cats_quantized_linear(x, sx, cats.cats_pack_quantized_matrix(w), sw, y)
    check_linear(x, sx, w, sw, y)
    y.fill_(-7)
    assert (flat == -7).all()   # nothing beside the rows


# rows on both sides of every border between variants, columns and inner lengths that no tile divides
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,inner", [
    (1, 1, 1), (1, 16, 64), (1, 17, 65), (1, 256, 256), (2, 3, 15), (1, 1000, 1001), (1, 4096, 4096), (1, 688, 11008),
    (7, 100, 100), (15, 256, 688), (16, 256, 256), (16, 31, 16), (17, 33, 17), (31, 130, 130), (32, 512, 1000), (33, 256, 320),
    (48, 1000, 64), (63, 2003, 1001), (64, 256, 4096), (65, 300, 500), (80, 272, 272), (96, 4100, 200), (100, 100, 5000),
    (127, 640, 640), (128, 1000, 1500), (129, 250, 700), (160, 400, 63), (192, 257, 1025), (255, 255, 255), (256, 256, 128),
    (257, 513, 129), (300, 1030, 400), (384, 768, 256), (500, 130, 1001), (513, 1025, 192), (1000, 1000, 1000),
    (1025, 511, 77), (2100, 300, 130)])
def test_linear(rows, cols, inner, dtype):
    run_linear(rows, cols, inner, dtype)


# one size for each tile that a product is cut into on 256 compute units (tests/test_quant_choice.py), none of them whole
TILE_SIZES = {(16, 16): (13, 1003), (16, 32): (9, 4107), (16, 48): (9, 12001), (32, 16): (27, 4091), (32, 32): (30, 4107),
              (32, 48): (29, 12001), (32, 64): (31, 15307), (32, 96): (29, 21001), (32, 112): (27, 27001), (32, 128): (31, 32001),
              (64, 32): (62, 8001), (64, 48): (57, 10007), (64, 64): (254, 4077), (64, 96): (61, 21001), (64, 112): (61, 27001),
              (64, 128): (63, 32001), (96, 96): (95, 21001), (128, 64): (509, 4077), (128, 96): (125, 21001), (96, 128): (763, 4077),
              (128, 112): (125, 27001), (128, 128): (1021, 4077), (128, 192): (500, 12201), (128, 256): (2001, 4077),
              (256, 192): (1001, 12201), (256, 256): (4001, 4077)}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("inner", [77, 1337])   # less than a step; several for each wave, the last one cut
@pytest.mark.parametrize("tile", sorted(TILE_SIZES))
def test_linear_every_tile(tile, inner, dtype):
    run_linear(*TILE_SIZES[tile], inner, dtype)


# few rows and some hundred megabytes of weights, which pass the caches by: one size for each tile that takes them all in one row tile
ONCE_SIZES = {(16, 16): (9, 4077, 22001), (16, 32): (3, 8177, 11203), (16, 48): (3, 22001, 4099), (32, 16): (31, 4077, 22001),
              (32, 32): (29, 4107, 22001), (32, 48): (29, 12001, 7501), (32, 64): (31, 15307, 6003), (32, 96): (29, 21001, 4301),
              (32, 112): (27, 27001, 3401), (32, 128): (31, 32001, 2807), (64, 32): (59, 8001, 11203), (64, 48): (57, 10007, 9003),
              (64, 64): (61, 15307, 6003), (64, 96): (61, 21001, 4301), (64, 112): (61, 27001, 3401), (64, 128): (63, 32001, 2807),
              (96, 96): (95, 21001, 4301), (128, 64): (125, 15307, 6003), (128, 96): (125, 21001, 4301), (96, 128): (95, 32001, 2807),
              (128, 112): (125, 27001, 3401), (128, 128): (125, 32001, 2807)}


@pytest.mark.parametrize("tile", sorted(ONCE_SIZES))
def test_linear_weights_past_the_caches(tile):
    run_linear(*ONCE_SIZES[tile], torch.bfloat16)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,inner", [(4001, 4177, 333), (3800, 8200, 1290), (300, 43501, 333), (513, 33000, 600), (999, 24504, 333),
                                             (500, 12200, 333)])
def test_linear_several_tiles_a_workgroup(rows, cols, inner, dtype):
    """More of the largest tiles than compute units: a workgroup's next tile is under way while it stores one.  (The last size: whole
    lines of y from tiles of 192 columns.)"""
    run_linear(rows, cols, inner, dtype)


# sizes whose last columns are a launch of their own (tests/test_quant_choice.py)
CUT_SIZES = [(700, 22001, 2000), (700, 22008, 2000), (4001, 12501, 333), (1500, 10800, 1000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols,inner", CUT_SIZES)
def test_linear_in_two_launches(rows, cols, inner, dtype):
    run_linear(rows, cols, inner, dtype)
    if rows == 700:
        run_linear(rows, cols, inner, dtype, x_ld=2016, y_ld=22017)


@pytest.mark.parametrize("rows", [1, 40, 130, 520])
@pytest.mark.parametrize("x_ld,y_ld", [(1024, 1003), (1040, 1004), (1008, 1024)])
def test_linear_strides(rows, x_ld, y_ld):
    run_linear(rows, 1000, 1001, torch.float32, x_ld=x_ld, y_ld=y_ld)
    run_linear(rows, 1000, 1001, torch.bfloat16, x_ld=x_ld, y_ld=y_ld)


@pytest.mark.parametrize("rows", [1, 20, 200, 600])
def test_linear_largest_sums(rows):
    """-128 times -128 at the longest inner length: the sum is 16384 * 131071, one below 2^31 / 16384."""
    inner = cats.CATS_QUANT_MAX_INNER
    x = torch.full((rows, inner + 1), -128, dtype=torch.int8, device="cuda")[:, :inner]
    w = torch.full((33, inner), -128, dtype=torch.int8, device="cuda")
    w[1::2] = 127
    y = torch.empty(rows, 33, device="cuda")
    one = torch.ones(rows, device="cuda")
    cats.cats_quantized_linear(x, one, cats.cats_pack_quantized_matrix(w), torch.ones(33, device="cuda"), y)
    want = torch.tensor([float(16384 * inner) if n % 2 == 0 else float(-128 * 127 * inner) for n in range(33)])
    assert torch.equal(y.cpu(), want.expand(rows, 33))


def test_linear_scales_next_to_the_range():
    """A row of the smallest scale, one with a large scale: the product goes by the row's scale first."""
    x = torch.full((3, 64), 100, dtype=torch.int8, device="cuda")
    w = torch.full((16, 64), 100, dtype=torch.int8, device="cuda")
    sx = torch.tensor([2.0 ** -126, 1e30, float("nan")], device="cuda")
    sw = torch.full((16,), 1e-4, device="cuda")
    y = torch.empty(3, 16, device="cuda")
    cats.cats_quantized_linear(x, sx, cats.cats_pack_quantized_matrix(w), sw, y)
    want = 640000 * f64(sx)[:, None] * f64(sw)[None, :]
    assert (np.abs(f64(y)[:2] - want[:2]) <= 3.01 * 2.0 ** -24 * want[:2]).all()
    assert torch.isnan(y[2]).all()


def test_pack_layout():
    rng = rng_of(7)
    for rows, cols, ld in [(16, 64, 64), (5, 3, 16), (33, 130, 144), (100, 1001, 1008), (100, 1001, 1003), (20, 64, 65), (17, 320, 320)]:
        w = whole_numbers(rng, rows, cols, ld=ld)
        packed = cats.cats_pack_quantized_matrix(w).cpu().numpy()
        full = np.zeros(((rows + 15) // 16 * 16, (cols + 255) // 256 * 256), np.int8)
        full[:rows, :cols] = w.cpu().numpy()
        # [row block][row][chunk][quarter][16] -> [row block][chunk][quarter][row][16]
        want = full.reshape(-1, 16, full.shape[1] // 64, 4, 16).transpose(0, 2, 3, 1, 4).reshape(-1)
        assert np.array_equal(packed, want)


def test_offsets_beyond_32_bits():
    """Rows gigabytes apart, and weights of more than 2^31 bytes."""
    rows, cols, ld = 3, 72, 1 << 30
    big = torch.empty(rows * ld, dtype=torch.int8, device="cuda")
    q = big.as_strided((rows, cols), (ld, 1))
    src = normal(rng_of(8), rows, cols)
    scale = torch.empty(rows, device="cuda")
    cats.cats_quantize_rows(src, q, scale)
    check_rows(f64(src), q, scale, 0.0)
    w = whole_numbers(rng_of(9), 40, cols)
    ld = cats.CATS_QUANT_MAX_LD - 16   # the longest stride of the product's x
    x = torch.empty(rows * ld, dtype=torch.int8, device="cuda").as_strided((rows, cols), (ld, 1))
    x.copy_(q)
    q, ld = x, 1 << 30
    y = torch.empty(2 * ld + 64, device="cuda").as_strided((rows, 40), (ld, 1))
    sw = torch.full((40,), 1e-3, device="cuda")
    cats.cats_quantized_linear(q, scale, cats.cats_pack_quantized_matrix(w), sw, y)
    check_linear(q, scale, w, sw, y)
    del big, q, x, y
    inner, n = 16400, 131104   # 2.15e9 bytes
    w = torch.randint(-128, 128, (n, inner), dtype=torch.int8, device="cuda")
    wp = cats.cats_pack_quantized_matrix(w)
    sw = torch.full((n,), 1e-3, device="cuda")
    tail = torch.arange(n - 70, n, device="cuda")
    for rows in (2, 70):
        x = whole_numbers(rng_of(10), rows, inner)
        sx = torch.full((rows,), 1e-2, device="cuda")
        y = torch.empty(rows, n, device="cuda")
        cats.cats_quantized_linear(x, sx, wp, sw, y)
        check_linear(x, sx, w[tail], sw[tail], y[:, tail])
        check_linear(x, sx, w[:70], sw[:70], y[:, :70])


def test_most_rows_and_most_columns():
    most = cats.CATS_QUANT_MAX_ROWS
    src = torch.randn(most, 8, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    q, _ = padded(most, 8, torch.int8)
    scale = torch.empty(most, device="cuda")
    cats.cats_quantize_rows(src, q, scale)
    check_rows(f64(src), q, scale, 0.0)
    w = whole_numbers(rng_of(13), 3, 8)
    y, sw = torch.empty(most, 3, device="cuda"), torch.full((3,), 1e-3, device="cuda")
    cats.cats_quantized_linear(q, scale, cats.cats_pack_quantized_matrix(w), sw, y)
    check_linear(q, scale, w, sw, y)
    del src, y
    x = whole_numbers(rng_of(14), 2, 16)   # and the other way round
    y, one = torch.empty(2, most, device="cuda"), torch.ones(2, device="cuda")
    w = torch.randint(-128, 128, (most, 16), dtype=torch.int8, device="cuda")
    cats.cats_quantized_linear(x, one, cats.cats_pack_quantized_matrix(w), scale, y)
    check_linear(x, one, w, scale, y)


# ---------------------------------------------------------------- use
def test_no_rows():
    q, s = torch.empty(0, 64, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda")
    cats.cats_quantize_rows(torch.empty(0, 64, device="cuda"), q, s)
    cats.cats_swiglu_quantize(torch.empty(0, 128, device="cuda"), q, s)
    cats.cats_rmsnorm_quantize(torch.empty(0, 64, device="cuda"), torch.ones(64, dtype=torch.bfloat16, device="cuda"), EPS, q, s)
    w = cats.cats_pack_quantized_matrix(torch.ones(16, 64, dtype=torch.int8, device="cuda"))
    cats.cats_quantized_linear(q, s, w, torch.ones(16, device="cuda"), torch.empty(0, 16, device="cuda"))


class Block:
    """A feed-forward block in 8 bits: norm, gate|up product, SwiGLU, down product; the residual addition rides in the next norm."""

    def __init__(self, rows, hidden, ffn, seed):
        rng = rng_of(11, rows, hidden, ffn, seed)
        self.rows, self.hidden, self.ffn = rows, hidden, ffn
        self.x, self.gain = normal(rng, rows, hidden), torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
        self.w = []
        for out, inner in ((2 * ffn, hidden), (hidden, ffn)):
            w = normal(rng, out, inner, torch.bfloat16)
            q, s = padded(out, inner, torch.int8)[0], torch.empty(out, device="cuda")
            cats.cats_quantize_rows(w, q, s)
            self.w.append((q, s, cats.cats_pack_quantized_matrix(q)))
        self.q1, self.q2, self.q3 = (padded(rows, n, torch.int8)[0] for n in (hidden, ffn, hidden))
        self.s1, self.s2, self.s3 = (torch.empty(rows, device="cuda") for _ in range(3))
        self.gu = torch.empty(rows, 2 * ffn, dtype=torch.bfloat16, device="cuda")
        self.down, self.x_out = torch.empty(rows, hidden, device="cuda"), torch.empty(rows, hidden, device="cuda")

    def run(self, stream=None):
        cats.cats_rmsnorm_quantize(self.x, self.gain, EPS, self.q1, self.s1, stream=stream)
        cats.cats_quantized_linear(self.q1, self.s1, self.w[0][2], self.w[0][1], self.gu, stream=stream)
        cats.cats_swiglu_quantize(self.gu, self.q2, self.s2, stream=stream)
        cats.cats_quantized_linear(self.q2, self.s2, self.w[1][2], self.w[1][1], self.down, stream=stream)
        cats.cats_rmsnorm_quantize(self.x, self.gain, EPS, self.q3, self.s3, delta=self.down, x_out=self.x_out, stream=stream)

    def outputs(self):
        return [t.clone() for t in (self.q1, self.s1, self.gu, self.q2, self.s2, self.down, self.x_out, self.q3, self.s3)]


@pytest.mark.parametrize("rows", [1, 19, 63, 300])
def test_block_step_by_step(rows):
    """The operators in a row; every step against its definition on the inputs that the step before left."""
    b = Block(rows, 256, 688, 0)
    b.run()
    torch.cuda.synchronize()
    check_rows(norm_of(f64(b.x), 1.0), b.q1, b.s1, D)
    check_linear(b.q1, b.s1, b.w[0][0], b.w[0][1], b.gu)
    assert b.gu.abs().max() <= 2000
    # |g| reaches some hundreds here: gates above 88 are open and below -88 closed to float32's end, between them
    # exp's error is at most (2 * 88 + 2) 2^-24, 183 roundings in all with those behind it
    check_rows(silu_mul(f64(b.gu), 688), b.q2, b.s2, 183 * 2.0 ** -24)
    check_linear(b.q2, b.s2, b.w[1][0], b.w[1][1], b.down)
    assert torch.equal(b.x_out, b.x + b.down)
    check_rows(norm_of(f64(b.x_out), 1.0), b.q3, b.s3, D)


def test_repeated_captured_and_concurrent_runs_give_the_same_bits():
    blocks = [Block(63, 256, 688, 1), Block(300, 512, 688, 2)]
    want = []
    for b in blocks:
        b.run()
        want.append(b.outputs())

    def same(b, w):
        return all(torch.equal(p, q) for p, q in zip(b.outputs(), w))

    streams = [torch.cuda.Stream() for _ in blocks]
    torch.cuda.synchronize()
    for _ in range(3):   # two streams at once
        for b, s in zip(blocks, streams):
            b.run(stream=s)
    torch.cuda.synchronize()
    assert all(same(b, w) for b, w in zip(blocks, want))
    graphs = []
    for b, s in zip(blocks, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            b.run(stream=torch.cuda.current_stream())
        graphs.append(g)
    for i in range(4):   # replays with other work and synchronisation between them
        for b, g in zip(blocks, graphs):
            b.gu.zero_(), b.down.zero_(), b.q3.zero_()
            torch.cuda.synchronize()
            g.replay()
            if i % 2:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert all(same(b, w) for b, w in zip(blocks, want))
