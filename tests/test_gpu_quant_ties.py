"""Plain rows in 8 bits: 127 v / max|v| is rounded as the exact quotient is, ties to even, whatever the type of the row."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2605_11186_amd as cats

pytestmark = pytest.mark.gpu

SMALLEST = 2.0 ** -126


def exact(row):
    top = max(Fraction(float(np.abs(row).max())), 127 * Fraction(SMALLEST))
    return [round(Fraction(float(v)) * 127 / top) for v in row]   # of a Fraction: ties to even


def near_ties(top, rng):
    """The largest value, every tie of 127 v / top as far as float32 comes to it, and the numbers beside it."""
    k = np.arange(-127, 127) + 0.5
    t = (np.float64(top) * k / 127).astype(np.float32)
    away = np.abs(np.nextafter(t, np.float32(np.inf))), np.abs(np.nextafter(t, np.float32(-np.inf)))
    row = np.concatenate([[top, -top, 0.0, top / 3], t, np.copysign(away[0], t), np.copysign(away[1], t)]).astype(np.float32)
    row[np.abs(row) > top] = top
    return rng.permutation(row)


TOPS = [1.0, 127.0, 1.6369617, 1.5, 1.9999999, 1.0000001, 3.4028234e38, 2.5e38, 1.2e-38 * 200, 1e-36, 2e-36, 1e-40]


@pytest.mark.parametrize("cols", [768, 766, 765])   # whole pieces; rows of 766 values and 765, value by value
def test_float32_next_to_ties(cols):
    rng = np.random.default_rng(cols)
    tops = TOPS + list(rng.uniform(0.5, 2, 20) * 2.0 ** rng.integers(-100, 100, 20))
    rows = np.stack([np.resize(near_ties(np.float32(t), rng), 768)[:cols] for t in tops])
    src = torch.from_numpy(rows).cuda()
    q, scale = torch.empty(rows.shape, dtype=torch.int8, device="cuda"), torch.empty(len(rows), device="cuda")
    cats.cats_quantize_rows(src, q, scale)
    got, want = q.cpu().numpy(), np.array([exact(r) for r in rows])
    assert np.array_equal(got, want), np.argwhere(got != want)[:5]


def test_the_two_examples():
    """127 v / max|v| = 1.5 less a little: 1; 34.5 and 2.1e-6: 35."""
    row = np.zeros((2, 8), np.float32)
    row[0, :3] = 1.0, np.nextafter(np.float32(1.5 / 127), np.float32(0)), np.float32(0.0118110236)
    row[1, :2] = 1.6369617, 0.44468647
    q, scale = torch.empty(2, 8, dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
    cats.cats_quantize_rows(torch.from_numpy(row).cuda(), q, scale)
    assert q.cpu().tolist() == [exact(r) for r in row]
    assert q[1, 1].item() == 35


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_random_rows(dtype):
    """Rows as they come.  |2 * 127 v - k max|v||, k odd, is a whole multiple of v's last bit: a quotient is a tie or at least 2^-33 of
    itself from one, and float64 tells which."""
    src = torch.from_numpy(np.random.default_rng(4).standard_normal((300, 4096)).astype(np.float32)).cuda().to(dtype)
    q, scale = torch.empty(300, 4096, dtype=torch.int8, device="cuda"), torch.empty(300, device="cuda")
    cats.cats_quantize_rows(src, q, scale)
    v = src.double().cpu().numpy()
    y = 127 * v / np.abs(v).max(1, keepdims=True)   # one rounding: 127 v is exact
    assert np.array_equal(q.cpu().numpy(), np.rint(y))
