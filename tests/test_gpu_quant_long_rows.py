"""Rows in 8 bits of more than 16384 columns, whose threads hold 64 values each: every piece of a row in use, aligned and not."""
import pytest
import torch

import paper_2605_11186_amd as cats
from test_gpu_quant import D, EPS, check_rows, f64, norm_of, normal, padded, rng_of, silu_mul

pytestmark = pytest.mark.gpu

# columns, elements from row to row, first element: value by value to the last one; aligned memory, odd length; whole pieces; odd memory
PLACES = [(65535, 65535, 1), (65529, 65536, 0), (65528, 65536, 0), (65536, 65537, 3), (16385, 16400, 0), (32769, 32769, 2)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols,ld,offset", PLACES)
def test_long_rows(cols, ld, offset, dtype):
    rows, rng = 3, rng_of(21, cols, ld)
    q, q_flat = padded(rows, cols, torch.int8, ld=ld, offset=offset, fill=77)
    scale = torch.empty(rows, device="cuda")

    src = normal(rng, rows, cols, dtype, ld=ld, offset=offset)
    cats.cats_quantize_rows(src, q, scale)
    check_rows(f64(src), q, scale, 0.0)

    gate_up = normal(rng, rows, 2 * cols, dtype, ld=2 * ld, offset=offset)
    gate_up[1] *= 4
    gate_up.clamp_(-20, 20)
    cats.cats_swiglu_quantize(gate_up, q, scale)
    check_rows(silu_mul(f64(gate_up), cols), q, scale, D)

    gain = torch.from_numpy(1 + 0.1 * rng.standard_normal(cols)).cuda().to(torch.bfloat16)
    x, x_flat = padded(rows, cols, torch.float32, ld=ld, offset=offset, fill=-3)
    x.copy_(normal(rng, rows, cols))
    before = x.clone()
    cats.cats_rmsnorm_quantize(x, gain, EPS, q, scale)
    check_rows(norm_of(f64(x), f64(gain)), q, scale, D)
    delta = normal(rng, rows, cols, dtype, ld=ld, offset=offset)
    cats.cats_rmsnorm_quantize(x, gain, EPS, q, scale, delta=delta)   # in place
    assert torch.equal(x, before + delta.float())
    check_rows(norm_of(f64(x), f64(gain)), q, scale, D)
    q.fill_(77)   # nothing beside the rows
    x.fill_(-3)
    assert (q_flat == 77).all() and (x_flat == -3).all()
