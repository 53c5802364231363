"""No rows: nothing is enqueued and nothing refused, whatever the lengths of the rows that are not there."""
import pytest
import torch

import paper_2605_11186_amd as cats

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inner", [1, 17, 63, 64, 1001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_product_of_no_rows(inner, dtype):
    w = cats.cats_pack_quantized_matrix(torch.ones(20, inner, dtype=torch.int8, device="cuda"))
    x, y = torch.empty(0, inner, dtype=torch.int8, device="cuda"), torch.empty(0, 20, dtype=dtype, device="cuda")
    cats.cats_quantized_linear(x, torch.empty(0, device="cuda"), w, torch.ones(20, device="cuda"), y)
    some = torch.ones(3, inner, dtype=torch.int8, device="cuda")[:0]
    cats.cats_quantized_linear(some, torch.empty(0, device="cuda"), w, torch.ones(20, device="cuda"), y)


@pytest.mark.parametrize("cols", [1, 7, 20001])
def test_rows_of_no_rows(cols):
    q, s = torch.empty(0, cols, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda")
    x, gain = torch.empty(0, cols, device="cuda"), torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    cats.cats_quantize_rows(x, q, s)
    cats.cats_swiglu_quantize(torch.empty(0, 2 * cols, device="cuda"), q, s)
    cats.cats_rmsnorm_quantize(x, gain, 1e-6, q, s)
    cats.cats_rmsnorm_quantize(x, gain, 1e-6, q, s, delta=x)
