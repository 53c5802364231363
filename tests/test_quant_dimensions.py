"""Operands in 8 bits that are no matrices, or no vectors, are refused like all that do not fit (runs without a GPU)."""
import pytest
import torch

import paper_2605_11186_amd as cats

X, Q, S, G = torch.zeros(2, 64), torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2), torch.zeros(64, dtype=torch.bfloat16)
W, SW, Y = torch.zeros(4096, dtype=torch.int8), torch.zeros(16), torch.zeros(2, 16)
CALLS = {
    "quantize_src": lambda f: cats.cats_quantize_rows(f(X), Q, S),
    "quantize_q": lambda f: cats.cats_quantize_rows(X, f(Q), S),
    "quantize_scale": lambda f: cats.cats_quantize_rows(X, Q, f(S)),
    "norm_x": lambda f: cats.cats_rmsnorm_quantize(f(X), G, 1e-6, Q, S),
    "norm_q": lambda f: cats.cats_rmsnorm_quantize(X, G, 1e-6, f(Q), S),
    "norm_gain": lambda f: cats.cats_rmsnorm_quantize(X, f(G), 1e-6, Q, S),
    "norm_delta": lambda f: cats.cats_rmsnorm_quantize(X, G, 1e-6, Q, S, delta=f(X)),
    "norm_x_out": lambda f: cats.cats_rmsnorm_quantize(X, G, 1e-6, Q, S, delta=X, x_out=f(X)),
    "swiglu_gate_up": lambda f: cats.cats_swiglu_quantize(f(torch.zeros(2, 128)), Q, S),
    "swiglu_q": lambda f: cats.cats_swiglu_quantize(torch.zeros(2, 128), f(Q), S),
    "pack_src": lambda f: cats.cats_pack_quantized_matrix(f(Q)),
    "linear_x": lambda f: cats.cats_quantized_linear(f(Q), S, W, SW, Y),
    "linear_w": lambda f: cats.cats_quantized_linear(Q, S, f(W), SW, Y),
    "linear_w_scale": lambda f: cats.cats_quantized_linear(Q, S, W, f(SW), Y),
    "linear_out": lambda f: cats.cats_quantized_linear(Q, S, W, SW, f(Y)),
}


@pytest.mark.parametrize("change", [torch.ravel, lambda t: t[None], lambda t: t[None, None], lambda t: t.sum()],
                         ids=["flat", "one_more", "two_more", "number"])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_refused(name, change):
    with pytest.raises(cats.CatsError) as e:
        CALLS[name](change)
    assert e.value.status == cats.CATS_EINVAL
