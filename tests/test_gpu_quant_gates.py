"""SwiGLU rows in 8 bits whose gates are far below zero, against the definition in 64 bits.

With d the relative error of the kernel's float32 v, the quotient 127 v / max|v| is off by at most 127 (2 d + 1.5 * 2^-23): v and the
largest one, and the factor of one rounding and one ulp of a reciprocal.
  g >= -20: the product of g and log2(e), off by 2^-24 of it and by the constant's 2^-26, is off by at most 20 (2^-24 + 2^-26) as an
  exponent of e; exp2 and the reciprocal an ulp each (2^-23), three roundings of 2^-24: 32 * 2^-24 in all, 2^-19.
  g < -20: exp(g / 2) twice, each an ulp of exp2 and two roundings, with the exponent's rounding made good, and three products:
  11 * 2^-24; 1 + exp(g) is 1 to within 2^-28.
So the quotient is off by at most 127 (2^-18 + 1.5 * 2^-23) = 5.1e-4 < 2^-10: whole numbers beyond 2^-10 of a tie are the definition's."""
import numpy as np
import pytest
import torch

import paper_2605_11186_amd as cats

pytestmark = pytest.mark.gpu

D = 2.0 ** -19
# (lowest gate, highest gate, size of the other factor); exp(g / 2) is a normal number of float32 down to g = -174
GATES = [(-88.72, -87.34, 1.0), (-88.72, -87.34, 1e3), (-88, -30, 1.0), (-88, -30, 1e3), (-90, -60, 1e30), (-103, -85, 1e38), (-174, -100, 1e38),
         (-40, -35, 1e-20), (-25, -15, 1.0), (-20.001, -19.999, 1.0), (-60, 5, 1e-3)]


def check(gate_up, cols, q, scale):
    gu = gate_up.detach().cpu().double().numpy()
    g, u = gu[:, :cols], gu[:, cols:]
    v = g / (1 + np.exp(-g)) * u
    top = np.maximum(np.abs(v).max(1), 127 * 2.0 ** -126)
    scale = scale.cpu().double().numpy()
    assert (np.abs(scale * 127 / top - 1) <= D + 2.0 ** -23).all()
    y = v * 127 / top[:, None]
    away = np.abs(np.abs(y - np.rint(y)) - 0.5) > 2.0 ** -10
    assert away.mean() > 0.9
    got = q.cpu().double().numpy()
    assert np.array_equal(got[away], np.rint(y)[away])
    assert (np.abs(got - y) <= 0.5 + 2.0 ** -10).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [64, 999, 4096, 11008])
def test_gates_far_below_zero(cols, dtype):
    rng = np.random.default_rng(cols)
    rows = len(GATES)
    g = np.stack([rng.uniform(lo, hi, cols) for lo, hi, _ in GATES])
    u = np.stack([rng.uniform(0.5, 1, cols) * rng.choice([-1, 1], cols) * size for _, _, size in GATES])
    gate_up = torch.from_numpy(np.concatenate([g, u], 1).astype(np.float32)).cuda().to(dtype)
    q = torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device="cuda")[:, :cols]
    scale = torch.empty(rows, device="cuda")
    cats.cats_swiglu_quantize(gate_up, q, scale)
    check(gate_up, cols, q, scale)


def test_a_value_does_not_depend_on_its_neighbours():
    """A row of ordinary gates, and the same with a closed one in it: all other values keep their bits."""
    rng = np.random.default_rng(3)
    cols = 4096
    row = torch.from_numpy(rng.standard_normal((1, 2 * cols)).astype(np.float32) * 6).cuda().clamp_(-19, 19)
    gate_up = row.repeat(3, 1)
    gate_up[1, 100], gate_up[2, 8:4000:8] = -50.0, -90.0
    q, scale = torch.empty(3, cols, dtype=torch.int8, device="cuda"), torch.empty(3, device="cuda")
    cats.cats_swiglu_quantize(gate_up, q, scale)
    assert scale[0] == scale[1]
    kept = torch.ones(cols, dtype=torch.bool, device="cuda")
    kept[100] = False
    assert torch.equal(q[0][kept], q[1][kept])
    top = int((row[0, :cols] / (1 + (-row[0, :cols]).exp()) * row[0, cols:]).abs().argmax())
    if top % 8 or not 8 <= top < 4000:   # the largest value is still there
        kept[8:4000:8] = False
        assert scale[0] == scale[2] and torch.equal(q[0][kept], q[2][kept])


def test_infinite_gates_and_factors():
    """An infinity on either side of a product, whatever the other side: the row is not a number."""
    inf = float("inf")
    for g, u in ((-inf, 1.0), (inf, 1.0), (-50.0, inf), (-500.0, inf), (1.0, -inf), (float("nan"), 1.0), (-50.0, float("nan"))):
        gate_up = torch.full((2, 128), -30.0, device="cuda")
        gate_up[1, 5], gate_up[1, 64 + 5] = g, u
        q, scale = torch.full((2, 64), 77, dtype=torch.int8, device="cuda"), torch.empty(2, device="cuda")
        cats.cats_swiglu_quantize(gate_up, q, scale)
        assert torch.isnan(scale[1]) and not q[1].any()
        assert torch.isfinite(scale[0]) and (q[0] == 127).all()
