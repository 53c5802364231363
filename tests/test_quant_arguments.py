"""What the operators in 8-bit integers refuse, before any device work: runs without a GPU.  The addresses are made up; a
call that got as far as the device would not come back with the status asked for here."""
import pytest
import torch

import paper_2605_11186_amd as cats

P = 1 << 20   # some aligned address
BIG_ROWS, BIG_COLS, BIG_INNER = cats.CATS_QUANT_MAX_ROWS + 1, cats.CATS_QUANT_MAX_COLS + 1, cats.CATS_QUANT_MAX_INNER + 1
E, CAP = cats.CATS_EINVAL, cats.CATS_ECAPACITY

QUANTIZE = dict(src=P, type=0, ld=64, rows=2, cols=64, q=P, q_ld=64, scale=P, stream=None)
NORM = dict(x=P, x_ld=64, delta=P, delta_type=1, delta_ld=64, gain=P, eps=1e-6, rows=2, cols=64, x_out=P, x_out_ld=64, q=P,
            q_ld=64, scale=P, stream=None)
SWIGLU = dict(src=P, type=1, ld=128, rows=2, cols=64, q=P, q_ld=64, scale=P, stream=None)
PACK = dict(src=P, ld=64, rows=16, cols=64, dst=P, stream=None)
LINEAR = dict(x=P, x_ld=64, x_scale=P, w=P, w_scale=P, y=P, y_type=0, y_ld=16, rows=2, cols=16, inner=64, stream=None)


def call(name, base, **changed):
    assert set(changed) <= set(base)
    return getattr(cats.library(), name)(*{**base, **changed}.values())


@pytest.mark.parametrize("changed,status", [
    (dict(src=None), E), (dict(q=None), E), (dict(scale=None), E), (dict(type=2), E), (dict(type=-1), E),
    (dict(ld=63), E), (dict(q_ld=63), E), (dict(rows=-1), E), (dict(cols=0), E), (dict(src=P + 2), E),
    (dict(scale=P + 1), E), (dict(type=1, src=P + 1), E), (dict(rows=BIG_ROWS), CAP),
    (dict(cols=BIG_COLS, ld=BIG_COLS, q_ld=BIG_COLS), CAP), (dict(rows=0), cats.CATS_OK)])
def test_quantize_rows(changed, status):
    assert call("cats_quantize_rows", QUANTIZE, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(x=None), E), (dict(gain=None), E), (dict(q=None), E), (dict(scale=None), E), (dict(delta=None), E),
    (dict(x_out=None), E), (dict(delta_type=2), E), (dict(eps=0.0), E), (dict(eps=-1.0), E), (dict(eps=float("nan")), E),
    (dict(eps=float("inf")), E), (dict(x_ld=63), E), (dict(delta_ld=63), E), (dict(x_out_ld=63), E), (dict(q_ld=63), E),
    (dict(x_out_ld=128), E), (dict(x_out=P + 2), E), (dict(gain=P + 1), E), (dict(delta=P + 1), E), (dict(rows=-1), E),
    (dict(cols=0), E), (dict(rows=BIG_ROWS), CAP),
    (dict(cols=BIG_COLS, x_ld=BIG_COLS, delta_ld=BIG_COLS, x_out_ld=BIG_COLS, q_ld=BIG_COLS), CAP),
    (dict(rows=0), cats.CATS_OK), (dict(rows=0, delta=None, x_out=None), cats.CATS_OK)])
def test_rmsnorm_quantize(changed, status):
    assert call("cats_rmsnorm_quantize", NORM, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(src=None), E), (dict(type=7), E), (dict(ld=127), E), (dict(q=None), E), (dict(scale=None), E), (dict(cols=0), E),
    (dict(rows=-5), E), (dict(src=P + 1), E), (dict(rows=BIG_ROWS), CAP), (dict(rows=0), cats.CATS_OK),
    (dict(cols=BIG_COLS, ld=2 * BIG_COLS, q_ld=BIG_COLS), CAP), (dict(cols=2 ** 31 - 1, ld=2 ** 31), E)])
def test_swiglu_quantize(changed, status):
    assert call("cats_swiglu_quantize", SWIGLU, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(src=None), E), (dict(dst=None), E), (dict(dst=P + 8), E), (dict(rows=0), E), (dict(cols=0), E), (dict(ld=63), E),
    (dict(cols=BIG_INNER, ld=BIG_INNER), CAP), (dict(rows=BIG_ROWS), CAP)])
def test_pack_quantized_matrix(changed, status):
    assert call("cats_pack_quantized_matrix", PACK, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(x=None), E), (dict(x_scale=None), E), (dict(w=None), E), (dict(w_scale=None), E), (dict(y=None), E),
    (dict(y_type=2), E), (dict(x=P + 8), E), (dict(x_ld=72), E), (dict(x_ld=48), E), (dict(y_ld=15), E), (dict(w=P + 8), E),
    (dict(y=P + 2), E), (dict(x_scale=P + 2), E), (dict(w_scale=P + 2), E), (dict(rows=-1), E), (dict(cols=0), E),
    (dict(inner=0), E), (dict(inner=BIG_INNER, x_ld=BIG_INNER // 16 * 16 + 16), CAP), (dict(rows=BIG_ROWS), CAP),
    (dict(cols=BIG_ROWS, y_ld=BIG_ROWS), CAP), (dict(x_ld=cats.CATS_QUANT_MAX_LD), CAP), (dict(rows=2 ** 20, cols=2 ** 20, y_ld=2 ** 20), CAP),
    (dict(rows=0), cats.CATS_OK)])
def test_quantized_linear(changed, status):
    assert call("cats_quantized_linear", LINEAR, **changed) == status


def test_layers_need_a_context():
    layers = (cats.QuantizedLayer * 1)()
    assert cats.library().cats_verify_layers_quantized(None, layers, 0, 1, P, P, 0, None) == E


def test_packed_bytes():
    assert cats.cats_packed_quantized_bytes(1, 1) == 4096
    assert cats.cats_packed_quantized_bytes(16, 256) == 4096
    assert cats.cats_packed_quantized_bytes(17, 257) == 16384
    assert cats.cats_packed_quantized_bytes(0, 64) == cats.cats_packed_quantized_bytes(64, -1) == 0
    assert cats.cats_packed_quantized_bytes(2 ** 21, 131071) == 2 ** 21 * 131072   # beyond 32 bits


def test_binding_refuses_what_does_not_fit():
    """Shapes, types and places that the C call cannot see."""
    x, q, s = torch.zeros(2, 64), torch.zeros(2, 64, dtype=torch.int8), torch.zeros(2)
    g = torch.zeros(64, dtype=torch.bfloat16)
    w, sw, y = torch.zeros(4096, dtype=torch.int8), torch.zeros(16), torch.zeros(2, 16)
    bad = [
        lambda: cats.cats_quantize_rows(x.double(), q, s),
        lambda: cats.cats_quantize_rows(x, q[:, :63], s),
        lambda: cats.cats_quantize_rows(x, q.to(torch.uint8), s),
        lambda: cats.cats_quantize_rows(x, q, s[:1]),
        lambda: cats.cats_quantize_rows(x, torch.zeros(64, 2, dtype=torch.int8).t(), s),
        lambda: cats.cats_quantize_rows(x, q, s),   # host memory
        lambda: cats.cats_rmsnorm_quantize(x, g.float(), 1e-6, q, s),
        lambda: cats.cats_rmsnorm_quantize(x, g, 1e-6, q, s, x_out=x),
        lambda: cats.cats_rmsnorm_quantize(x, g, 1e-6, q, s, delta=x[:1]),
        lambda: cats.cats_swiglu_quantize(x, q, s),
        lambda: cats.cats_pack_quantized_matrix(q.float()),
        lambda: cats.cats_quantized_linear(q, s, w[:1024], sw, y),
        lambda: cats.cats_quantized_linear(q, s, w, sw, y.half()),
        lambda: cats.cats_quantized_linear(q, s, w, sw[:8], y),
        lambda: cats.cats_quantized_linear(torch.zeros(1, 63, dtype=torch.int8), s[:1], w, sw, y[:1]),   # 63 bytes of memory
        lambda: cats.cats_quantized_linear(q, s, w, sw, y),
    ]
    for f in bad:
        with pytest.raises(cats.CatsError) as e:
            f()
        assert e.value.status == cats.CATS_EINVAL


@pytest.mark.skipif(torch.cuda.is_available(), reason="on a device these calls would run")
@pytest.mark.parametrize("name,base", [("cats_quantize_rows", QUANTIZE), ("cats_rmsnorm_quantize", NORM), ("cats_swiglu_quantize", SWIGLU),
                                       ("cats_pack_quantized_matrix", PACK), ("cats_quantized_linear", LINEAR)])
def test_a_failure_of_the_device_has_its_text(name, base):
    lib = cats.library()
    assert call(name, base) == cats.CATS_EHIP
    assert lib.cats_strerror(cats.CATS_EHIP) == b"no ROCm-capable device is detected"
