"""A decoder layer in 8 bits at the sizes of the 7B and 13B models against its definition, block by block.

Of a layer only the updated rows and the appended cache rows can be seen, and a whole layer is known no better than the roundings on its
way let it be: a value next to a tie, moved by a float32 rounding, takes a row's products along.  So each block is looked at alone.

Attention block: the output weights are the identity (127 on the diagonal, scale 1 / 127) and the down weights zero, so that x' - x is the
attention output in 8 bits.  Feed-forward block: the output weights are zero; the block is the operators one behind the other, each of
which is held against its definition in 64 bits on the inputs that the step before left, and the layer against them."""
import numpy as np
import pytest
import torch

import paper_2605_11186_amd as cats
import synth
from test_gpu_quant import D, EPS, check_linear, check_rows, f64

pytestmark = pytest.mark.gpu

MAX_CTX = 320
# hidden, ffn, nodes, context rows
SIZES = [(4096, 11008, 63, 200), (4096, 11008, 1, 130), (5120, 13824, 128, 70), (5120, 13824, 20, 0)]


class Case:
    def __init__(self, hidden, ffn, nodes, ctx_len):
        self.H, self.F, self.T, self.S, self.heads = hidden, ffn, nodes, ctx_len, hidden // 128
        self.gen = torch.Generator(device="cuda").manual_seed(hidden + nodes)
        self.x = self.normal(nodes, hidden)
        gains = [(1 + 0.1 * self.normal(hidden)).to(torch.bfloat16) for _ in range(2)]
        self.weights = dict(wq=self.bf16(hidden, hidden), wk=self.bf16(hidden, hidden), wv=self.bf16(hidden, hidden), wo=None,
                            w_gate=self.bf16(ffn, hidden), w_up=self.bf16(ffn, hidden), w_down=None, g_attn=gains[0], g_ffn=gains[1])
        parent, depth = synth.random_tree(nodes, 9, 5)
        self.parent, self.depth = np.asarray(parent, np.int32), np.asarray(depth, np.int32)
        self.k = self.normal(self.heads, MAX_CTX, 128).to(torch.bfloat16)
        self.v = self.normal(self.heads, 128, MAX_CTX).to(torch.bfloat16)
        self.ctx = cats.cats_create(cats.ModelDesc(1, hidden, self.heads, 128, ffn, 1000, MAX_CTX, 128, EPS, 1e4, 0))

    def normal(self, *shape, by=1.0):
        return torch.empty(*shape, device="cuda").normal_(0, by, generator=self.gen)

    def bf16(self, *shape):
        return self.normal(*shape, by=0.02).to(torch.bfloat16)

    def run(self, weights):
        """The layer's x' - x in 64 bits, x', the caches behind it and the quantised layer."""
        layer, h, k, v = cats.quantize_layer(weights), self.x.clone(), self.k.clone(), self.v.clone()
        cats.cats_set_tree(self.ctx, np.zeros(self.T, np.int32), self.parent, self.depth)
        cats.cats_verify_layers_quantized(self.ctx, cats.quantized_layer_array([layer]), 0, 1, h, cats.kv_array([k], [v]), self.S)
        torch.cuda.synchronize()
        return h.double() - self.x.double(), h, k, v, layer

    def rows(self, gain):
        """rmsnorm(x) * gain in 8 bits by the operator, held against the definition."""
        q, s = torch.empty(self.T, self.H, dtype=torch.int8, device="cuda"), torch.empty(self.T, device="cuda")
        cats.cats_rmsnorm_quantize(self.x, gain, EPS, q, s)
        x = f64(self.x)
        check_rows(x / np.sqrt((x * x).mean(1, keepdims=True) + EPS) * f64(gain), q, s, D)
        return q, s

    def product(self, q, s, packed, scale, *matrices):
        """Its product by the operator, held against the definition."""
        y = torch.empty(q.shape[0], scale.numel(), device="cuda")
        cats.cats_quantized_linear(q, s, packed, scale, y)
        w = torch.cat(matrices)
        wq, ws = torch.empty(w.shape, dtype=torch.int8, device="cuda"), torch.empty(w.shape[0], device="cuda")
        cats.cats_quantize_rows(w, wq, ws)
        assert torch.equal(ws, scale)
        check_linear(q, s, wq, ws, y)
        return y


@pytest.fixture(params=SIZES, ids=lambda p: "x".join(map(str, p)))
def case(request):
    c = Case(*request.param)
    yield c
    torch.cuda.synchronize()
    cats.cats_destroy(c.ctx)


def test_attention_block(case):
    c = case
    eye = torch.eye(c.H, device="cuda").to(torch.bfloat16)
    got, _, k, v, layer = c.run(c.weights | dict(wo=eye, w_down=torch.zeros(c.H, c.F, dtype=torch.bfloat16, device="cuda")))
    w = c.weights
    qkv = c.product(*c.rows(w["g_attn"]), layer["w_qkv"], layer["s_qkv"], w["wq"], w["wk"], w["wv"]).double()
    q, kn, vn = (t.reshape(c.T, c.heads, 128) for t in qkv.chunk(3, 1))
    pos = torch.from_numpy(c.S + c.depth.astype(np.float64)).cuda()
    ang = (pos[:, None] * 1e4 ** (-2.0 * torch.arange(64, device="cuda", dtype=torch.float64) / 128))[:, None]

    def rotate(t):
        a, b = t[..., :64], t[..., 64:]
        return torch.cat([a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()], -1)

    q, kn = rotate(q), rotate(kn)
    # appended rows: bf16 (2^-8 of a value, which is a whole last bit) of values that float32 angles, sines and products leave 2^-15 of the
    # largest from exact (positions up to 330: an angle is off by 330 * 2^-24)
    for got_rows, want in ((k[:, c.S:c.S + c.T].transpose(0, 1), kn), (v[:, :, c.S:c.S + c.T].permute(2, 0, 1), vn)):
        assert ((got_rows.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15 * want.abs().max()).all()
    assert torch.equal(k[:, :c.S], c.k[:, :c.S]) and torch.equal(v[:, :, :c.S], c.v[:, :, :c.S])
    sees = torch.zeros(c.T, c.T, dtype=torch.bool, device="cuda")
    for i in range(c.T):
        j = i
        while j >= 0:
            sees[i, j] = True
            j = int(c.parent[j])
    sees = torch.cat([torch.ones(c.T, c.S, dtype=torch.bool, device="cuda"), sees], 1)
    want = torch.empty(c.T, c.heads, 128, dtype=torch.float64, device="cuda")
    reach = torch.empty(c.T, c.heads, 128, dtype=torch.float64, device="cuda")   # sum of p |v|: what an error of p counts for
    for h in range(c.heads):
        keys, values = torch.cat([c.k[h, :c.S].double(), kn[:, h]]), torch.cat([c.v[h, :, :c.S].double().t(), vn[:, h]])
        p = torch.softmax((q[:, h] @ keys.t().contiguous() / 128 ** 0.5).masked_fill(~sees, float("-inf")), 1)
        want[:, h], reach[:, h] = p @ values, p @ values.abs()
    want, reach = want.reshape(c.T, c.H), reach.reshape(c.T, c.H)
    # The output is off by 2^-8 of reach at most (weights p in 16 bits, 2^-9 of each and of their sum), rounded to bf16 (2^-9 of it), then to
    # half a step of 1/127 of the row's largest value, which is off by the same; x' - x takes two float32 roundings of x' on top.
    off = 2.0 ** -8 * reach + 2.0 ** -9 * want.abs()
    step = (want.abs() + off).amax(1, keepdim=True) / 127
    assert ((got - want).abs() <= off + 0.51 * step + 2.0 ** -23 * (c.x.double().abs() + want.abs())).all()
    assert want.abs().max() > 0.1


def test_feed_forward_block(case):
    c = case
    down = c.bf16(c.H, c.F)
    _, h, _, _, layer = c.run(c.weights | dict(wo=torch.zeros(c.H, c.H, dtype=torch.bfloat16, device="cuda"), w_down=down))
    w = c.weights
    gu = c.product(*c.rows(w["g_ffn"]), layer["w_gate_up"], layer["s_gate_up"], w["w_gate"], w["w_up"])
    q, s = torch.empty(c.T, c.F, dtype=torch.int8, device="cuda"), torch.empty(c.T, device="cuda")
    cats.cats_swiglu_quantize(gu, q, s)
    assert gu.abs().max() < 20
    g, u = np.split(f64(gu), 2, 1)
    check_rows(g / (1 + np.exp(-g)) * u, q, s, D)
    y = c.product(q, s, layer["w_down"], layer["s_down"], down)
    # the same bytes are multiplied; up to three pieces of the inner length, three roundings each and two of their sum, where the operator
    # has three of all, and one of x + y: |piece| <= 2 max|y|
    assert ((h - (c.x + y)).abs().max() <= 2.0 ** -24 * (34 * y.abs().max() + 2 * h.abs().max())).item()
    assert y.abs().max() > 0.5
