"""Decoder layers in 8 bits (cats_verify_layers_quantized) against the layer's definition in 64 bits: rows quantised where
the operators quantise them, rotation at ctx_len + depth, attention over the context and each node's ancestors.

The reference follows the kernel's roundings that are part of the definition (8-bit rows, the attention output in bf16 in front of
them); what is left apart is float32 arithmetic and the 16-bit queries, keys and values of the call's own rows (2^-17 each), which now
and then move a value over a rounding border: one step of 1/127 of a row's largest value in one of its inputs, far inside the
2e-2 of a tensor's largest value that whole layers are held to here."""
import numpy as np
import pytest
import torch

import paper_2605_11186_amd as cats
import synth
from gpu_common import REL_TOL, Pair, bf16_to_f32_np, rel_err, to_dev_bf16

pytestmark = pytest.mark.gpu

WIDE = synth.ModelDims(2, 512, 4, 128, 1040, 1000)   # heads of 128; ffn not a multiple of a product's step


def quantized(v):
    top = np.maximum(np.abs(v).max(1, keepdims=True), 127 * 2.0 ** -126)
    return np.rint(v * 127 / top) * (top / 127)


def to_bf16(v):
    return torch.from_numpy(v).to(torch.bfloat16).double().numpy()


def norm(x, gain, eps):
    return x / np.sqrt((x * x).mean(1, keepdims=True) + eps) * gain


def weights_of(d, seed, layer):
    """The quantised layer on the device, and its matrices' values."""
    w = {k: to_dev_bf16(v) for k, v in synth.layer_weights(d, seed, layer).items()}
    ref = {k: quantized(w[k].double().cpu().numpy()) for k in cats.MATRIX_FIELDS}
    ref |= {k: w[k].double().cpu().numpy() for k in ("g_attn", "g_ffn")}
    return cats.quantize_layer(w), ref


def reference(d, x, layers, kc, vc, ctx_len, parent, depth):
    """x [T][H]; kc, vc [layer][ctx rows][H]: returns the updated rows and each layer's new keys and values."""
    T, nh, hd = len(parent), d.n_heads, d.head_dim
    pos = ctx_len + np.asarray(depth, dtype=np.float64)
    ang = pos[:, None] * d.rope_base ** (-2.0 * np.arange(hd // 2) / hd)
    cos, sin = np.cos(ang)[:, None], np.sin(ang)[:, None]
    sees = np.zeros((T, T), dtype=bool)
    for i in range(T):
        j = i
        while j >= 0:
            sees[i, j] = True
            j = parent[j]
    new = []

    def rotate(v):
        v = v.reshape(T, nh, hd)
        a, b = v[..., : hd // 2], v[..., hd // 2:]
        return np.concatenate([a * cos - b * sin, a * sin + b * cos], -1)

    for l, w in enumerate(layers):
        h = quantized(norm(x, w["g_attn"], d.rms_eps))
        q, k, v = rotate(h @ w["wq"].T), rotate(h @ w["wk"].T), (h @ w["wv"].T).reshape(T, nh, hd)
        keys = np.concatenate([kc[l][:ctx_len].reshape(-1, nh, hd), k])
        values = np.concatenate([vc[l][:ctx_len].reshape(-1, nh, hd), v])
        s = np.einsum("tnd,knd->ntk", q, keys) / np.sqrt(hd)
        s[:, :, ctx_len:][:, ~sees] = -np.inf
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        o = np.einsum("ntk,knd->tnd", p, values).reshape(T, -1)
        x = x + quantized(to_bf16(o)) @ w["wo"].T
        h = quantized(norm(x, w["g_ffn"], d.rms_eps))
        g, u = h @ w["w_gate"].T, h @ w["w_up"].T
        x = x + quantized(g / (1 + np.exp(-g)) * u) @ w["w_down"].T
        new.append((k.reshape(T, -1), v.reshape(T, -1)))
    return x, new


class Model:
    def __init__(self, dims, seed, max_ctx=320, max_tree=128):
        self.d, self.max_ctx = dims, max_ctx
        both = [weights_of(dims, seed, l) for l in range(dims.n_layers)]
        self.dev, self.ref = [b[0] for b in both], [b[1] for b in both]
        self.arr = cats.quantized_layer_array(self.dev)
        self.ctx = cats.cats_create(cats.ModelDesc(dims.n_layers, dims.hidden, dims.n_heads, dims.head_dim, dims.ffn, dims.vocab,
                                                   max_ctx, max_tree, dims.rms_eps, dims.rope_base, 0))

    def caches(self, seed, ctx_len):
        """Random committed rows on both sides; all other rows are NaN on the device."""
        d = self.d
        kr, vr, ks, vs = [], [], [], []
        for l in range(d.n_layers):
            rows = [torch.from_numpy(synth.f32_from_bf16_bits(b)).cuda().to(torch.bfloat16)
                    for b in synth.random_kv_context(d, seed, l, ctx_len)]
            k, v = cats.kv_from_rows(*rows, d.n_heads, d.head_dim, self.max_ctx)
            k[:, ctx_len:] = float("nan")
            v[:, :, ctx_len:] = float("nan")
            ks.append(k), vs.append(v)
            kr.append(rows[0].double().cpu().numpy()), vr.append(rows[1].double().cpu().numpy())
        return kr, vr, ks, vs

    def close(self):
        torch.cuda.synchronize()
        cats.cats_destroy(self.ctx)


@pytest.fixture(scope="module", params=[synth.TINY, WIDE], ids=["heads64", "heads128"])
def model(request):
    m = Model(request.param, 3)
    yield m
    m.close()


def tree_of(nodes, seed):
    parent, depth = synth.random_tree(nodes, 9, seed)
    return np.asarray(parent, dtype=np.int32), np.asarray(depth, dtype=np.int32)


@pytest.mark.parametrize("nodes,ctx_len", [(1, 0), (1, 130), (2, 37), (15, 128), (63, 0), (63, 190), (128, 161)])
def test_layers(model, nodes, ctx_len):
    d = model.d
    parent, depth = tree_of(nodes, nodes)
    kr, vr, ks, vs = model.caches(5, ctx_len)
    x = synth.random_hidden(d, 6, nodes)
    hidden = torch.from_numpy(np.asarray(x, dtype=np.float32)).cuda()
    cats.cats_set_tree(model.ctx, np.zeros(nodes, np.int32), parent, depth)
    cats.cats_verify_layers_quantized(model.ctx, model.arr, 0, d.n_layers, hidden, cats.kv_array(ks, vs), ctx_len)
    torch.cuda.synchronize()
    want, new = reference(d, np.asarray(x, dtype=np.float64), model.ref, kr, vr, ctx_len, parent, depth)
    e = [rel_err(hidden.cpu().numpy(), want)]
    for l in range(d.n_layers):
        k, v = cats.kv_to_rows(ks[l], vs[l], ctx_len + nodes)
        assert np.array_equal(bf16_to_f32_np(k[:ctx_len]), kr[l].astype(np.float32))   # the context stays
        e += [rel_err(bf16_to_f32_np(k[ctx_len:]), new[l][0]), rel_err(bf16_to_f32_np(v[ctx_len:]), new[l][1])]
        assert torch.isnan(ks[l][:, ctx_len + nodes:]).all() and torch.isnan(vs[l][:, :, ctx_len + nodes:]).all()
    print(f"nodes {nodes} ctx {ctx_len}: hidden {e[0]:.1e}, keys and values at most {max(e[1:]):.1e}")
    assert max(e) <= REL_TOL
    # one layer after the other: the same bits
    again = torch.from_numpy(np.asarray(x, dtype=np.float32)).cuda()
    for l in range(d.n_layers):
        cats.cats_verify_layers_quantized(model.ctx, model.arr, l, l + 1, again, cats.kv_array(ks, vs), ctx_len)
    assert torch.equal(again, hidden)


@pytest.mark.parametrize("ctx_len", [127, 128, 1029, 2100, 4400])   # 1, 1, 9, 17 and 18 chunks of keys
@pytest.mark.parametrize("dims", [synth.TINY, WIDE], ids=["heads64", "heads128"])
def test_a_single_node_behind_long_contexts(dims, ctx_len):
    model = Model(dims, 3, max_ctx=4480, max_tree=1)
    try:
        kr, vr, ks, vs = model.caches(5, ctx_len)
        x = synth.random_hidden(dims, 6, 1)
        hidden = torch.from_numpy(np.asarray(x, dtype=np.float32)).cuda()
        cats.cats_set_tree(model.ctx, np.zeros(1, np.int32), *tree_of(1, 1))
        cats.cats_verify_layers_quantized(model.ctx, model.arr, 0, dims.n_layers, hidden, cats.kv_array(ks, vs), ctx_len)
        torch.cuda.synchronize()
        want, new = reference(dims, np.asarray(x, dtype=np.float64), model.ref, kr, vr, ctx_len, *tree_of(1, 1))
        e = [rel_err(hidden.cpu().numpy(), want)]
        for l in range(dims.n_layers):
            k, v = cats.kv_to_rows(ks[l], vs[l], ctx_len + 1)
            assert np.array_equal(bf16_to_f32_np(k[:ctx_len]), kr[l].astype(np.float32))
            e += [rel_err(bf16_to_f32_np(k[ctx_len:]), new[l][0]), rel_err(bf16_to_f32_np(v[ctx_len:]), new[l][1])]
            assert torch.isnan(ks[l][:, ctx_len + 1:]).all() and torch.isnan(vs[l][:, :, ctx_len + 1:]).all()
        assert max(e) <= REL_TOL
    finally:
        model.close()


@pytest.mark.parametrize("hidden,ctx_len", [(2048, 700), (4096, 1500), (5120, 1000), (8192, 300), (8192, 1530), (8192, 1700)])
def test_a_single_node_as_the_root_of_two(hidden, ctx_len):
    """A single node's attention has kernels of its own up to a number of chunks: the root of a tree sees the same rows."""
    heads, ffn = hidden // 128, 1024
    gen = torch.Generator(device="cuda").manual_seed(23)

    def random(*shape, by=1.0):
        return torch.empty(*shape, device="cuda").normal_(0, by, generator=gen).to(torch.bfloat16)

    one = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
    layer = cats.quantize_layer(dict(wq=random(hidden, hidden, by=0.02), wk=random(hidden, hidden, by=0.02), wv=random(hidden, hidden, by=0.02),
                                     wo=random(hidden, hidden, by=0.02), w_gate=random(ffn, hidden, by=0.02), w_up=random(ffn, hidden, by=0.02),
                                     w_down=random(hidden, ffn, by=0.02), g_attn=one, g_ffn=one))
    ctx = cats.cats_create(cats.ModelDesc(1, hidden, heads, 128, ffn, 1000, 2048, 2, 1e-6, 1e4, 0))
    try:
        k0, v0 = random(heads, 2048, 128), random(heads, 128, 2048)
        x = torch.empty(2, hidden, device="cuda").normal_(generator=gen)
        rows = []
        for nodes in (1, 2):
            k, v, h = k0.clone(), v0.clone(), x[:nodes].clone()
            cats.cats_set_tree(ctx, np.zeros(nodes, np.int32), np.asarray([-1, 0][:nodes], np.int32), np.arange(nodes, dtype=np.int32))
            cats.cats_verify_layers_quantized(ctx, cats.quantized_layer_array([layer]), 0, 1, h, cats.kv_array([k], [v]), ctx_len)
            torch.cuda.synchronize()
            rows.append([t.float().cpu().numpy() for t in (h[0] - x[0], k[:, ctx_len], v[:, :, ctx_len])])
        assert max(rel_err(a, b) for a, b in zip(*rows)) <= REL_TOL
    finally:
        torch.cuda.synchronize()
        cats.cats_destroy(ctx)


# hidden, feed-forward columns and nodes at which the output and down products come in 2 and 3 pieces (test_quant_choice checks that)
PIECES = [(4096, 11008, 63, (1, 2)), (5120, 13824, 63, (2, 3)), (4096, 11008, 128, (2, 2)), (2048, 8192, 40, (1, 2)),
          (7168, 1024, 90, (3, 1))]


@pytest.mark.parametrize("zero", ["wo", "w_down"])
@pytest.mark.parametrize("hidden,ffn,nodes", [p[:3] for p in PIECES])
def test_products_in_pieces(hidden, ffn, nodes, zero):
    """A layer over a tree and over its first 16 nodes, for which no product is cut.  With an output product of zeros the down product
    has the same bytes to multiply in both, in all rows; with a down product of zeros the output product has for the root, which
    behind no context sees itself alone.  So the rows differ by float32 roundings: for each of at most three pieces p three in the
    scales and two in the sum, three for the whole product y, one each where x comes on top.  y and p are sums of random signs, |p| <= 2
    max|y| = 2 Y for certain: 2^-24 (5 * 3 * 2 Y + 3 Y + 2 max|h|), Y <= max|h| + max|x| <= 2 max|h| or it is smaller still: 68 * 2^-24."""
    heads = hidden // 128
    gen = torch.Generator(device="cuda").manual_seed(29)

    def random(*shape, by=0.02):
        return torch.empty(*shape, device="cuda").normal_(0, by, generator=gen).to(torch.bfloat16)

    # gains at an odd multiple of two bytes make the norms read value by value
    one = torch.ones(hidden + 1, dtype=torch.bfloat16, device="cuda")[zero == "w_down":][:hidden]
    weights = dict(wq=random(hidden, hidden), wk=random(hidden, hidden), wv=random(hidden, hidden), wo=random(hidden, hidden),
                   w_gate=random(ffn, hidden), w_up=random(ffn, hidden), w_down=random(hidden, ffn), g_attn=one, g_ffn=one)
    weights[zero].zero_()
    layer, ctx_len = cats.quantize_layer(weights), 150 if zero == "wo" else 0
    ctx = cats.cats_create(cats.ModelDesc(1, hidden, heads, 128, ffn, 1000, 320, 128, 1e-6, 1e4, 0))
    try:
        k, v = random(heads, 320, 128, by=1), random(heads, 128, 320, by=1)
        x = torch.empty(nodes, hidden, device="cuda").normal_(generator=gen)
        parent, depth = tree_of(nodes, 7)
        rows = []
        for n in (nodes, 16):
            h = x[:n].clone()
            cats.cats_set_tree(ctx, np.zeros(n, np.int32), parent[:n], depth[:n])
            cats.cats_verify_layers_quantized(ctx, cats.quantized_layer_array([layer]), 0, 1, h, cats.kv_array([k], [v]), ctx_len)
            torch.cuda.synchronize()
            rows.append(h[:16 if zero == "wo" else 1])
        assert torch.isfinite(rows[0]).all() and (rows[0] - x[:len(rows[0])]).abs().max() > 1
        assert (rows[0] - rows[1]).abs().max() <= 68 * 2.0 ** -24 * rows[1].abs().max()
    finally:
        torch.cuda.synchronize()
        cats.cats_destroy(ctx)


@pytest.mark.parametrize("nodes", [1, 20, 63, 128])
def test_a_call_whose_weights_pass_the_caches(nodes):
    """Two layers of 202 MB of weights in one call (past the caches) and one after the other (through them): the same bits."""
    d = synth.V7B
    gen = torch.Generator(device="cuda").manual_seed(17)

    def matrix(rows, cols):
        return torch.empty(rows, cols, device="cuda").normal_(0, 0.02, generator=gen).to(torch.bfloat16)

    H, F, one = d.hidden, d.ffn, torch.ones(d.hidden, dtype=torch.bfloat16, device="cuda")
    layers = [cats.quantize_layer(dict(wq=matrix(H, H), wk=matrix(H, H), wv=matrix(H, H), wo=matrix(H, H), w_gate=matrix(F, H),
                                       w_up=matrix(F, H), w_down=matrix(H, F), g_attn=one, g_ffn=one)) for _ in range(2)]
    ctx = cats.cats_create(cats.ModelDesc(2, H, d.n_heads, d.head_dim, F, d.vocab, 256, 128, d.rms_eps, d.rope_base, 0))
    try:
        parent, depth = tree_of(nodes, 4)
        cats.cats_set_tree(ctx, np.zeros(nodes, np.int32), parent, depth)
        ks = [torch.zeros(d.n_heads, 256, d.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        vs = [torch.zeros(d.n_heads, d.head_dim, 256, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        arr, kv = cats.quantized_layer_array(layers), cats.kv_array(ks, vs)
        x = torch.empty(nodes, H, device="cuda").normal_(generator=gen)
        both, each = x.clone(), x.clone()
        cats.cats_verify_layers_quantized(ctx, arr, 0, 2, both, kv, 40)
        rows = [t.clone() for t in ks + vs]
        for l in range(2):
            cats.cats_verify_layers_quantized(ctx, arr, l, l + 1, each, kv, 40)
        assert torch.isfinite(both).all() and not torch.equal(both, x)
        assert torch.equal(both, each) and all(torch.equal(a, b) for a, b in zip(rows, ks + vs))
    finally:
        torch.cuda.synchronize()
        cats.cats_destroy(ctx)


def test_whole_step_beside_the_bf16_step():
    """Embedding rows, 8-bit layers, LM head, acceptance and roll-back: the step of a target in 8 bits.  Its logits are near those of
    the bf16 target (8 bits a row: some per cent), and the context serves both kinds of step."""
    d = synth.TINY
    pair = Pair(d, 7, max_ctx=192, max_tree=16)
    try:
        S = 128
        kc, vc = pair.oracle_cache_random(7, S)
        parent, depth = synth.complete_binary_tree(3)
        T = len(parent)
        tok = synth.distinct_sibling_tokens(parent, d.vocab, 7)
        layers = [cats.quantize_layer(w) for w in pair.d_layers]
        arr = cats.quantized_layer_array(layers)
        cats.cats_set_tree(pair.ctx, tok, parent, depth)

        def quantized_step():
            ks, vs = pair.device_cache_from_oracle(kc, vc, S)
            kv = cats.kv_array(ks, vs)
            hidden = pair.d_embed[torch.from_numpy(np.asarray(tok)).cuda().long()].float()
            logits, amax = torch.empty(T, d.vocab, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda")
            cats.cats_verify_layers_quantized(pair.ctx, arr, 0, d.n_layers, hidden, kv, S)
            cats.cats_lm_head_argmax(pair.ctx, hidden, pair.d_final["g_final"], pair.d_final["w_lm"], amax, logits_out=logits)
            res = cats.AcceptResult()
            cats.cats_accept_and_compact(pair.ctx, amax, kv, 0, d.n_layers, S, pair.res_dev, out_host=res)
            return hidden, logits, amax, res.as_dict(), [k[:, : res.new_ctx_len].clone() for k in ks]

        def bf16_step():
            ks, vs = pair.device_cache_from_oracle(kc, vc, S)
            logits = torch.empty(T, d.vocab, device="cuda")
            cats.cats_verify_tree(pair.ctx, pair.layers_arr, 0, pair.L, pair.d_embed, None, pair.d_final["g_final"],
                                  pair.d_final["w_lm"], cats.kv_array(ks, vs), S, pair.res_dev, logits_out=logits)
            return logits

        plain = bf16_step()
        first = quantized_step()
        assert torch.equal(bf16_step(), plain)   # the 8-bit step leaves nothing behind that the bf16 step reads
        second = quantized_step()
        for a, b in zip(first[:3], second[:3]):
            assert torch.equal(a, b)
        assert first[3] == second[3] == pair.oracle.accept(tok, parent, depth, first[2].cpu().numpy(), S)
        assert all(torch.equal(a, b) for a, b in zip(first[4], second[4]))
        e = rel_err(first[1].cpu().numpy(), plain.cpu().numpy())
        print(f"logits of the 8-bit step, off the bf16 step by {e:.1e} of the largest")
        assert e <= 0.1
    finally:
        pair.close()


def test_captured_and_replayed(model):
    d, nodes, ctx_len = model.d, 31, 70
    parent, depth = tree_of(nodes, 8)
    _, _, ks, vs = model.caches(9, ctx_len)
    x = torch.from_numpy(np.asarray(synth.random_hidden(d, 10, nodes), dtype=np.float32)).cuda()
    cats.cats_set_tree(model.ctx, np.zeros(nodes, np.int32), parent, depth)
    kv = cats.kv_array(ks, vs)

    def eager():
        h = x.clone()
        cats.cats_verify_layers_quantized(model.ctx, model.arr, 0, d.n_layers, h, kv, ctx_len)
        torch.cuda.synchronize()
        return h

    want = eager()
    h, g = x.clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        cats.cats_verify_layers_quantized(model.ctx, model.arr, 0, d.n_layers, h, kv, ctx_len, stream=torch.cuda.current_stream())
    for i in range(4):
        h.copy_(x)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(h, want)
        assert torch.equal(eager(), want)


def test_refusals(model):
    d = model.d
    lib, (_, _, ks, vs) = cats.library(), model.caches(5, 64)
    kv = cats.kv_array(ks, vs)
    fresh = cats.cats_create(cats.ModelDesc(d.n_layers, d.hidden, d.n_heads, d.head_dim, d.ffn, d.vocab, 128, 16, d.rms_eps,
                                            d.rope_base, 0))
    hidden = torch.zeros(8, d.hidden, device="cuda")

    def status(ctx=None, layers=model.arr, lb=0, le=d.n_layers, h=hidden.data_ptr(), kv_arr=kv, ctx_len=64):
        return lib.cats_verify_layers_quantized(model.ctx if ctx is None else ctx, layers, lb, le, h, kv_arr, ctx_len, None)

    assert lib.cats_verify_layers_quantized(None, model.arr, 0, 1, hidden.data_ptr(), kv, 64, None) == cats.CATS_EINVAL
    assert status(ctx=fresh) == cats.CATS_ESTATE
    parent, depth = tree_of(8, 8)
    cats.cats_set_tree(model.ctx, np.zeros(8, np.int32), parent, depth)
    assert status(ctx_len=model.max_ctx - 7) == cats.CATS_ECAPACITY
    for bad in (dict(ctx_len=-1), dict(lb=-1), dict(le=d.n_layers + 1), dict(lb=1, le=0), dict(layers=None), dict(kv_arr=None),
                dict(h=None), dict(h=hidden.data_ptr() + 4)):
        assert status(**bad) == cats.CATS_EINVAL, bad
    for field, _ in cats.QuantizedLayer._fields_:
        for off in (None, 1):
            arr = cats.quantized_layer_array(model.dev)
            setattr(arr[1], field, None if off is None else getattr(arr[1], field) + off)
            assert status(layers=arr) == cats.CATS_EINVAL, (field, off)
            assert status(layers=arr, le=1) == cats.CATS_OK   # the layer is not in the range
    assert status(lb=1, le=1, layers=None, kv_arr=None) == cats.CATS_OK
    torch.cuda.synchronize()
    cats.cats_destroy(fresh)
