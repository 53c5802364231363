"""Performance cases of the decoder layer's operators in 8-bit integers.

A target model whose weights and activations are held in 8 bits runs its layers on four operators, and each case
here is one call of one of them, as a program that runs such a layer makes it:

  rmsnorm   x' = x + delta, v = x' / sqrt(mean(x'^2) + eps) * gain, every row of v in 8 bits with one scale
  linear    y[t][n] = (sum over k of xq[t][k] wq[n][k]) * x_scale[t] * w_scale[n]
  swiglu    v = g / (1 + exp(-g)) * u for rows g | u, every row of v in 8 bits with one scale
  quantize  every row of a matrix in 8 bits with one scale

A row v in 8 bits: q = 127 v / max|v| rounded to whole numbers (ties to even), scale = max|v| / 127, never below 2^-126
(zeros, and rows next to nothing).  The values that q and scale stand for are returned in bfloat16, whose 8 bits are what
they carry.

Shapes are those of the benchmark's 7B and 13B models and of the tests' small one; `draw` gives more of the same
ranges.  Rows: tree nodes of a verification step (1 to 128), or the tokens of a prompt.
"""
import math

import torch

own = False

EPS = 1e-6
TINY = 2.0 ** -126  # the smallest scale: a row of zeros has it


def listed():
    return [
        # the tests' small model, one token: output projection; nothing but latency
        dict(name="linear_tiny_t1", op="linear", rows=1, cols=256, inner=256, out="f32"),
        # one token of the 7B model (plain decoding, a step of the draft loop): gate and up projections
        dict(name="linear_7b_gate_up_t1", op="linear", rows=1, cols=22016, inner=4096, out="bf16"),
        # the benchmark's 63-node tree: gate and up projections
        dict(name="linear_7b_gate_up_t63", op="linear", rows=63, cols=22016, inner=4096, out="bf16"),
        # the largest tree on the 13B model: q, k and v projections, kept in 32 bits for the rotation behind them
        dict(name="linear_13b_qkv_t128", op="linear", rows=128, cols=15360, inner=5120, out="f32"),
        # sizes that no tile divides
        dict(name="linear_odd_t77", op="linear", rows=77, cols=2003, inner=1001, out="f32"),
        # a prompt of 4096 tokens through the 7B model's down projection
        dict(name="linear_7b_down_t4096", op="linear", rows=4096, cols=4096, inner=11008, out="bf16"),
        # one token of the 7B model
        dict(name="rmsnorm_7b_t1", op="rmsnorm", rows=1, cols=4096, delta="f32"),
        # a prompt of 8192 tokens through the 13B model's norm
        dict(name="rmsnorm_13b_t8192", op="rmsnorm", rows=8192, cols=5120, delta="bf16"),
        # the 63-node tree
        dict(name="swiglu_7b_t63", op="swiglu", rows=63, cols=11008, src="bf16"),
        # a prompt on the 13B model
        dict(name="swiglu_13b_t4096", op="swiglu", rows=4096, cols=13824, src="bf16"),
        # attention output of the largest tree on the 13B model
        dict(name="quantize_13b_t128", op="quantize", rows=128, cols=5120, src="bf16"),
        # a weight matrix by output channel: the 7B model's LM head
        dict(name="quantize_7b_lm_head", op="quantize", rows=32000, cols=4096, src="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "rmsnorm", "swiglu", "quantize"])
    while True:
        rows = _log_int(rng, 1, 128) if rng.random() < 0.6 else _log_int(rng, 128, 8192)
        cols = rng.choice([256, 688, 4096, 5120, 11008, 13824]) if rng.random() < 0.5 else _log_int(rng, 16, 16384)
        if op == "linear":
            inner = rng.choice([256, 688, 4096, 5120, 11008, 13824]) if rng.random() < 0.5 else _log_int(rng, 16, 16384)
            if rows * cols * inner <= 4096 * 4096 * 11008:
                return dict(op=op, rows=rows, cols=cols, inner=inner, out=rng.choice(["f32", "bf16"]))
        elif rows * cols <= 8192 * 5120:
            if op == "rmsnorm":
                return dict(op=op, rows=rows, cols=cols, delta=rng.choice(["none", "f32", "bf16"]))
            return dict(op=op, rows=rows, cols=cols, src=rng.choice(["f32", "bf16"]))


_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _round16(n):
    return (n + 15) // 16 * 16


def _normal(gen, rows, cols, dtype=torch.float32):
    """Rows that start at multiples of 16 elements, whatever the number of columns."""
    t = torch.empty(rows, _round16(cols), dtype=torch.float32, device="cuda").normal_(generator=gen)
    return t.to(dtype)[:, :cols]


def _int8(gen, rows, cols):
    """Values as rows with a scale of their own hold them: normal, the largest near the end of the range."""
    t = torch.empty(rows, _round16(cols), dtype=torch.float32, device="cuda").normal_(0.0, 32.0, generator=gen)
    return t.round_().clamp_(-127, 127).to(torch.int8)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    op, R, C = case["op"], case["rows"], case["cols"]
    s = dict(op=op)

    def uniform(n, lo, hi):
        return torch.empty(n, dtype=torch.float32, device="cuda").uniform_(lo, hi, generator=gen)

    if op == "linear":
        K = case["inner"]
        s["x"], s["x_scale"] = _int8(gen, R, K), uniform(R, 0.005, 0.05)
        s["w"], s["w_scale"] = _int8(gen, C, K), uniform(C, 2e-4, 1e-3)
        s["type"] = _TYPES[case["out"]]
        if own:
            import paper_2605_11186_amd as cats
            s["w"] = cats.cats_pack_quantized_matrix(s["w"])   # laid out once, as the model is loaded
            s["y"] = torch.empty(R, C, dtype=s["type"], device="cuda")
        return s
    if op == "rmsnorm":
        # a residual stream: a few channels are much larger than the others
        s["x"] = _normal(gen, R, C)
        s["x"] *= 1.0 + 20.0 * (uniform(C, 0.0, 1.0) < 0.004)
        s["delta"] = None if case["delta"] == "none" else _normal(gen, R, C, _TYPES[case["delta"]])
        s["gain"] = (1.0 + 0.02 * torch.empty(C, device="cuda").normal_(generator=gen)).to(torch.bfloat16)
    elif op == "swiglu":
        s["gate_up"] = _normal(gen, R, 2 * C, _TYPES[case["src"]])
    else:
        s["src"] = _normal(gen, R, C, _TYPES[case["src"]])
    if own:
        s["q"] = torch.empty(R, _round16(C), dtype=torch.int8, device="cuda")[:, :C]
        s["scale"] = torch.empty(R, dtype=torch.float32, device="cuda")
        s["values"] = torch.empty(R, C, dtype=torch.bfloat16, device="cuda")
        if s.get("delta") is not None:
            s["x_out"] = torch.empty(R, C, dtype=torch.float32, device="cuda")
    return s


def _plain_rows(v):
    """Rows in 8 bits: the values that they stand for, and their scales."""
    top = v.abs().amax(1).clamp(min=127.0 * TINY)
    q = torch.round(v * 127.0 / top[:, None])
    scale = top / 127.0
    return (q * scale[:, None]).to(torch.bfloat16), scale


def run(state):
    op = state["op"]
    if own:
        import paper_2605_11186_amd as cats
        stream = torch.cuda.current_stream()
        if op == "linear":
            cats.cats_quantized_linear(state["x"], state["x_scale"], state["w"], state["w_scale"], state["y"], stream=stream)
            return state["y"]
        q, scale = state["q"], state["scale"]
        if op == "rmsnorm":
            cats.cats_rmsnorm_quantize(state["x"], state["gain"], EPS, q, scale, delta=state["delta"],
                                   x_out=state.get("x_out"), stream=stream)
            return (state.get("x_out"), torch.mul(q, scale[:, None], out=state["values"]), scale)
        if op == "swiglu":
            cats.cats_swiglu_quantize(state["gate_up"], q, scale, stream=stream)
        else:
            cats.cats_quantize_rows(state["src"], q, scale, stream=stream)
        return (torch.mul(q, scale[:, None], out=state["values"]), scale)
    if op == "linear":
        acc = torch.matmul(state["x"].float(), state["w"].float().t())
        return (acc * state["x_scale"][:, None] * state["w_scale"]).to(state["type"])
    if op == "rmsnorm":
        x = state["x"] if state["delta"] is None else state["x"] + state["delta"].float()
        norm = torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
        values, scale = _plain_rows(x / norm * state["gain"].float())
        return (None if state["delta"] is None else x, values, scale)
    if op == "swiglu":
        g, u = state["gate_up"].float().chunk(2, 1)
        return _plain_rows(g / (1.0 + torch.exp(-g)) * u)
    return _plain_rows(state["src"].float())


def work(case):
    R, C = case["rows"], case["cols"]
    size = {"f32": 4, "bf16": 2, "none": 0}
    if case["op"] == "linear":
        K = case["inner"]
        return dict(bytes=R * K + C * K + 4 * R + 4 * C + size[case["out"]] * R * C, flops=2 * R * C * K)
    if case["op"] == "rmsnorm":
        d = case["delta"]
        return dict(bytes=R * C * (4 + size[d] + (0 if d == "none" else 4) + 1) + 2 * C + 4 * R, flops=8 * R * C)
    if case["op"] == "swiglu":
        return dict(bytes=R * C * (2 * size[case["src"]] + 1) + 4 * R, flops=10 * R * C)
    return dict(bytes=R * C * (size[case["src"]] + 1) + 4 * R, flops=4 * R * C)


def exact(case, seed):
    global own
    was, own = own, False   # the inputs alone: no operator's buffers
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "linear":
        # whole numbers below 2^53: every partial sum is exact
        y = s["x"].double() @ s["w"].double().t()
        y *= s["x_scale"].double()[:, None]
        y *= s["w_scale"].double()[None, :]
        return y
    x = None
    if case["op"] == "rmsnorm":
        v = s["x"].double()
        if s["delta"] is not None:
            v = v + s["delta"].double()
            x = v
        v = v * (v.pow(2).sum(1, keepdim=True) / case["cols"] + EPS).rsqrt() * s["gain"].double()
    elif case["op"] == "swiglu":
        both = s["gate_up"].double()
        g, u = both[:, :case["cols"]], both[:, case["cols"]:]
        v = g * u / (1.0 + torch.exp(-g))
    else:
        v = s["src"].double()
    step = torch.maximum(v.abs().max(1).values / 127.0, torch.tensor(TINY, dtype=torch.float64, device=v.device))
    values = (v / step[:, None]).round() * step[:, None]
    return (x, values, step) if case["op"] == "rmsnorm" else (values, step)
