"""Timed cases of the 8-bit building blocks: rows normalised into 8 bits, rows and weights put into 8 bits, the
matrix product of the two, and a feed-forward branch made of them.

8-bit tensors are e4m3 elements with one power-of-two scale (E8M0) for every 128 consecutive elements of a row, or for
every 128 x 128 block of a weight.  The scales of a row are padded to whole 32-bit words (4 * ceil(columns / 512) bytes).

  rms       h = x[rows] + add[rows];  h * gain / sqrt(mean(h^2) + eps) in 8 bits, and h itself where asked
  quantize  rows (1 x 128) or a weight (128 x 128) in 8 bits
  linear    act(A W^T + bias), A and W in 8 bits, the result in bf16 or in 8 bits
  ffn       rms, linear with GELU and 8-bit result, linear: the feed-forward branch of a block

Shapes: the repository's 2B-shaped block (1920 channels, FFN 7680, 17550 video + 226 text tokens, 4485 of them
refreshed) and generic ones.  Activations are N(0, 1) with a few channels 20 times as large, as normalised streams of
trained models have them; weights N(0, 0.02), gains around 1.
"""
import math

import torch

own = False

HIDDEN, FFN, TOKENS, TEXT, REFRESHED = 1920, 7680, 17776, 226, 4485
BLOCK = 128
EPS = 1e-6


def _rms(name, rows, hidden, fp32, add, keep_sum, of=0):
    """`of`: the rows are listed, out of so many."""
    return {"name": name, "op": "rms", "rows": rows, "hidden": hidden, "fp32": fp32, "add": add, "sum": keep_sum, "of": of}


def _quantize(name, rows, cols, fp32, block_rows):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "fp32": fp32, "block_rows": block_rows}


def _linear(name, m, n, k, gelu, quantized):
    return {"name": name, "op": "linear", "m": m, "n": n, "k": k, "gelu": gelu, "quantized": quantized}


def listed():
    return [
        # one token: launch and latency are all there is
        _rms("rms_token", 1, HIDDEN, True, True, True),
        # the refreshed rows of a cached step, gathered from the fp32 stream (which is updated elsewhere)
        _rms("rms_refreshed", REFRESHED, HIDDEN, True, True, False, of=TOKENS),
        # every row of a full step: the branch is added to the stream on the way
        _rms("rms_all", TOKENS, HIDDEN, True, True, True),
        # a mid-size model with a bf16 stream: odd row count, a width that ends inside a block
        _rms("rms_odd", 1543, 1008, False, False, False),
        # the attention output of a full step, before the out-projection
        _quantize("quantize_rows", TOKENS, HIDDEN, False, 1),
        # a weight, when a model is loaded
        _quantize("quantize_weight", FFN, HIDDEN, False, 128),
        # one token through a wide layer (embeddings of the timestep): bound by the weight's bytes
        _linear("linear_token", 1, FFN, HIDDEN, True, False),
        # the text rows through FFN2: few rows, long k
        _linear("linear_text", TEXT, HIDDEN, FFN, False, False),
        # QKV of the refreshed rows
        _linear("linear_refreshed_qkv", REFRESHED, 3 * HIDDEN, HIDDEN, False, False),
        # FFN1 and FFN2 of all rows: the largest products of the block
        _linear("linear_all_ffn1", TOKENS, FFN, HIDDEN, True, True),
        _linear("linear_all_ffn2", TOKENS, HIDDEN, FFN, False, False),
        # the feed-forward branch of the refreshed rows, the operators in a row
        {"name": "ffn_refreshed", "op": "ffn", "rows": REFRESHED, "hidden": HIDDEN, "ffn": FFN, "fp32": True, "of": TOKENS},
    ]


def _log(rng, low, high):
    return math.exp(rng.uniform(math.log(low), math.log(high)))


def _width(rng, low, high):
    return 16 * max(1, round(_log(rng, low, high) / 16))


def draw(rng):
    """Another case: 1 to 17776 rows, widths of 64 to 8192 in steps of 16, no product larger than the largest listed."""
    op = rng.choice(("rms", "rms", "quantize", "linear", "linear", "linear", "ffn"))
    rows = round(_log(rng, 1, TOKENS))
    if op == "rms":
        hidden = _width(rng, 64, HIDDEN if rows > 8000 else 8192)
        return {"op": op, "rows": rows, "hidden": hidden, "fp32": rng.random() < 0.6, "add": rng.random() < 0.7,
                "sum": rng.random() < 0.5, "of": rng.choice((0, rows + rng.randint(0, rows)))}
    if op == "quantize":
        return {"op": op, "rows": rows, "cols": _width(rng, 64, HIDDEN if rows > 8000 else 8192), "fp32": rng.random() < 0.3,
                "block_rows": rng.choice((1, 1, 128))}
    if op == "ffn":
        hidden = _width(rng, 64, HIDDEN)
        return {"op": op, "rows": min(rows, TOKENS // 2), "hidden": hidden, "ffn": 4 * hidden, "fp32": rng.random() < 0.6,
                "of": rng.choice((0, TOKENS))}
    n, k = _width(rng, 64, 8192), _width(rng, 64, 8192)
    while rows * n * k > TOKENS * HIDDEN * FFN or rows * max(n, k) > TOKENS * FFN:
        rows = max(1, rows // 2)
    return {"op": op, "m": rows, "n": n, "k": k, "gelu": rng.random() < 0.4, "quantized": rng.random() < 0.4}


# ---- the format, in elementary operations ---------------------------------------------------------

def _pitch(cols):
    return (cols + 511) // 512 * 4


def _quantized(v, block_rows):
    """v (fp32) as (e4m3 elements, E8M0 scales [row blocks, _pitch])."""
    rows, cols = v.shape
    row_blocks, col_blocks = -(-rows // block_rows), -(-cols // BLOCK)
    padded = torch.zeros(row_blocks * block_rows, col_blocks * BLOCK, dtype=torch.float32, device=v.device)
    padded[:rows, :cols] = v
    blocks = padded.view(row_blocks, block_rows, col_blocks, BLOCK)
    size = blocks.abs()
    largest = torch.where(torch.isfinite(size), size, torch.zeros_like(size)).amax(dim=(1, 3))
    mantissa, exponent = torch.frexp(largest)                    # mantissa in [1/2, 1): 448 is 7/8 * 2^9
    e = exponent - 9 + (mantissa > 0.875).to(exponent.dtype)
    e = torch.where(largest == 0, torch.zeros_like(e), e).clamp(-127, 127)
    q = (blocks * torch.ldexp(torch.ones_like(largest), -e)[:, None, :, None]).to(torch.float8_e4m3fn)
    scales = torch.full((row_blocks, _pitch(cols)), 127, dtype=torch.uint8, device=v.device)
    scales[:, :col_blocks] = (e + 127).to(torch.uint8)
    q = q.view(torch.uint8).reshape(row_blocks * block_rows, -1)[:rows, :cols].contiguous().view(torch.float8_e4m3fn)
    return q, scales.view(torch.float8_e8m0fnu)


def _values(q, scales, dtype=torch.float32):
    """What the elements stand for."""
    rows, cols = q.shape
    e = scales.view(torch.uint8).to(torch.int32) - 127
    factor = torch.ldexp(torch.ones(e.shape, dtype=dtype, device=e.device), e)
    factor = factor.repeat_interleave(BLOCK, dim=1)[:, :cols]
    if scales.shape[0] != rows:                                  # a weight
        factor = factor.repeat_interleave(BLOCK, dim=0)[:rows]
    return q.to(dtype) * factor


def _gelu(v):
    return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))


# ---- inputs ---------------------------------------------------------------------------------------

def _activations(rows, cols, gen):
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    x[:, torch.randint(0, cols, (max(1, cols // 200),), generator=gen, device="cuda")] *= 20.0
    return x


def _weight(n, k, gen):
    return _quantized((torch.randn(n, k, generator=gen, device="cuda") * 0.02).to(torch.bfloat16).float(), 128)


def _vector(n, gen, mean=0.0):
    return (torch.randn(n, generator=gen, device="cuda") * 0.02 + mean).to(torch.bfloat16)


def _room(rows, cols):
    return (torch.zeros(rows, cols, dtype=torch.float8_e4m3fn, device="cuda"),
            torch.zeros(rows, _pitch(cols), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu))


def _rms_inputs(case, gen, keep_sum, add):
    rows, hidden, of = case["rows"], case["hidden"], case["of"]
    dtype = torch.float32 if case["fp32"] else torch.bfloat16
    total = of if of else rows
    state = {"x": _activations(total, hidden, gen).to(dtype), "gain": _vector(hidden, gen, mean=1.0),
             "add": torch.randn(total, hidden, generator=gen, device="cuda").to(torch.bfloat16) if add else None,
             "rows": torch.randperm(total, generator=gen, device="cuda")[:rows].to(torch.int32) if of else None,
             "sum": torch.zeros(rows, hidden, dtype=dtype, device="cuda") if keep_sum else None}
    state["q"], state["scales"] = _room(rows, hidden)
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, state = case["op"], {"case": dict(case)}
    if op == "rms":
        state.update(_rms_inputs(case, gen, case["sum"], case["add"]))
    elif op == "quantize":
        rows, cols = case["rows"], case["cols"]
        x = _activations(rows, cols, gen) if case["block_rows"] == 1 else 0.02 * torch.randn(rows, cols, generator=gen, device="cuda")
        state["x"] = x if case["fp32"] else x.to(torch.bfloat16)
        state["q"], state["scales"] = _room(rows, cols)
        state["scales"] = state["scales"][:-(-rows // case["block_rows"])].contiguous()
    elif op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        state["a"], state["a_scales"] = _quantized(_activations(m, k, gen), 1)
        state["w"], state["w_scales"] = _weight(n, k, gen)
        state["bias"] = _vector(n, gen)
        state["scratch"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        if case["quantized"]:
            state["q"], state["scales"] = _room(m, n)
        else:
            state["c"] = torch.zeros(m, n, dtype=torch.bfloat16, device="cuda")
    else:
        rows, hidden, ffn = case["rows"], case["hidden"], case["ffn"]
        state.update(_rms_inputs(case, gen, False, True))
        state["w1"], state["w1_scales"] = _weight(ffn, hidden, gen)
        state["w2"], state["w2_scales"] = _weight(hidden, ffn, gen)
        state["bias1"], state["bias2"] = _vector(ffn, gen), _vector(hidden, gen)
        state["scratch"] = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        state["mid"], state["mid_scales"] = _room(rows, ffn)
        state["c"] = torch.zeros(rows, hidden, dtype=torch.bfloat16, device="cuda")
    return state


# ---- one pass -------------------------------------------------------------------------------------

def _plain_rms(s):
    h = s["x"] if s["rows"] is None else s["x"][s["rows"].long()]
    h = h.float()
    if s["add"] is not None:
        h = h + (s["add"] if s["rows"] is None else s["add"][s["rows"].long()]).float()
    y = h * torch.rsqrt((h * h).mean(dim=1, keepdim=True) + EPS) * s["gain"].float()
    q, scales = _quantized(y, 1)
    return q, scales, h


def _plain_linear(a, a_scales, w, w_scales, bias, gelu):
    v = torch.matmul(_values(a, a_scales), _values(w, w_scales).t()) + bias.float()
    return _gelu(v) if gelu else v


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if own:
        from paper_2508_17588_amd import binding as B
        if op == "rms":
            B.hero_gather_rms_fp8(s["x"], s["add"], s["rows"], case["rows"], s["gain"], EPS, s["q"], s["scales"], s["sum"])
            return {"q": s["q"], "scales": s["scales"], "sum": s["sum"]}
        if op == "quantize":
            B.hero_quantize_fp8(s["x"], s["q"], s["scales"], case["block_rows"])
            return {"q": s["q"], "scales": s["scales"]}
        if op == "linear" and case["quantized"]:
            B.hero_linear_fp8_quantized(s["a"], s["a_scales"], s["w"], s["w_scales"], s["bias"], s["q"], s["scales"],
                                        int(case["gelu"]), s["scratch"])
            return {"q": s["q"], "scales": s["scales"]}
        if op == "linear":
            B.hero_linear_fp8(s["a"], s["a_scales"], s["w"], s["w_scales"], s["bias"], s["c"], int(case["gelu"]), s["scratch"])
            return {"c": s["c"]}
        B.hero_gather_rms_fp8(s["x"], s["add"], s["rows"], case["rows"], s["gain"], EPS, s["q"], s["scales"])
        B.hero_linear_fp8_quantized(s["q"], s["scales"], s["w1"], s["w1_scales"], s["bias1"], s["mid"], s["mid_scales"], 1, s["scratch"])
        B.hero_linear_fp8(s["mid"], s["mid_scales"], s["w2"], s["w2_scales"], s["bias2"], s["c"], 0, s["scratch"])
        return {"c": s["c"]}
    if op == "rms":
        q, scales, h = _plain_rms(s)
        return {"q": q, "scales": scales, "sum": h.to(s["x"].dtype) if case["sum"] else None}
    if op == "quantize":
        q, scales = _quantized(s["x"].float(), case["block_rows"])
        return {"q": q, "scales": scales}
    if op == "linear":
        v = _plain_linear(s["a"], s["a_scales"], s["w"], s["w_scales"], s["bias"], case["gelu"])
        if case["quantized"]:
            q, scales = _quantized(v, 1)
            return {"q": q, "scales": scales}
        return {"c": v.to(torch.bfloat16)}
    q, scales, _ = _plain_rms(s)
    mid, mid_scales = _quantized(_plain_linear(q, scales, s["w1"], s["w1_scales"], s["bias1"], True), 1)
    return {"c": _plain_linear(mid, mid_scales, s["w2"], s["w2_scales"], s["bias2"], False).to(torch.bfloat16)}


def work(case):
    op = case["op"]
    if op == "rms":
        r, h, x = case["rows"], case["hidden"], 4 if case["fp32"] else 2
        per_element = x + 1 + (2 if case["add"] else 0) + (x if case["sum"] else 0)
        return {"bytes": r * h * per_element + r * _pitch(h) + 2 * h + (4 * r if case["of"] else 0), "flops": 5 * r * h}
    if op == "quantize":
        r, c = case["rows"], case["cols"]
        return {"bytes": r * c * ((4 if case["fp32"] else 2) + 1) + -(-r // case["block_rows"]) * _pitch(c), "flops": 2 * r * c}
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        out = m * n + m * _pitch(n) if case["quantized"] else 2 * m * n
        return {"bytes": m * k + n * k + m * _pitch(k) + -(-n // BLOCK) * _pitch(k) + 2 * n + out, "flops": 2 * m * n * k}
    r, h, f = case["rows"], case["hidden"], case["ffn"]
    return {"bytes": r * h * ((4 if case["fp32"] else 2) + 2) + 2 * h * f + 2 * r * h, "flops": 4 * r * h * f}


# ---- the definition in 64 bits --------------------------------------------------------------------

def _exact_values(q, scales, weight):
    v, rows = q.double(), q.shape[0]
    exponents = scales.view(torch.uint8).double() - 127.0
    for b in range(-(-q.shape[1] // 128)):
        f = torch.exp2(exponents[:, b])
        v[:, 128 * b:128 * b + 128] *= f[torch.arange(rows, device=q.device) // (128 if weight else 1)][:, None]
    return v


def _exact_scaled(y, block_rows):
    """y over the scales of its blocks, before any rounding, and the scales."""
    rows, cols = y.shape
    t = torch.empty_like(y)
    scales = torch.ones(-(-rows // block_rows), _pitch(cols), dtype=torch.float64, device=y.device)
    for b in range(-(-cols // 128)):
        part = y[:, 128 * b:128 * b + 128]
        largest = part.abs().amax(dim=1)
        if block_rows > 1:
            largest = torch.nn.functional.pad(largest, (0, -rows % block_rows)).view(-1, block_rows).amax(dim=1)
        _, e = torch.frexp(largest / 448.0)                      # 2^(e-1) <= largest / 448 < 2^e
        low = torch.exp2((e - 1).double())
        scale = torch.where(448.0 * low >= largest, low, 2.0 * low)
        scale = torch.where(largest == 0.0, torch.ones_like(scale), scale.clamp(2.0 ** -127, 2.0 ** 127))
        scales[:, b] = scale
        t[:, 128 * b:128 * b + 128] = part / scale[torch.arange(rows, device=y.device) // block_rows][:, None]
    return t, scales


def _exact_stored(y):
    """The values that y's rows stand for once they are held in 8 bits: what a next operator reads."""
    t, scales = _exact_scaled(y, 1)
    _, top = torch.frexp(t)
    step = torch.exp2((top - 1).clamp(min=-6).double() - 3.0)    # three fraction bits; subnormals below 2^-6
    return torch.round(t / step) * step * scales.repeat_interleave(128, dim=1)[:, :t.shape[1]]


def _exact_rms(s):
    h = s["x"].double()
    if s["add"] is not None:
        h = h + s["add"].double()
    if s["rows"] is not None:
        h = h[s["rows"].long()]
    return h / torch.sqrt(h.square().sum(dim=1, keepdim=True) / h.shape[1] + EPS) * s["gain"].double(), h


def _exact_linear(a, w, bias, gelu):
    v = a @ w.t() + bias.double()
    if gelu:
        v = v / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    return v


def exact(case, seed):
    # (8-bit results, like those in bf16, are given as they are before they are rounded for storage)
    s, op = prepare(case, seed), case["op"]
    if op == "rms":
        y, h = _exact_rms(s)
        q, scales = _exact_scaled(y, 1)
        return {"q": q, "scales": scales, "sum": h if case["sum"] else None}
    if op == "quantize":
        q, scales = _exact_scaled(s["x"].double(), case["block_rows"])
        return {"q": q, "scales": scales}
    if op == "linear":
        v = _exact_linear(_exact_values(s["a"], s["a_scales"], False), _exact_values(s["w"], s["w_scales"], True), s["bias"], case["gelu"])
        if case["quantized"]:
            q, scales = _exact_scaled(v, 1)
            return {"q": q, "scales": scales}
        return {"c": v}
    w1, w2 = _exact_values(s["w1"], s["w1_scales"], True), _exact_values(s["w2"], s["w2_scales"], True)
    mid = _exact_stored(_exact_linear(_exact_stored(_exact_rms(s)[0]), w1, s["bias1"], True))
    return {"c": _exact_linear(mid, w2, s["bias2"], False)}
