"""What stands around and beside a layer's 8-bit product in a training step, as programs call it.

* ``norm``: a layer norm's forward pass (``layer_norm``), from one token on;
* ``norm_train``: forward and backward of it (``layer_norm_backward``): the input's gradient with the residual path's
  added, the gradients of weight and bias in binary32 as ``encode`` takes them;
* ``dropout``: a sublayer's output through dropout onto the residual path, and its gradient (``dropout``; the mask comes
  from a counter-based generator, forward and backward draw it again);
* ``pack``: a matrix to 4-bit numbers with a scale for each block of 32, along its rows and along its columns
  (``quantize_mx4``), and back (``dequantize_mx4``);
* ``linear``: a layer's product in these numbers, activations quantised on the way (``linear_mx4``);
* ``product``: the product of two operands that are quantised already (``matmul_mx4``);
* ``train``: the layer's step of training: weights quantised both ways, forward and backward (``linear_mx4_backward``),
  the outputs' gradient rounded up or down by chance, so that its mean is kept.

The shapes are the matrices of the networks whose gradients the other workloads stand for (gates, embedding and output
layer of a 2 x 1500 LSTM, 20 sequences of 35 tokens), plain powers of two, and sizes that are a multiple of nothing.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
BLOCK = 32                      # numbers that share a scale


def listed():
    return [
        # One token's norm: what answering one request waits for.
        _norm("norm_1x1500", "norm", 1, 1500, "bf16", "bf16"),
        # A residual path kept in binary32, normed for bfloat16 products.
        _norm("norm_8192x4096", "norm", 8192, 4096, "f32", "bf16"),
        # The LSTM's width in training, 20 sequences of 35 tokens.
        _norm("norm_train_700x1500", "norm_train", 700, 1500, "bf16", "bf16"),
        # A wide layer in training, 16384 tokens on one device.
        _norm("norm_train_16384x4096", "norm_train", 16_384, 4096, "bf16", "bf16"),
        # Dropout between the LSTM's layers.
        _dropout("dropout_700x1500", 700, 1500, "bf16", 0.5),
        # Dropout of a wide layer, onto the residual path.
        _dropout("dropout_16384x4096", 16_384, 4096, "bf16", 0.1),
        # The embedding's weights, quantised for the forward and for the backward product.
        {"name": "pack_10000x1500", "kind": "pack", "m": 10_000, "k": 1500, "type": "f32", "drawn": False},
        # One token through the LSTM's output layer.
        _linear("linear_1x1500_10000", 1, 1500, 10_000, "bf16"),
        # A prompt through a wide layer: the matrix units decide.
        _linear("linear_2048x4096_16384", 2048, 4096, 16_384, "bf16"),
        # Two operands that are quantised already, no size a multiple of anything, binary32 out.
        {"name": "product_1499x5001x2003", "kind": "product", "m": 1499, "k": 5001, "n": 2003, "type": "f32"},
        # The LSTM's gates in training.
        _train("train_700x1500_6000", 700, 1500, 6000),
        # A wide layer in training, 8192 tokens on one device: the largest step.
        _train("train_8192x4096_4096", 8192, 4096, 4096),
    ]


def _norm(name, kind, m, k, x_type, y_type):
    return {"name": name, "kind": kind, "m": m, "k": k, "type": x_type, "out": y_type}


def _dropout(name, m, k, kind, p):
    return {"name": name, "kind": "dropout", "m": m, "k": k, "type": kind, "p": p}


def _linear(name, m, k, n, kind):
    return {"name": name, "kind": "linear", "m": m, "k": k, "n": n, "type": kind}


def _train(name, m, k, n):
    return {"name": name, "kind": "train", "m": m, "k": k, "n": n, "type": "bf16"}


def draw(rng):
    def spread(lo, hi):
        return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))

    kind = rng.choice(["norm", "norm_train", "norm_train", "dropout", "pack", "linear", "linear", "product", "train"])
    while True:
        if kind in ("norm", "norm_train", "dropout", "pack"):
            m, k = spread(1, 20_000), spread(16, 24_000)
            if not 1024 <= m * k <= 1 << 26:
                continue
            case = {"kind": kind, "m": m, "k": k, "type": rng.choice(["f32", "bf16", "f16"])}
            if kind == "dropout":
                return {**case, "p": rng.choice([0.1, 0.2, 0.5, 0.9])}
            if kind == "pack":
                return {**case, "drawn": rng.random() < 0.5}
            return {**case, "out": rng.choice([case["type"], "bf16"])}
        m = spread(1, 4096) if kind == "linear" else spread(64, 8192)
        k, n = spread(64, 16_384), spread(64, 16_384)
        if n * k > 1 << 26 or m * n * k > 1 << 37 or m * n * k < 1 << 18:
            continue
        types = {"linear": ["bf16", "f16", "f32"], "product": ["f32", "bf16"], "train": ["bf16"]}[kind]
        return {"kind": kind, "m": m, "k": k, "n": n, "type": rng.choice(types)}


def _activations(m, k, gen):
    """Tokens of differing sizes, a few channels much larger than the others."""
    x = torch.randn(m, k, device=DEV, generator=gen) * torch.exp(0.5 * torch.randn(m, 1, device=DEV, generator=gen))
    return x * (1.0 + 9.0 * (torch.rand(k, device=DEV, generator=gen) < 0.01))


def _packed(rows, k, gen):
    """A quantised operand as a program keeps it: two numbers a byte in rows that start at multiples of 16 bytes, the
    scales of a block of all rows side by side (2^(byte - 127))."""
    have, blocks = (k + 1) // 2, -(-k // BLOCK)
    store = torch.zeros(rows, -(-have // 16) * 16, dtype=torch.uint8, device=DEV)
    store[:, :have] = torch.randint(0, 256, (rows, have), device=DEV, generator=gen, dtype=torch.uint8)
    if k % 2:
        store[:, have - 1] &= 15
    scale = torch.empty(blocks, -(-rows // 16) * 16, dtype=torch.uint8, device=DEV)
    scale.copy_(torch.randint(117, 121, scale.shape, device=DEV, generator=gen, dtype=torch.uint8))
    return store[:, :have], scale[:, :rows]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    kind, m, k = case["kind"], case["m"], case["k"]
    state = {"case": case, "seed": 42, "step": seed & 0xFFFF_FFFF}       # what the generator's draws belong to
    if kind == "product":
        state["a"], state["a_scale"] = _packed(m, k, gen)
    else:
        state["x"] = _activations(m, k, gen).to(TYPES[case["type"]])
    if kind in ("norm", "norm_train"):
        state["gamma"] = 1.0 + 0.2 * torch.randn(k, device=DEV, generator=gen)
        state["beta"] = 0.1 * torch.randn(k, device=DEV, generator=gen)
        if kind == "norm_train":
            state["dy"] = (1e-3 * _activations(m, k, gen)).to(TYPES[case["out"]])
            state["add"] = (1e-3 * _activations(m, k, gen)).to(TYPES[case["type"]])
    if kind == "dropout":
        state["residual"] = torch.randn(m, k, device=DEV, generator=gen).to(TYPES[case["type"]])
        state["dy"] = (1e-3 * _activations(m, k, gen)).to(TYPES[case["type"]])
    if kind in ("linear", "product"):
        state["w"], state["w_scale"] = _packed(case["n"], k, gen)
    if kind == "train":
        state["w"] = torch.randn(case["n"], k, device=DEV, generator=gen) / math.sqrt(k)
        state["dy"] = (1e-3 * _activations(m, case["n"], gen)).to(torch.bfloat16)
    if kind in ("linear", "product", "train"):
        state["bias"] = 0.1 * torch.randn(case["n"], device=DEV, generator=gen)
    return state


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---- through the framework ----------------------------------------------------------------------------------------

def _room_for(rows, k):
    """Memory for a quantised matrix, as in _packed()."""
    have = (k + 1) // 2
    q = torch.empty(rows, -(-have // 16) * 16, dtype=torch.uint8, device=DEV)[:, :have]
    return q, torch.empty(-(-k // BLOCK), -(-rows // 16) * 16, dtype=torch.uint8, device=DEV)[:, :rows]


def _run_own(state):
    import paper_2005_10761_amd as rt
    case = state["case"]
    kind, m, k = case["kind"], case["m"], case["k"]
    if kind in ("norm", "norm_train"):
        x, gamma = state["x"], state["gamma"]
        y = torch.empty(m, k, dtype=TYPES[case["out"]], device=DEV)
        mean, rstd = torch.empty(m, device=DEV), torch.empty(m, device=DEV)
        rt.layer_norm(x, gamma, state["beta"], y, mean, rstd, eps=EPS)
        if kind == "norm":
            return {"y": y, "mean": mean, "rstd": rstd}
        dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
        rt.layer_norm_backward(state["dy"], x, mean, rstd, gamma, dx, dgamma, dbeta, add=state["add"])
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx, "dgamma": dgamma, "dbeta": dbeta}
    if kind == "dropout":
        y, dx = torch.empty_like(state["x"]), torch.empty_like(state["x"])
        rt.dropout(state["x"], y, case["p"], state["seed"], state["step"], residual=state["residual"])
        rt.dropout(state["dy"], dx, case["p"], state["seed"], state["step"])
        return {"y": y, "dx": dx}
    if kind == "pack":
        x, drawn = state["x"], {"seed": state["seed"], "step": state["step"]} if case["drawn"] else {}
        (q, s), (qt, st) = _room_for(m, k), _room_for(k, m)
        rt.quantize_mx4(x, q, s, along="rows", **drawn)
        rt.quantize_mx4(x, qt, st, along="columns", **drawn)
        rows, columns = torch.empty_like(x), torch.empty(k, m, dtype=x.dtype, device=DEV)
        rt.dequantize_mx4(q, s, rows)
        rt.dequantize_mx4(qt, st, columns)
        return {"rows": rows, "columns": columns}
    n, out_type = case["n"], TYPES[case["type"]]
    y = torch.empty(m, n, dtype=out_type, device=DEV)
    if kind == "linear":
        rt.linear_mx4(state["x"], state["w"], state["w_scale"], y, bias=state["bias"])
        return y
    if kind == "product":
        rt.matmul_mx4(state["a"], state["a_scale"], state["w"], state["w_scale"], y, bias=state["bias"])
        return y
    (w, w_scale), (w_turned, w_turned_scale) = _room_for(n, k), _room_for(k, n)
    rt.quantize_mx4(state["w"], w, w_scale, along="rows")
    rt.quantize_mx4(state["w"], w_turned, w_turned_scale, along="columns")
    rt.linear_mx4(state["x"], w, w_scale, y, bias=state["bias"])
    dx, dw, db = torch.empty_like(state["x"]), torch.empty_like(state["w"]), torch.empty(n, device=DEV)
    rt.linear_mx4_backward(state["dy"], state["x"], w_turned, w_turned_scale, dx, dw, db, seed=state["seed"], step=state["step"])
    return {"y": y, "dx": dx, "dw": dw, "db": db}


# ---- the plain forms, in 32 bits ----------------------------------------------------------------------------------

ROUNDS = 10
FORWARD, ALONG_ROWS, ALONG_COLUMNS = 1, 2, 3       # what draws are for: the upper byte of the counter's second word


def _draws(count, what, seed, step):
    """16-bit numbers of Philox4x32-10, eight of each counter (whole numbers of 64 bits; products wrap)."""
    low = 0xFFFF_FFFF
    group = torch.arange(-(-count // 8), device=DEV)
    c0, c1 = group & low, (group >> 32) | (what << 24)
    c2, c3 = torch.full_like(group, step & low), torch.full_like(group, step >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(ROUNDS):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:count]


def _normed(x, gamma, beta):
    mean = x.mean(1)
    centred = x - mean[:, None]
    rstd = torch.rsqrt(centred.square().mean(1) + EPS)
    return centred * rstd[:, None] * gamma + beta, mean, rstd


def _norm_gradients(dy, x, mean, rstd, gamma, add):
    normal = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    inner = g - g.mean(1, keepdim=True) - normal * (g * normal).mean(1, keepdim=True)
    return rstd[:, None] * inner + add, (dy * normal).sum(0), dy.sum(0)


def _dropped(x, p, state):
    below = round(p * 65536)
    kept = _draws(x.numel(), FORWARD, state["seed"], state["step"]).view_as(x) >= below
    return torch.where(kept, x * (65536 / (65536 - below)), 0.0)


def _in_blocks(x):
    """[rows, blocks, 32] of [rows, k], zeros behind a row's end."""
    rows, k = x.shape
    blocks = -(-k // BLOCK)
    return torch.nn.functional.pad(x, (0, blocks * BLOCK - k)).view(rows, blocks, BLOCK)


def _four_bits(x, draws=None):
    """The values that x's rows become in blocks of 32: the nearest ones, ties to even, or by chance one of the two around."""
    blocks = _in_blocks(x)
    largest = blocks.abs().amax(2, keepdim=True)
    mantissa, exponent = torch.frexp(largest)           # largest = mantissa 2^exponent, 1/2 <= mantissa < 1
    up = mantissa >= 0.875 if draws is None else mantissa > 0.75
    exponent = torch.where(largest > 0, exponent - 3 + up.int(), -127).clamp(min=-127)
    # (2^-exponent and 2^exponent in two factors each: one of them may be outside of the normal numbers)
    half = exponent // 2
    t = torch.ldexp(torch.ldexp(blocks, -half), half - exponent)
    size = t.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    if draws is None:
        number = torch.round(size / step) * step
    else:
        below = torch.floor(size / step)
        number = (below + (draws.view_as(t) + 0.5 < 65536 * (size / step - below)).float()) * step
    values = torch.ldexp(torch.ldexp(torch.copysign(number, t), half), exponent - half)
    return values.flatten(1)[:, :x.shape[1]]


def _drawn_four_bits(x, what, state):
    count = x.shape[0] * -(-x.shape[1] // BLOCK) * BLOCK
    return _four_bits(x, _draws(count, what, state["seed"], state["step"]))


def _values(q, scale, k):
    """The numbers behind a quantised operand."""
    nibbles = torch.stack([q & 15, q >> 4], 2).flatten(1)[:, :k].int()
    magnitude = nibbles & 7
    number = torch.where(magnitude < 2, 0.5 * magnitude, torch.ldexp(1.0 + 0.5 * (magnitude & 1), (magnitude >> 1) - 1))
    number = torch.where(nibbles > 7, -number, number)
    return number * torch.exp2(scale.T.float() - 127).repeat_interleave(BLOCK, 1)[:, :k]


def _run_plain(state):
    case = state["case"]
    kind, out_type = case["kind"], TYPES[case["type"]]
    if kind in ("norm", "norm_train"):
        x, gamma = state["x"].float(), state["gamma"]
        y, mean, rstd = _normed(x, gamma, state["beta"])
        y = y.to(TYPES[case["out"]])
        if kind == "norm":
            return {"y": y, "mean": mean, "rstd": rstd}
        dx, dgamma, dbeta = _norm_gradients(state["dy"].float(), x, mean, rstd, gamma, state["add"].float())
        return {"y": y, "mean": mean, "rstd": rstd, "dx": dx.to(out_type), "dgamma": dgamma, "dbeta": dbeta}
    if kind == "dropout":
        y = _dropped(state["x"].float(), case["p"], state) + state["residual"].float()
        return {"y": y.to(out_type), "dx": _dropped(state["dy"].float(), case["p"], state).to(out_type)}
    if kind == "pack":
        x = state["x"].float()
        if case["drawn"]:
            rows, columns = _drawn_four_bits(x, ALONG_ROWS, state), _drawn_four_bits(x.T, ALONG_COLUMNS, state)
        else:
            rows, columns = _four_bits(x), _four_bits(x.T)
        return {"rows": rows.to(out_type), "columns": columns.to(out_type)}
    if kind == "linear":
        w = _values(state["w"], state["w_scale"], case["k"])
        return (torch.matmul(_four_bits(state["x"].float()), w.T) + state["bias"]).to(out_type)
    if kind == "product":
        a, w = _values(state["a"], state["a_scale"], case["k"]), _values(state["w"], state["w_scale"], case["k"])
        return (torch.matmul(a, w.T) + state["bias"]).to(out_type)
    x, w, dy = state["x"].float(), state["w"], state["dy"].float()
    y = torch.matmul(_four_bits(x), _four_bits(w).T) + state["bias"]
    dx = torch.matmul(_drawn_four_bits(dy, ALONG_ROWS, state), _four_bits(w.T).T)
    dw = torch.matmul(_drawn_four_bits(dy.T, ALONG_COLUMNS, state), _four_bits(x.T).T)
    return {"y": y.to(out_type), "dx": dx.to(out_type), "dw": dw, "db": dy.sum(0)}


# ---- from the definitions, in 64 bits -----------------------------------------------------------------------------

def _exact_draws(rows, columns, what, seed, step):
    """[rows, columns] draws (columns a multiple of 8), the products of Philox's rounds by halves of 16 bits."""
    def product(c, by):
        high, low = c >> 16, c & 0xFFFF
        a, b = high * (by >> 16), low * (by & 0xFFFF)
        cross = high * (by & 0xFFFF)
        other = low * (by >> 16)
        middle = (b >> 16) + (cross & 0xFFFF) + (other & 0xFFFF)
        return a + (cross >> 16) + (other >> 16) + (middle >> 16), ((middle & 0xFFFF) << 16) | (b & 0xFFFF)

    count = rows * columns // 8 + (rows * columns % 8 > 0)
    group = torch.arange(count, device=DEV, dtype=torch.int64)
    word = [group % (1 << 32), group // (1 << 32) + what * (1 << 24), torch.zeros_like(group) + step % (1 << 32),
            torch.zeros_like(group) + step // (1 << 32)]
    key = [seed % (1 << 32), seed // (1 << 32)]
    for _ in range(10):
        high0, low0 = product(word[0], 0xD2511F53)
        high1, low1 = product(word[2], 0xCD9E8D57)
        word = [high1 ^ word[1] ^ key[0], low1, high0 ^ word[3] ^ key[1], low0]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    out = torch.empty(count, 8, dtype=torch.int64, device=DEV)
    for i in range(4):
        out[:, 2 * i], out[:, 2 * i + 1] = word[i] % 65536, word[i] // 65536
    return out.flatten()[:rows * columns].view(rows, columns)


LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_four_bits(x, draws=None):
    """By the table of numbers: which two are around, and which of them is taken."""
    x = x.double()
    rows, k = x.shape
    wide = torch.zeros(rows, -(-k // BLOCK) * BLOCK, dtype=torch.float64, device=DEV)
    wide[:, :k] = x
    largest = wide.view(rows, -1, BLOCK).abs().max(2).values
    # the least power of two by which the largest comes below 7 (nearest), to 6 or below (drawn)
    power = torch.floor(torch.log2(torch.where(largest > 0, largest, 1.0))) - 4
    for _ in range(3):
        over = largest >= 7 * torch.exp2(power) if draws is None else largest > 6 * torch.exp2(power)
        power = torch.where(over, power + 1, power)
    scale = torch.exp2(torch.where(largest > 0, power, -127.0).clamp(min=-127)).repeat_interleave(BLOCK, 1)
    t = wide.abs() / scale
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=DEV)
    at = (torch.bucketize(t, levels, right=True) - 1).clamp(0, 6)
    lower, upper = levels[at], levels[at + 1]
    fraction = (t - lower) / (upper - lower)
    if draws is None:
        take = (fraction > 0.5) | ((fraction == 0.5) & (at % 2 == 1))        # an odd place: its neighbour is the even one
    else:
        take = draws + 0.5 < 65536 * fraction
    return (torch.where(take, upper, lower) * scale * torch.where(wide < 0, -1.0, 1.0))[:, :k]


def _exact_drawn(x, what, state):
    return _exact_four_bits(x, _exact_draws(x.shape[0], -(-x.shape[1] // BLOCK) * BLOCK, what, state["seed"], state["step"]))


def _exact_values(q, scale, k):
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64, device=DEV)
    out = torch.empty(q.shape[0], 2 * q.shape[1], dtype=torch.float64, device=DEV)
    out[:, 0::2], out[:, 1::2] = table[q.long() % 16], table[q.long() // 16]
    column = torch.arange(k, device=DEV) // BLOCK
    return out[:, :k] * torch.exp2(scale.double() - 127).T[:, column]


def exact(case, seed):
    state = prepare(case, seed)
    kind, m, k = case["kind"], case["m"], case["k"]
    if kind in ("norm", "norm_train"):
        x, gamma = state["x"].double(), state["gamma"].double()
        mean = x.sum(1, keepdim=True) / k
        spread = torch.sqrt((x - mean).pow(2).sum(1, keepdim=True) / k + EPS)
        unit = (x - mean) / spread
        out = {"y": unit * gamma + state["beta"].double(), "mean": mean[:, 0], "rstd": 1 / spread[:, 0]}
        if kind == "norm":
            return out
        dy = state["dy"].double()
        sums = (dy * gamma).sum(1, keepdim=True), (dy * gamma * unit).sum(1, keepdim=True)
        return {**out, "dx": (dy * gamma - (sums[0] + unit * sums[1]) / k) / spread + state["add"].double(),
                "dgamma": (dy * unit).sum(0), "dbeta": dy.sum(0)}
    if kind == "dropout":
        chance = round(case["p"] * 65536) / 65536
        wide = -(-(m * k) // 8) * 8
        kept = _exact_draws(1, wide, 1, state["seed"], state["step"])[0, :m * k].view(m, k) >= chance * 65536
        return {"y": state["x"].double() * kept / (1 - chance) + state["residual"].double(),
                "dx": state["dy"].double() * kept / (1 - chance)}
    if kind == "pack":
        x = state["x"]
        if case["drawn"]:
            return {"rows": _exact_drawn(x, 2, state), "columns": _exact_drawn(x.T, 3, state)}
        return {"rows": _exact_four_bits(x), "columns": _exact_four_bits(x.T)}
    bias = state["bias"].double()
    if kind in ("linear", "product"):
        a = _exact_four_bits(state["x"]) if kind == "linear" else _exact_values(state["a"], state["a_scale"], k)
        return a @ _exact_values(state["w"], state["w_scale"], k).T + bias
    x, w, dy = state["x"], state["w"], state["dy"]
    return {"y": _exact_four_bits(x) @ _exact_four_bits(w).T + bias,
            "dx": _exact_drawn(dy, 2, state) @ _exact_four_bits(w.T).T,
            "dw": _exact_drawn(dy.T, 3, state) @ _exact_four_bits(x.T).T,
            "db": dy.double().sum(0)}


def work(case):
    kind, m, k, size = case["kind"], case["m"], case["k"], SIZE[case["type"]]
    if kind == "norm":
        return {"bytes": m * k * (size + SIZE[case["out"]]) + 8 * k + 8 * m, "flops": 8 * m * k}
    if kind == "norm_train":
        # x, add, dy read, y and dx written; weight and bias read, their gradients written
        return {"bytes": m * k * (3 * size + 2 * SIZE[case["out"]]) + 16 * k + 8 * m, "flops": 22 * m * k}
    if kind == "dropout":
        return {"bytes": 5 * m * k * size, "flops": 4 * m * k}
    if kind == "pack":
        return {"bytes": 3 * m * k * size, "flops": 4 * m * k}
    n = case["n"]
    four = lambda rows, length: rows * ((length + 1) // 2 + -(-length // BLOCK))   # noqa: E731
    if kind == "train":
        # x, dy, w, bias read; y, dx, dw, db written; three products
        return {"bytes": 2 * (m * k + m * n) * size + 8 * n * k + 8 * n, "flops": 6 * m * k * n}
    left = four(m, k) if kind == "product" else m * k * size
    return {"bytes": left + four(n, k) + 4 * n + m * n * size, "flops": 2 * m * k * n}
