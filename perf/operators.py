"""The operators around the sparse exchange of a matrix parameter, as a training or serving program calls them.

* ``linear``: a layer's product in 8-bit integers with a scale for each token and each channel (``linear_i8``), from
  one token to a long prompt;
* ``product``: the same product of two operands that are already 8-bit (``matmul_i8``);
* ``train``: the layer's step of training: the weights quantised both ways (``quantize_i8``), forward and backward
  (``linear_i8_backward``), the weights' gradient in binary32 as ``encode`` takes it;
* ``orthogonalize``: Newton-Schulz orthogonalisation of updates of equal shapes;
* ``update``: the master's step: n sparse messages, averaged, into the momentum, orthogonalised, into the weights
  (``aggregate_update_orthogonal``).

The shapes are the matrices of the networks whose gradients the other workloads stand for (convolutions of ResNets as
out x in*kh*kw, the gate and embedding matrices of a 2 x 1500 LSTM), and plain powers of two.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
QUINTIC = (3.4445, -4.7750, 2.0315)     # the coefficients in common use for this iteration
STEPS, EPS = 5, 1e-7
ETA, MU, DECAY = 0.02, 0.95, 0.1


def listed():
    return [
        # One token through the LSTM's output layer: what answering one request waits for.
        _linear("linear_1x1500_10000", 1, 1500, 10_000, "bf16"),
        # A few requests decoded together, through a wide layer: the weights' bytes decide.
        _linear("linear_13x4096_16384", 13, 4096, 16_384, "bf16"),
        # A prompt through the same layer: the matrix units decide.
        _linear("linear_2048x4096_16384", 2048, 4096, 16_384, "bf16"),
        # Two operands that are 8-bit already, no size a multiple of anything, sums of 5001 terms, binary32 out.
        {"name": "product_1499x5001x2003", "kind": "product", "m": 1499, "k": 5001, "n": 2003, "type": "f32"},
        # The LSTM's gates in training: 20 sequences of 35 tokens.
        _train("train_700x1500_6000", 700, 1500, 6000),
        # A wide layer in training, 8192 tokens on one device: the largest step.
        _train("train_8192x4096_4096", 8192, 4096, 4096),
        # The four convolutions of a ResNet's first stage, 64 x 64*3*3: the smallest matrices, where launches count.
        _orthogonalize("ortho_64x576_x4", 4, 64, 576, "f32"),
        # The third stage's convolutions, gradients kept in bfloat16.
        _orthogonalize("ortho_256x2304_x3", 3, 256, 2304, "bf16"),
        # The gate matrices of both LSTM layers, tall.
        _orthogonalize("ortho_6000x1500_x4", 4, 6000, 1500, "f32"),
        # One large square matrix.
        _orthogonalize("ortho_4096x4096", 1, 4096, 4096, "bf16"),
        # The master's step for the fourth stage's convolutions, five workers at 99.9% compression.
        _update("update_512x4608_x3", 3, 512, 4608, 5),
        # The master's step for the LSTM's gates.
        _update("update_6000x1500_x4", 4, 6000, 1500, 5),
    ]


def _linear(name, m, k, n, kind):
    return {"name": name, "kind": "linear", "m": m, "k": k, "n": n, "type": kind}


def _train(name, m, k, n):
    return {"name": name, "kind": "train", "m": m, "k": k, "n": n, "type": "bf16"}


def _orthogonalize(name, count, rows, cols, kind):
    return {"name": name, "kind": "orthogonalize", "count": count, "rows": rows, "cols": cols, "type": kind}


def _update(name, count, rows, cols, workers):
    return {"name": name, "kind": "update", "count": count, "rows": rows, "cols": cols, "workers": workers, "type": "f32",
            "nesterov": True}


def draw(rng):
    def spread(lo, hi):
        return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))

    kind = rng.choice(["linear", "linear", "product", "train", "orthogonalize", "orthogonalize", "update"])
    while True:
        if kind in ("linear", "product", "train"):
            m = spread(1, 4096) if kind == "linear" else spread(64, 8192)
            k, n = spread(64, 16_384), spread(64, 16_384)
            if n * k > 1 << 26 or m * n * k > 1 << 37 or m * n * k < 1 << 18:
                continue
            types = {"linear": ["bf16", "f16", "f32"], "product": ["f32", "bf16"], "train": ["bf16"]}[kind]
            return {"kind": kind, "m": m, "k": k, "n": n, "type": rng.choice(types)}
        rows, cols, count = spread(16, 10_000), spread(16, 10_000), rng.choice([1, 1, 2, 3, 4, 6])
        case = {"kind": kind, "count": count, "rows": rows, "cols": cols}
        if work({**case, "type": "f32", "workers": 8})["flops"] > 1e12 or count * rows * cols < 4096:
            continue
        if kind == "orthogonalize":
            return {**case, "type": rng.choice(["f32", "bf16", "f16"])}
        return {**case, "type": "f32", "workers": rng.randrange(1, 9), "nesterov": rng.random() < 0.5}


def _message(case):
    """Entries that one worker sends for one matrix: a thousandth of it."""
    return max(1, case["rows"] * case["cols"] // 1000)


def _padded(values):
    """8-bit rows as a program lays them out once: each starts at a multiple of 16 bytes."""
    rows, cols = values.shape
    store = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.int8, device=DEV)
    store[:, :cols] = values
    return store[:, :cols]


def _gradient(case, gen):
    """What gradients of matrices look like: a few strong directions over noise."""
    count, rows, cols = case["count"], case["rows"], case["cols"]
    rank = min(16, rows, cols)
    left = torch.randn(count, rows, rank, device=DEV, generator=gen)
    right = torch.randn(count, rank, cols, device=DEV, generator=gen)
    strength = 2.0 ** -torch.arange(rank, device=DEV, dtype=torch.float32)
    return 1e-3 * (torch.matmul(left * strength, right) + torch.randn(count, rows, cols, device=DEV, generator=gen))


def _activations(m, k, gen):
    """Tokens of differing sizes, a few channels much larger than the others."""
    x = torch.randn(m, k, device=DEV, generator=gen) * torch.exp(0.5 * torch.randn(m, 1, device=DEV, generator=gen))
    return x * (1.0 + 9.0 * (torch.rand(k, device=DEV, generator=gen) < 0.01))


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    state = {"case": case}
    if case["kind"] in ("orthogonalize", "update"):
        gradient = _gradient(case, gen)
        if case["kind"] == "orthogonalize":
            state["x"] = list(gradient.to(TYPES[case["type"]]).unbind(0))
            return state
        count, n, k = case["count"], case["workers"], _message(case)
        d = case["rows"] * case["cols"]
        # distinct ascending indices, one of each of k equal stretches
        step = d // k
        at = torch.randint(0, step, (count, n, k), device=DEV, generator=gen) + step * torch.arange(k, device=DEV)
        state["idx"] = list(at.to(torch.int32).reshape(count, n * k).unbind(0))
        state["val"] = list((1e-2 * torch.randn(count, n * k, device=DEV, generator=gen)).unbind(0))
        state["velocity"] = list(gradient.unbind(0))
        weights = torch.randn(count, case["rows"], case["cols"], device=DEV, generator=gen) / math.sqrt(case["cols"])
        state["omega"] = list(weights.unbind(0))
        return state
    m, k, n = case["m"], case["k"], case["n"]
    if case["kind"] == "product":
        state["a"] = _padded(torch.randint(-127, 128, (m, k), device=DEV, generator=gen, dtype=torch.int8))
        state["a_scale"] = 0.02 * torch.exp(0.5 * torch.randn(m, device=DEV, generator=gen))
    else:
        state["x"] = _activations(m, k, gen).to(TYPES[case["type"]])
    if case["kind"] == "train":
        state["w"] = torch.randn(n, k, device=DEV, generator=gen) / math.sqrt(k)
        state["dy"] = (1e-3 * _activations(m, n, gen)).to(torch.bfloat16)
    else:
        state["w"] = _padded((32.0 * torch.randn(n, k, device=DEV, generator=gen)).clamp_(-127, 127).to(torch.int8))
        state["w_scale"] = (1.0 + torch.rand(n, device=DEV, generator=gen)) / (32.0 * math.sqrt(k))
    state["bias"] = 0.1 * torch.randn(n, device=DEV, generator=gen)
    return state


def run(state):
    return (_run_own if own else _run_plain)(state)


# ---- through the framework ----------------------------------------------------------------------------------------

def _rows_of_bytes(rows, cols):
    return torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device=DEV)[:, :cols]


def _run_own(state):
    import paper_2005_10761_amd as rt
    case = state["case"]
    kind, out_type = case["kind"], TYPES[case["type"]]
    if kind == "linear":
        out = torch.empty(case["m"], case["n"], dtype=out_type, device=DEV)
        rt.linear_i8(state["x"], state["w"], state["w_scale"], out, bias=state["bias"])
        return out
    if kind == "product":
        out = torch.empty(case["m"], case["n"], dtype=out_type, device=DEV)
        rt.matmul_i8(state["a"], state["a_scale"], state["w"], state["w_scale"], out, bias=state["bias"])
        return out
    if kind == "train":
        m, k, n = case["m"], case["k"], case["n"]
        w_rows, w_rows_scale = _rows_of_bytes(n, k), torch.empty(n, device=DEV)
        w_cols, w_cols_scale = _rows_of_bytes(k, n), torch.empty(k, device=DEV)
        rt.quantize_i8(state["w"], w_rows, w_rows_scale, along="rows")
        rt.quantize_i8(state["w"], w_cols, w_cols_scale, along="columns")
        y = torch.empty(m, n, dtype=out_type, device=DEV)
        rt.linear_i8(state["x"], w_rows, w_rows_scale, y, bias=state["bias"])
        dx, dw = torch.empty_like(state["x"]), torch.empty_like(state["w"])
        db = torch.empty(n, device=DEV)
        rt.linear_i8_backward(state["dy"], state["x"], w_cols, w_cols_scale, dx, dw, db)
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if kind == "orthogonalize":
        outs = [torch.empty_like(x) for x in state["x"]]
        rt.orthogonalize(state["x"], outs, steps=STEPS, coefficients=QUINTIC, eps=EPS)
        return outs
    rt.aggregate_update_orthogonal(state["idx"], state["val"], case["workers"], _message(case), ETA, 1.0, MU, state["omega"],
                                   state["velocity"], nesterov=case["nesterov"], decay=DECAY, steps=STEPS,
                                   coefficients=QUINTIC, eps=EPS)
    return {"omega": state["omega"], "velocity": state["velocity"]}


# ---- the plain forms, in 32 bits ----------------------------------------------------------------------------------

def _quantized(x, dim):
    """Whole numbers of -127 .. 127 (as binary32) and the scale of each row (dim 1) or column (dim 0)."""
    scale = x.abs().amax(dim, keepdim=True) / torch.full((), 127.0, device=DEV)     # (by a number it would be a product)
    return torch.where(scale > 0, torch.round(x / scale), 0.0), scale


def _steps(x):
    for _ in range(STEPS):
        a = torch.matmul(x, x.mT)
        x = QUINTIC[0] * x + torch.matmul(QUINTIC[1] * a + QUINTIC[2] * torch.matmul(a, a), x)
    return x


def _orthogonal(g):
    """Of a stack of matrices."""
    x = g.mT.contiguous() if g.shape[1] > g.shape[2] else g
    x = _steps(x / (torch.sqrt(x.square().sum((1, 2), keepdim=True)) + EPS))
    return x.mT if g.shape[1] > g.shape[2] else x


def _run_plain(state):
    case = state["case"]
    kind, out_type = case["kind"], TYPES[case["type"]]
    if kind == "linear":
        q, s = _quantized(state["x"].float(), 1)
        return (torch.matmul(q, state["w"].float().T) * s * state["w_scale"] + state["bias"]).to(out_type)
    if kind == "product":
        acc = torch.matmul(state["a"].float(), state["w"].float().T)
        return (acc * state["a_scale"][:, None] * state["w_scale"] + state["bias"]).to(out_type)
    if kind == "train":
        x, w, dy = state["x"].float(), state["w"], state["dy"].float()
        xr, xrs = _quantized(x, 1)
        wr, wrs = _quantized(w, 1)
        y = torch.matmul(xr, wr.T) * xrs * wrs[:, 0] + state["bias"]
        dyr, dyrs = _quantized(dy, 1)
        wc, wcs = _quantized(w, 0)
        dx = torch.matmul(dyr, wc) * dyrs * wcs
        dyc, dycs = _quantized(dy, 0)
        xc, xcs = _quantized(x, 0)
        dw = torch.matmul(dyc.T, xc) * dycs.T * xcs
        return {"y": y.to(out_type), "dx": dx.to(out_type), "dw": dw, "db": dy.sum(0)}
    if kind == "orthogonalize":
        return list(_orthogonal(torch.stack(state["x"]).float()).to(out_type).unbind(0))
    rows, cols = case["rows"], case["cols"]
    velocity, omega = torch.stack(state["velocity"]), torch.stack(state["omega"])
    sent = torch.zeros(case["count"], rows * cols, device=DEV)
    sent.scatter_add_(1, torch.stack(state["idx"]).long(), torch.stack(state["val"]))
    average = (sent / case["workers"]).view_as(velocity)
    velocity = MU * velocity + average
    moved = _orthogonal(MU * velocity + average if case["nesterov"] else velocity)
    omega = (1 - ETA * DECAY) * omega - ETA * moved
    torch._foreach_copy_(state["velocity"], list(velocity.unbind(0)))
    torch._foreach_copy_(state["omega"], list(omega.unbind(0)))
    return {"omega": state["omega"], "velocity": state["velocity"]}


# ---- from the definitions, in 64 bits -----------------------------------------------------------------------------

def _exact_numbers(x, by_row):
    """The 8-bit numbers that binary32 quotients by a binary32 scale round to, and the scales."""
    x = x.double() if by_row else x.double().T
    largest = x.abs().max(1).values
    scale = (largest / 127).float().double()
    quotient = (x / torch.where(scale > 0, scale, 1.0)[:, None]).float().double()
    return torch.where((scale > 0)[:, None], quotient.round(), 0.0), scale


def _exact_polar(g):
    """One matrix through the iteration, the fifth power term by term."""
    g = g.double()
    if g.shape[0] > g.shape[1]:
        return _exact_polar(g.T).T
    x = g / (g.norm() + EPS)
    for _ in range(STEPS):
        a = x @ x.T
        x = QUINTIC[0] * x + QUINTIC[1] * (a @ x) + QUINTIC[2] * (a @ (a @ x))
    return x


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "orthogonalize":
        return [_exact_polar(x) for x in state["x"]]
    if kind == "update":
        omegas, velocities = [], []
        for idx, val, velocity, omega in zip(state["idx"], state["val"], state["velocity"], state["omega"]):
            sent = torch.zeros(velocity.numel(), dtype=torch.float64, device=DEV)
            sent.index_add_(0, idx.long(), val.double())
            average = sent.view_as(velocity) / case["workers"]
            v = MU * velocity.double() + average
            step = _exact_polar(MU * v + average if case["nesterov"] else v)
            velocities.append(v)
            omegas.append(omega.double() * (1 - ETA * DECAY) - ETA * step)
        return {"omega": omegas, "velocity": velocities}
    w = state["w"].double()
    if kind == "product":
        return (state["a"].double() @ w.T) * torch.outer(state["a_scale"].double(), state["w_scale"].double()) + state["bias"].double()
    xr, xrs = _exact_numbers(state["x"], True)
    if kind == "linear":
        return (xr @ w.T) * torch.outer(xrs, state["w_scale"].double()) + state["bias"].double()
    wr, wrs = _exact_numbers(state["w"], True)
    wc, wcs = _exact_numbers(state["w"], False)
    xc, xcs = _exact_numbers(state["x"], False)
    dyr, dyrs = _exact_numbers(state["dy"], True)
    dyc, dycs = _exact_numbers(state["dy"], False)
    return {"y": (xr @ wr.T) * torch.outer(xrs, wrs) + state["bias"].double(),
            "dx": (dyr @ wc.T) * torch.outer(dyrs, wcs),
            "dw": (dyc @ xc.T) * torch.outer(dycs, xcs),
            "db": state["dy"].double().sum(0)}


def work(case):
    size = SIZE[case["type"]]
    if case["kind"] in ("orthogonalize", "update"):
        m, n, count = min(case["rows"], case["cols"]), max(case["rows"], case["cols"]), case["count"]
        # X X^T and its square are symmetric: half of each
        flops = count * STEPS * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)
        moved = 2 * m * n * size if case["kind"] == "orthogonalize" else 16 * m * n + 8 * case["workers"] * _message(case)
        return {"bytes": count * moved, "flops": flops}
    m, k, n = case["m"], case["k"], case["n"]
    if case["kind"] == "train":
        # x, dy, w, bias read; y, dx, dw, db written; three products
        return {"bytes": 2 * (m * k + m * n) * size + 8 * n * k + 8 * n, "flops": 6 * m * k * n}
    left = m * k * (1 if case["kind"] == "product" else size) + (4 * m if case["kind"] == "product" else 0)
    return {"bytes": left + n * k + 8 * n + m * n * size, "flops": 2 * m * k * n}
