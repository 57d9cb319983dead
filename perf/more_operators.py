"""What is measured of the operators that lead to the logits and back: the product with a restored checkpoint's
weights themselves, the norm before it, and activations kept in 8 bits for the backward pass.

`run` computes one pass of one operator, either in its plain form (elementary torch operations in 32 bits) or, with
`own` set, through the package.

    norm         y = (x - mean) rstd weight + bias (rms: no mean, no bias) and the gradients of x, weight and bias
    linear       y = act(x w^T + bias) + residual; what goes into the activation may be kept in 8 bits
    linear_grad  the gradients of x (+ add), w and bias from that of x w^T + bias
    act8         values in 8 bits and back
    act_grad     the gradient through an activation from what was kept, the activation's value again, the bias's gradient

Values in 8 bits: blocks of 32 consecutive columns share a scale s = A / 127, rounded up to 8 significant bits and at least
2^-126, with A the block's largest magnitude; a code is fl(x fl(1 / s)) rounded to the nearest whole number (fl: rounding to 32 bits).
Packed, R rows and C columns with B = ceil(C / 32): R rows of 32 B codes (one signed byte each, 0 past the last column),
then R rows of B scales as bfloat16.
"""
import math

import torch

own = False

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
ACTS = ["none", "gelu", "gelu_tanh", "silu"]
EPS = 1e-5


def listed():
    return [
        # --- norm
        # one token of the 7B shape on its way into a layer
        {"name": "norm 1x4096", "op": "norm", "rows": 1, "cols": 4096, "slack": 0, "dtype": "bf16", "rms": True, "keep": False, "grad": False},
        # rows of a wider buffer, nothing a multiple of a vector, in the type that the decoder leaves; both directions
        {"name": "norm 333x1000 slice gradient", "op": "norm", "rows": 333, "cols": 1000, "slack": 37, "dtype": "fp32", "rms": False, "keep": False, "grad": True},
        # a batch of fine-tuning through a norm of the 7B shape; its input is kept in 8 bits for the backward pass
        {"name": "norm 8192x4096 kept gradient", "op": "norm", "rows": 8192, "cols": 4096, "slack": 0, "dtype": "bf16", "rms": False, "keep": True, "grad": True},
        # --- linear
        # one new token through an MLP matrix of the 7B shape
        {"name": "linear 1 token", "op": "linear", "rows": 1, "k": 4096, "n": 11008, "slack": 0, "dtype": "bf16", "act": "silu", "bias": False, "residual": False, "keep": False},
        # a few sequences at once through the output embedding of the 1.4B shape
        {"name": "linear 16 tokens head", "op": "linear", "rows": 16, "k": 2048, "n": 50304, "slack": 0, "dtype": "fp16", "act": "none", "bias": False, "residual": False, "keep": False},
        # nothing a multiple of a tile: a ragged batch, a slice as input, everything in the epilogue
        {"name": "linear ragged", "op": "linear", "rows": 333, "k": 1000, "n": 4097, "slack": 24, "dtype": "bf16", "act": "gelu", "bias": True, "residual": True, "keep": False},
        # a batch of fine-tuning through the first MLP matrix of the 7B shape, what goes into the activation kept in 8 bits
        {"name": "linear 4096 tokens kept", "op": "linear", "rows": 4096, "k": 4096, "n": 11008, "slack": 0, "dtype": "bf16", "act": "gelu", "bias": True, "residual": False, "keep": True},
        # --- linear_grad
        # a short batch through the first MLP matrix of the 410M shape
        {"name": "linear gradient 200 tokens", "op": "linear_grad", "rows": 200, "k": 1024, "n": 4096, "slack": 0, "dtype": "fp16", "bias": True, "add": True},
        # a batch of fine-tuning through an MLP matrix of the 7B shape
        {"name": "linear gradient 4096 tokens", "op": "linear_grad", "rows": 4096, "k": 4096, "n": 11008, "slack": 0, "dtype": "bf16", "bias": True, "add": False},
        # --- activations in 8 bits
        # the input of a 7B shape's second MLP matrix, kept and brought back
        {"name": "act8 4096x11008", "op": "act8", "rows": 4096, "cols": 11008, "slack": 0, "dtype": "bf16"},
        # a ragged slice of a fused projection, kept as it is
        {"name": "activation gradient 333x1000", "op": "act_grad", "rows": 333, "cols": 1000, "slack": 37, "dtype": "fp32", "act": "silu", "kept": "plain", "again": False},
        # the backward pass of an MLP of the 7B shape, from 8 bits, with the activation's value for the next weight gradient
        {"name": "activation gradient 4096x11008", "op": "act_grad", "rows": 4096, "cols": 11008, "slack": 0, "dtype": "bf16", "act": "gelu", "kept": "act8", "again": True},
    ]


def _size(rng, low, high):
    """Spread over the logarithm; every other one rounded to a multiple of 64 where it is large enough."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return max(64, v // 64 * 64) if v >= 64 and rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["norm", "linear", "linear", "linear_grad", "act8", "act_grad"])
    slack = rng.choice([0, 0, rng.randint(1, 64)])
    if op == "norm":
        while True:
            rows, cols = _size(rng, 1, 16384), _size(rng, 64, 16384)
            if rows * cols <= 8192 * 4096:
                break
        grad = rng.random() < 0.6
        return {"op": op, "rows": rows, "cols": cols, "slack": slack, "dtype": rng.choice(sorted(DTYPE)), "rms": rng.random() < 0.5,
                "keep": grad and rng.random() < 0.5, "grad": grad}
    if op == "linear":
        while True:
            rows, k, n = _size(rng, 1, 8192), _size(rng, 64, 11008), _size(rng, 64, 50304)
            if rows * k * n <= 4096 * 4096 * 11008 and n * k <= 50304 * 2048 and rows * n <= 4096 * 11008:
                break
        return {"op": op, "rows": rows, "k": k, "n": n, "slack": slack, "dtype": rng.choice(["bf16", "fp16"]), "act": rng.choice(ACTS),
                "bias": rng.random() < 0.5, "residual": rng.random() < 0.4, "keep": rng.random() < 0.3}
    if op == "linear_grad":
        while True:
            rows, k, n = _size(rng, 1, 8192), _size(rng, 64, 11008), _size(rng, 64, 16384)
            if rows * k * n <= 4096 * 4096 * 11008 and n * k <= 11008 * 4096 and rows * max(n, k) <= 4096 * 11008:
                break
        return {"op": op, "rows": rows, "k": k, "n": n, "slack": slack, "dtype": rng.choice(["bf16", "fp16"]), "bias": rng.random() < 0.5, "add": rng.random() < 0.4}
    while True:
        rows, cols = _size(rng, 1, 16384), _size(rng, 64, 16384)
        if rows * cols <= 4096 * 11008:
            break
    if op == "act8":
        return {"op": op, "rows": rows, "cols": cols, "slack": slack, "dtype": rng.choice(sorted(DTYPE))}
    return {"op": op, "rows": rows, "cols": cols, "slack": slack, "dtype": rng.choice(sorted(DTYPE)), "act": rng.choice(ACTS[1:]),
            "kept": rng.choice(["act8", "plain"]), "again": rng.random() < 0.5}


# ---- inputs ----------------------------------------------------------------

def _activations(rows, cols, slack, dtype, gen, size=1.0):
    """Normals with a hundredth of the columns ten times as large, as hidden states have them: a view of a buffer
    whose rows are `slack` longer."""
    x = torch.randn(rows, cols + slack, generator=gen, device="cuda") * size
    big = torch.rand(cols + slack, generator=gen, device="cuda") < 0.01
    return (x * torch.where(big, 10.0, 1.0)).to(dtype)[:, :cols]


def _normals(gen, size, dtype, *shape):
    return (torch.randn(*shape, generator=gen, device="cuda") * size).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case)
    t, rows, slack = DTYPE[case["dtype"]], case["rows"], case["slack"]
    if case["op"] == "norm":
        cols = case["cols"]
        state["x"] = _activations(rows, cols, slack, t, gen)
        state["weight"] = (1.0 + torch.randn(cols, generator=gen, device="cuda") * 0.2).to(t)
        state["bias"] = None if case["rms"] else _normals(gen, 0.1, t, cols)
        if case["grad"]:
            state["dy"] = _normals(gen, 0.01, t, rows, cols)
    elif case["op"] == "linear":
        k, n = case["k"], case["n"]
        state["x"] = _activations(rows, k, slack, t, gen)
        state["w"] = _normals(gen, 0.02, t, n, k)
        state["bias"] = _normals(gen, 0.1, t, n) if case["bias"] else None
        state["residual"] = _activations(rows, n, slack, t, gen) if case["residual"] else None
    elif case["op"] == "linear_grad":
        k, n = case["k"], case["n"]
        state["dy"] = _normals(gen, 0.01, t, rows, n)
        state["x"] = _activations(rows, k, slack, t, gen)
        state["w"] = _normals(gen, 0.02, t, n, k)
        state["add"] = _normals(gen, 0.01, t, rows, k) if case["add"] else None
    else:
        x = _activations(rows, case["cols"], slack, t, gen, 1.5 if case["op"] == "act_grad" else 1.0)
        if case["op"] == "act8":
            state["x"] = x
        else:
            state["dy"] = _normals(gen, 0.01, t, rows, case["cols"])
            state["pre"] = _pack8(*_codes8(x)) if case["kept"] == "act8" else x     # what the forward pass kept
    return state


def work(case):
    rows, size = case["rows"], BYTES[case["dtype"]]
    if case["op"] in ("linear", "linear_grad"):
        k, n = case["k"], case["n"]
        if case["op"] == "linear":
            byte = 2 * (rows * k + n * k + rows * n) + 2 * n * case["bias"] + 2 * rows * n * case["residual"] + rows * n * 34 / 32 * case["keep"]
            return {"bytes": byte, "flops": 2 * rows * n * k}
        byte = 2 * (rows * n + rows * k + n * k) + 2 * rows * k * (2 if case["add"] else 1) + 4 * n * k + 4 * n * case["bias"]
        return {"bytes": byte, "flops": 4 * rows * n * k}
    e = rows * case["cols"]
    if case["op"] == "norm":
        # kept: written by the forward pass and read by the backward pass in place of x
        there = e * 2 * size + 8 * rows + case["cols"] * size * (1 if case["rms"] else 2)
        kept = e * 34 / 32
        back = e * 2 * size + (2 * kept if case["keep"] else e * size) + 8 * case["cols"]
        return {"bytes": there + (back if case["grad"] else 0), "flops": e * (20 if case["grad"] else 8)}
    if case["op"] == "act8":
        return {"bytes": e * (2 * size + 2 * 34 / 32), "flops": 6 * e}
    return {"bytes": e * (size * (3 if case["again"] else 2) + (34 / 32 if case["kept"] == "act8" else size)) + 4 * case["cols"], "flops": 30 * e}


# ---- plain forms -------------------------------------------------------------

def _blocks(x, b=32):
    x = torch.nn.functional.pad(x.to(torch.float32), (0, -x.shape[1] % b))
    return x.view(x.shape[0], -1, b)


def _codes8(x):
    """Codes [R, B, 32] (whole numbers in 32-bit floats) and scales [R, B] of x."""
    v = _blocks(x)
    largest = v.abs().amax(2)
    m, e = torch.frexp(largest / 127.0)
    s = torch.ldexp(torch.ceil(m * 256.0) / 256.0, e).clamp(min=2.0 ** -126)
    return torch.round(v * (1.0 / s)[:, :, None]), s


def _values8(codes, scales, cols):
    return (codes * scales[:, :, None]).flatten(1)[:, :cols]


def _pack8(codes, scales):
    return torch.cat([codes.to(torch.int8).flatten().view(torch.uint8), scales.to(torch.bfloat16).flatten().view(torch.uint8)])


def _unpack8(data, rows, cols):
    b = -(-cols // 32)
    codes = data[:rows * b * 32].view(torch.int8).view(rows, b, 32)
    scales = data[rows * b * 32:rows * b * 34].view(torch.bfloat16).view(rows, b)
    return codes.to(torch.float32), scales.to(torch.float32)


def _act(p, act):
    if act == "gelu":
        return 0.5 * p * (1.0 + torch.erf(p * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * p * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (p + 0.044715 * p ** 3)))
    return p / (1.0 + torch.exp(-p)) if act == "silu" else p


def _act_slope(p, act):
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(p * math.sqrt(0.5))) + p * torch.exp(-0.5 * p * p) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (p + 0.044715 * p ** 3))
        return 0.5 * (1.0 + t) + 0.5 * p * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * p * p)
    s = 1.0 / (1.0 + torch.exp(-p))
    return s * (1.0 + p * (1.0 - s))


def _plain_norm(s):
    x, w = s["x"].to(torch.float32), s["weight"].to(torch.float32)
    mean = torch.zeros_like(x[:, :1]) if s["rms"] else x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
    y = (x - mean) * rstd * w
    if s["bias"] is not None:
        y = y + s["bias"]
    out = {"y": y.to(s["x"].dtype)}
    if s["grad"]:
        if s["keep"]:
            x = _values8(*_codes8(x), s["cols"])
        dy = s["dy"].to(torch.float32)
        xh, g = (x - mean) * rstd, dy * w
        dx = g - xh * (g * xh).mean(1, keepdim=True)
        if not s["rms"]:
            dx = dx - g.mean(1, keepdim=True)
        out["dx"] = (dx * rstd).to(s["x"].dtype)
        out["dweight"] = (dy * xh).sum(0)
        if not s["rms"]:
            out["dbias"] = dy.sum(0)
    return out


def _plain_linear(s):
    p = s["x"].to(torch.float32) @ s["w"].to(torch.float32).T
    if s["bias"] is not None:
        p = p + s["bias"]
    y = _act(p, s["act"])
    if s["residual"] is not None:
        y = y + s["residual"]
    out = {"y": y.to(s["x"].dtype)}
    if s["keep"]:
        out["kept"] = _values8(*_codes8(p), s["n"]).to(s["x"].dtype)
    return out


def _plain_linear_grad(s):
    dy = s["dy"].to(torch.float32)
    dx = dy @ s["w"].to(torch.float32)
    if s["add"] is not None:
        dx = dx + s["add"]
    out = {"dx": dx.to(s["x"].dtype), "dw": dy.T @ s["x"].to(torch.float32)}
    if s["bias"]:
        out["dbias"] = dy.sum(0)
    return out


def _plain_act8(s):
    return _values8(*_codes8(s["x"]), s["cols"]).to(s["x"].dtype)


def _plain_act_grad(s):
    p = s["pre"].to(torch.float32) if s["kept"] == "plain" else _values8(*_unpack8(s["pre"], s["rows"], s["cols"]), s["cols"])
    d = s["dy"].to(torch.float32) * _act_slope(p, s["act"])
    out = {"dpre": d.to(s["dy"].dtype), "dbias": d.sum(0)}
    if s["again"]:
        out["a"] = _act(p, s["act"]).to(s["dy"].dtype)
    return out


# ---- the package's operators ---------------------------------------------------

_handles = {}


def _handle():
    """One handle of the library per device, as a program keeps it."""
    device = torch.cuda.current_device()
    if device not in _handles:
        from paper_2406_11257_b200 import binding
        _handles[device] = binding.Handle(workspace_numel=4096)
    return _handles[device]


def _own_norm(s):
    h = _handle()
    r = h.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, rms=s["rms"], keep=s["keep"])
    out = {"y": r.y}
    if s["grad"]:
        g = h.layer_norm_grad(s["dy"], r.kept if s["keep"] else s["x"], s["weight"], r)
        out["dx"], out["dweight"] = g.dx, g.dweight
        if not s["rms"]:
            out["dbias"] = g.dbias
    return out


def _own_linear(s):
    h = _handle()
    if not s["keep"]:
        return {"y": h.linear(s["x"], s["w"], s["bias"], act=s["act"], residual=s["residual"])}
    y, kept = h.linear_kept(s["x"], s["w"], s["bias"], act=s["act"], residual=s["residual"], keep="act8")
    return {"y": y, "kept": h.act8_restore(kept, s["x"].dtype)}


def _own_linear_grad(s):
    h = _handle()
    out = {"dx": h.linear_grad_input(s["dy"], s["w"], add=s["add"]), "dw": h.linear_grad_weight(s["dy"], s["x"])}
    if s["bias"]:
        out["dbias"] = h.bias_grad(s["dy"])
    return out


def _own_act8(s):
    h = _handle()
    return h.act8_restore(h.act8_quantize(s["x"]), s["x"].dtype)


def _own_act_grad(s):
    from paper_2406_11257_b200 import binding
    pre = s["pre"] if s["kept"] == "plain" else binding.Act8Matrix(s["pre"], s["rows"], s["cols"])
    g = _handle().act_grad(s["dy"], pre, s["act"], again=s["again"])
    return {"dpre": g.dpre, "dbias": g.dbias, "a": g.a} if s["again"] else {"dpre": g.dpre, "dbias": g.dbias}


def run(state):
    op = state["op"]
    if own:
        return {"norm": _own_norm, "linear": _own_linear, "linear_grad": _own_linear_grad, "act8": _own_act8, "act_grad": _own_act_grad}[op](state)
    return {"norm": _plain_norm, "linear": _plain_linear, "linear_grad": _plain_linear_grad, "act8": _plain_act8, "act_grad": _plain_act_grad}[op](state)


# ---- the definitions in 64 bits ---------------------------------------------------

def _kept64(x):
    """What 8 bits make of x: the largest magnitude of every 32 columns sets the step."""
    rows, cols = x.shape
    v = torch.zeros(rows, -(-cols // 32), 32, dtype=torch.float64, device=x.device)
    v.view(rows, -1)[:, :cols] = x
    a = (v.abs().max(2, keepdim=True).values / 127.0).float().double()
    # 8 significant bits: their unit is 2^(floor(log2 a) - 7)
    unit = torch.exp2(torch.frexp(a.clamp(min=2.0 ** -126)).exponent.double() - 8)
    step = (torch.ceil(a / unit) * unit).clamp(min=2.0 ** -126)
    inverse = (1.0 / step).float().double()
    q = torch.round((v * inverse).float()).double()
    return (q * step).view(rows, -1)[:, :cols]


def _act64(p, act):
    """The activation and its slope."""
    if act == "none":
        return p, torch.ones_like(p)
    if act == "gelu":
        cdf = torch.special.ndtr(p)
        return p * cdf, cdf + p * torch.exp(-p * p / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(p)
        return p * s, s + p * s * torch.sigmoid(-p)
    u = 2 * math.sqrt(2 / math.pi) * (p + 0.044715 * p * p * p)
    s = torch.sigmoid(u)
    return p * s, s + p * s * torch.sigmoid(-u) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * p * p)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x, w = s["x"].double(), s["weight"].double()
        mu = 0.0 if case["rms"] else x.sum(1, keepdim=True) / case["cols"]
        sigma = torch.sqrt(((x - mu) ** 2).sum(1, keepdim=True) / case["cols"] + EPS)
        y = (x - mu) / sigma * w
        out = {"y": y if s["bias"] is None else y + s["bias"].double()}
        if case["grad"]:
            xh = ((_kept64(s["x"].double()) if case["keep"] else x) - mu) / sigma
            dy = s["dy"].double()
            d = dy * w / sigma
            if not case["rms"]:
                out["dbias"] = torch.einsum("rc->c", dy)
                d = d - d.mean(1, keepdim=True)
            # the part along xh goes
            out["dx"] = d - xh * (torch.einsum("rc,rc->r", dy * w / sigma, xh) / case["cols"])[:, None]
            out["dweight"] = torch.einsum("rc,rc->c", dy, xh)
        return out
    if case["op"] == "linear":
        p = torch.einsum("rk,nk->rn", s["x"].double(), s["w"].double())
        if s["bias"] is not None:
            p += s["bias"].double()
        y = _act64(p, case["act"])[0]
        out = {"y": y if s["residual"] is None else y + s["residual"].double()}
        if case["keep"]:
            out["kept"] = _kept64(p)
        return out
    if case["op"] == "linear_grad":
        dy, x = s["dy"].double(), s["x"].double()
        dx = torch.einsum("rn,nk->rk", dy, s["w"].double())
        out = {"dx": dx if s["add"] is None else dx + s["add"].double(), "dw": torch.einsum("rn,rk->nk", dy, x)}
        if case["bias"]:
            out["dbias"] = torch.einsum("rn->n", dy)
        return out
    if case["op"] == "act8":
        return _kept64(s["x"].double())
    if case["kept"] == "act8":
        rows, b = case["rows"], -(-case["cols"] // 32)
        at = torch.arange(case["cols"], device="cuda")
        q = s["pre"][:rows * b * 32].view(torch.int8).view(rows, b * 32)[:, at].double()
        p = q * s["pre"][rows * b * 32:].view(torch.bfloat16).view(rows, b)[:, at // 32].double()
    else:
        p = s["pre"].double()
    a, slope = _act64(p, case["act"])
    d = s["dy"].double() * slope
    out = {"dpre": d, "dbias": torch.einsum("rn->n", d)}
    if case["again"]:
        out["a"] = a
    return out
