"""What is measured of the operators that score a restored checkpoint.

A restored weight matrix is held in microscaled 4-bit floating point (`quantise`), multiplied with
activations that are quantised on the way in (`linear`), and the logits are turned into log
probabilities of the checkpoint's tokens (`logprobs`).  `run` computes one pass of one operator, either
in its plain form (elementary torch operations in 32 bits) or, with `own` set, through the package.

Two microscaled formats:
    e8m0_32   blocks of 32 values share a power of two
    e4m3_16   blocks of 16 values share an 8-bit float (4 exponent, 3 mantissa bits), and the matrix a
              32-bit tensor scale: its largest magnitude over 6 * 448, rounded up to 8 significant bits
A packed matrix is one buffer of bytes.  With R rows, C columns and KT = ceil(C / 256): rows come in tiles
of 128 (the last tile has its rows rounded up to 8, h in all), columns in tiles of 256, and a tile is
    h * 128 bytes   codes, two per byte, the lower column in the low bits; row r's 128 bytes are eight
                    16-byte chunks, chunk c at place c ^ (r % 8)
    scales          one 512-byte piece per 4 blocks of columns: row 32 c + l, block k at byte 16 l + 4 c + k
                    (always 128 rows, 0 where there is no row)
Tiles lie one after another, the column tiles of a row tile first.
"""
import math

import numpy as np
import torch

own = False

BLOCK = {"e8m0_32": 32, "e4m3_16": 16}
DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
ROW_TILE, COL_TILE = 128, 256


def listed():
    return [
        # --- quantise: a matrix to 4 bits and back to the values that the codes stand for
        # the activations of one token of the 7B shape on their way into a layer
        {"name": "quantise 1x4096", "op": "quantise", "rows": 1, "cols": 4096, "slack": 0, "fmt": "e4m3_16", "dtype": "bf16", "measure": False},
        # a slice of a fused projection: odd row count, rows of a wider buffer
        {"name": "quantise 777x1000 slice", "op": "quantise", "rows": 777, "cols": 1000, "slack": 37, "fmt": "e8m0_32", "dtype": "fp16", "measure": False},
        # an MLP matrix of the 7B shape stored in 16 bits, tensor scale measured first
        {"name": "quantise 11008x4096", "op": "quantise", "rows": 11008, "cols": 4096, "slack": 0, "fmt": "e4m3_16", "dtype": "bf16", "measure": True},
        # the restored output embedding of the 7B shape, fp32 as the decoder leaves it
        {"name": "quantise 32000x4096 fp32", "op": "quantise", "rows": 32000, "cols": 4096, "slack": 0, "fmt": "e8m0_32", "dtype": "fp32", "measure": False},
        # --- linear: activations times a matrix that is held in 4 bits
        # one new token through an MLP matrix of the 7B shape
        {"name": "linear 1 token", "op": "linear", "rows": 1, "k": 4096, "n": 11008, "slack": 0, "fmt": "e4m3_16", "dtype": "bf16", "bias": False},
        # a few sequences at once through the output embedding of the 1.4B shape
        {"name": "linear 16 tokens head", "op": "linear", "rows": 16, "k": 2048, "n": 50304, "slack": 0, "fmt": "e8m0_32", "dtype": "fp16", "bias": False},
        # nothing a multiple of a tile: a ragged batch, a slice as input, a bias
        {"name": "linear ragged", "op": "linear", "rows": 333, "k": 1000, "n": 4097, "slack": 24, "fmt": "e8m0_32", "dtype": "bf16", "bias": True},
        # the scoring pass: a batch of text through the output embedding of the 7B shape
        {"name": "linear 4096 tokens head", "op": "linear", "rows": 4096, "k": 4096, "n": 32000, "slack": 0, "fmt": "e4m3_16", "dtype": "bf16", "bias": False},
        # --- logprobs: log probabilities of given tokens, entropy, the likeliest alternatives
        # one sampled token of the 410M / 1.4B shape, with twenty alternatives
        {"name": "logprobs 1 row top 20", "op": "logprobs", "rows": 1, "vocab": 50304, "slack": 0, "dtype": "fp32", "top": 20, "grad": False, "masked": False},
        # scoring a batch of text with the 7B shape's vocabulary
        {"name": "logprobs 4096 rows top 5", "op": "logprobs", "rows": 4096, "vocab": 32000, "slack": 0, "dtype": "bf16", "top": 5, "grad": False, "masked": False},
        # fine-tuning on a restored checkpoint: log probabilities, entropy and the gradient of both
        {"name": "logprobs 2048 rows gradient", "op": "logprobs", "rows": 2048, "vocab": 50304, "slack": 0, "dtype": "bf16", "top": 0, "grad": True, "masked": False},
        # odd sizes, rows of a padded buffer, forbidden words at minus infinity, ignored positions
        {"name": "logprobs ragged masked", "op": "logprobs", "rows": 333, "vocab": 4097, "slack": 15, "dtype": "fp32", "top": 3, "grad": True, "masked": True},
    ]


def _size(rng, low, high):
    """Spread over the logarithm; every other one rounded to a multiple of 64 where it is large enough."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    return max(64, v // 64 * 64) if v >= 64 and rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["quantise", "linear", "logprobs"])
    slack = rng.choice([0, 0, rng.randint(1, 64)])
    if op == "quantise":
        fmt, dtype = rng.choice(sorted(BLOCK)), rng.choice(sorted(DTYPE))
        while True:
            rows, cols = _size(rng, 1, 32000), _size(rng, 64, 11008)
            if rows * cols <= 32000 * 4096:
                break
        return {"op": op, "rows": rows, "cols": cols, "slack": slack, "fmt": fmt, "dtype": dtype, "measure": fmt == "e4m3_16" and rng.random() < 0.5}
    if op == "linear":
        while True:
            rows, k, n = _size(rng, 1, 8192), _size(rng, 64, 11008), _size(rng, 64, 50304)
            if rows * k * n <= 4096 * 4096 * 32000 and n * k <= 32000 * 4096 and rows * n <= 4096 * 32000:
                break
        return {"op": op, "rows": rows, "k": k, "n": n, "slack": slack, "fmt": rng.choice(sorted(BLOCK)), "dtype": rng.choice(["bf16", "fp16"]), "bias": rng.random() < 0.5}
    while True:
        rows, vocab = _size(rng, 1, 8192), _size(rng, 64, 131072)
        if rows * vocab <= 2048 * 50304:
            break
    return {"op": op, "rows": rows, "vocab": vocab, "slack": slack, "dtype": rng.choice(sorted(DTYPE)), "top": rng.choice([0, 1, 5, 20]), "grad": rng.random() < 0.5, "masked": rng.random() < 0.3}


# ---- inputs ----------------------------------------------------------------

def _tensor_scale(largest):
    """largest / (6 * 448), rounded up to 8 significant bits; 1 for a matrix of zeros."""
    m, e = torch.frexp(largest / 2688.0)
    return torch.where(largest > 0, torch.ldexp(torch.ceil(m * 256.0) / 256.0, e), torch.ones_like(largest))


def _activations(rows, cols, slack, dtype, gen):
    """Unit normals with a hundredth of the columns ten times as large, as hidden states have them: a view of a buffer
    whose rows are `slack` longer."""
    x = torch.randn(rows, cols + slack, generator=gen, device="cuda")
    big = torch.rand(cols + slack, generator=gen, device="cuda") < 0.01
    return (x * torch.where(big, 10.0, 1.0)).to(dtype)[:, :cols]


def _pack_tiles(codes, scales):
    """codes [T, h, KT, 256], scale bytes [T, 128, KT, J, 4] -> packed bytes, T row tiles of height h."""
    t, h, kt, _ = codes.shape
    j = scales.shape[3]
    b = (codes[..., 0::2] | (codes[..., 1::2] << 4)).view(t, h, kt, 8, 16)
    r = torch.arange(h, device=codes.device)
    p = torch.arange(8, device=codes.device)
    b = b[:, r[:, None, None], torch.arange(kt, device=codes.device)[None, :, None], (p[None, :] ^ (r % 8)[:, None])[:, None, :]]
    b = b.permute(0, 2, 1, 3, 4).reshape(t, kt, h * 128)
    s = scales.view(t, 4, 32, kt, j, 4).permute(0, 3, 4, 2, 1, 5).reshape(t, kt, j * 512)
    return torch.cat([b, s], 2).reshape(-1)


def _pack(codes, scales, fmt):
    rows, cols = codes.shape
    kt, per = -(-cols // COL_TILE), COL_TILE // BLOCK[fmt]
    full = rows // ROW_TILE
    rest = rows - full * ROW_TILE
    h = -(-rest // 8) * 8
    c = torch.nn.functional.pad(codes, (0, kt * COL_TILE - cols, 0, h - rest)).view(-1, kt, COL_TILE)
    s = torch.nn.functional.pad(scales, (0, kt * per - scales.shape[1], 0, (ROW_TILE - rest) % ROW_TILE)).view(-1, ROW_TILE, kt, per // 4, 4)
    parts = []
    if full:
        parts.append(_pack_tiles(c[:full * ROW_TILE].view(full, ROW_TILE, kt, COL_TILE), s[:full]))
    if rest:
        parts.append(_pack_tiles(c[full * ROW_TILE:].view(1, h, kt, COL_TILE), s[full:]))
    return torch.cat(parts)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case)
    if case["op"] == "quantise":
        x = _activations(case["rows"], case["cols"], case["slack"], DTYPE[case["dtype"]], gen)
        state["x"] = x
        # the tensor scale of a calibration run, where the call does not measure it: about its largest value
        state["g"] = _tensor_scale(torch.full((), 45.0, device="cuda")) if case["fmt"] == "e4m3_16" and not case["measure"] else None
    elif case["op"] == "linear":
        state["x"] = _activations(case["rows"], case["k"], case["slack"], DTYPE[case["dtype"]], gen)
        w = torch.randn(case["n"], case["k"], generator=gen, device="cuda") * 0.02
        state["gx"] = _tensor_scale(torch.full((), 45.0, device="cuda")) if case["fmt"] == "e4m3_16" else None
        state["gw"] = _tensor_scale(w.abs().amax()) if case["fmt"] == "e4m3_16" else None
        codes, scales = _codes(w, case["fmt"], state["gw"])
        state["w"] = _pack(codes, scales, case["fmt"])      # the weights as a user keeps them: packed once
        state["bias"] = torch.randn(case["n"], generator=gen, device="cuda") * 0.1 if case["bias"] else None
    else:
        rows, vocab = case["rows"], case["vocab"]
        z = torch.randn(rows, vocab + case["slack"], generator=gen, device="cuda") * 3.0
        if case["masked"]:
            z[torch.rand(z.shape, generator=gen, device="cuda") < 0.2] = -math.inf
        state["logits"] = z.to(DTYPE[case["dtype"]])[:, :vocab]
        tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        # mostly likely words: the better of two draws
        other = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        at = torch.arange(rows, device="cuda")
        tokens = torch.where(z[at, other] > z[at, tokens], other, tokens)
        if case["masked"]:
            tokens = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.1, torch.full_like(tokens, -1), tokens)
        state["tokens"] = tokens
        state["temper"] = 1.0 if not case["masked"] else 1.25      # logits are multiplied with it
        if case["grad"]:
            state["g_logprob"] = -torch.rand(rows, generator=gen, device="cuda") / rows
            state["g_entropy"] = torch.randn(rows, generator=gen, device="cuda") * (0.01 / rows)
    return state


def work(case):
    if case["op"] == "quantise":
        n = case["rows"] * case["cols"]
        return {"bytes": n * BYTES[case["dtype"]] * 2, "flops": 4 * n}
    if case["op"] == "linear":
        m, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": m * k * 2 + n * k * (0.5 + 1 / BLOCK[case["fmt"]]) + m * n * 2, "flops": 2 * m * n * k}
    e = case["rows"] * case["vocab"]
    size = BYTES[case["dtype"]]
    return {"bytes": e * size * (2 if case["grad"] else 1) + case["rows"] * (16 + 16 * case["top"]), "flops": e * (12 if case["grad"] else 5)}


# ---- plain forms -------------------------------------------------------------

def _blocks(x, fmt):
    x = x.to(torch.float32)
    b = BLOCK[fmt]
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % b))
    return x.view(x.shape[0], -1, b)


def _e2m1(t):
    """Nearest of 0, .5, 1, 1.5, 2, 3, 4, 6, ties to the even code, as a code of 4 bits (the sign on top)."""
    a = t.abs()
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    return (code | (torch.signbit(t).to(torch.uint8) << 3)).to(torch.uint8)


def _e4m3_byte(v):
    """Non-negative values, rounded to the nearest float of 4 exponent and 3 mantissa bits (at most 448), as its byte."""
    v = v.clamp(max=448.0)
    _, e = torch.frexp(v)
    e = (e - 1).clamp(min=-6)                                       # exponent, or the subnormals' one
    m = torch.round(torch.ldexp(v, 3 - e)).to(torch.int32)         # 8..16, or 0..8 among the subnormals
    return ((e + 6) * 8 + m).to(torch.uint8)


def _e4m3_value(b):
    b = b.to(torch.int32)
    e, m = b >> 3, (b & 7).to(torch.float32)
    return torch.where(e > 0, torch.ldexp(1.0 + m / 8.0, e - 7), torch.ldexp(m, torch.full_like(e, -9)))


def _codes(x, fmt, g):
    """Codes [R, C] and scale bytes [R, blocks] of x."""
    v = _blocks(x, fmt)
    largest = v.abs().amax(2)
    if fmt == "e8m0_32":
        _, e = torch.frexp(largest)
        e = torch.where(largest > 0, (e - 3).clamp(min=-127), torch.full_like(e, -127))
        t = torch.ldexp(v, -e[:, :, None])
        scale = (e + 127).to(torch.uint8)
    else:
        scale = _e4m3_byte(largest / (6.0 * g))
        s = (_e4m3_value(scale) * g)[:, :, None]
        t = torch.where(s > 0, v / s, torch.zeros_like(v))
    return _e2m1(t).flatten(1)[:, :x.shape[1]], scale


def _e2m1_value(code):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=code.device)
    return table[code.to(torch.int32)]


def _values(codes, scales, fmt, g):
    q = _blocks(_e2m1_value(codes), fmt)
    if fmt == "e8m0_32":
        v = torch.ldexp(q, scales.to(torch.int32)[:, :, None] - 127)
    else:
        v = q * _e4m3_value(scales)[:, :, None] * g
    return v.flatten(1)[:, :codes.shape[1]]


def _unpack_tiles(data, t, h, kt, j):
    d = data.view(t, kt, h * 128 + j * 512)
    r = torch.arange(h, device=data.device)
    p = torch.arange(8, device=data.device)
    b = d[:, :, :h * 128].view(t, kt, h, 8, 16)[:, :, r[:, None], p[None, :] ^ (r % 8)[:, None]]
    b = b.permute(0, 2, 1, 3, 4).reshape(t * h, kt * 128)
    codes = torch.stack([b & 15, b >> 4], 2).flatten(1)
    s = d[:, :, h * 128:].view(t, kt, j, 32, 4, 4).permute(0, 4, 3, 1, 2, 5).reshape(t * 128, kt * j * 4)
    return codes, s


def _unpack(data, rows, cols, fmt):
    kt, j = -(-cols // COL_TILE), COL_TILE // BLOCK[fmt] // 4
    full = rows // ROW_TILE
    rest = rows - full * ROW_TILE
    cut = full * kt * (ROW_TILE * 128 + j * 512)
    h = -(-rest // 8) * 8
    c0, s0 = _unpack_tiles(data[:cut], full, ROW_TILE, kt, j)
    c1, s1 = _unpack_tiles(data[cut:], 1, h, kt, j) if rest else (c0[:0], s0[:0])
    blocks = -(-cols // BLOCK[fmt])
    return torch.cat([c0, c1])[:rows, :cols], torch.cat([s0, s1])[:rows, :blocks]


def _plain_quantise(s):
    x, fmt = s["x"], s["fmt"]
    g = s["g"]
    if s["measure"]:
        g = _tensor_scale(x.to(torch.float32).abs().amax())
    return _values(*_codes(x, fmt, g), fmt, g).to(x.dtype)


def _plain_linear(s):
    x, fmt = s["x"], s["fmt"]
    a = _values(*_codes(x, fmt, s["gx"]), fmt, s["gx"])
    b = _values(*_unpack(s["w"], s["n"], s["k"], fmt), fmt, s["gw"])
    y = a @ b.T
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(x.dtype)


def _plain_logprobs(s):
    z = s["logits"].to(torch.float32) * s["temper"]
    tokens = s["tokens"]
    m = z.amax(1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    p = e / total
    log_total = torch.log(total)
    # exp is 0 where a word is forbidden: its term is 0, not 0 times minus infinity
    terms = torch.where(e > 0, e * d, torch.zeros_like(e))
    entropy = log_total - terms.sum(1, keepdim=True) / total
    kept = tokens >= 0
    picked = d.gather(1, tokens.clamp(min=0)[:, None])
    logprob = torch.where(kept, (picked - log_total)[:, 0], torch.zeros_like(total[:, 0]))
    out = {"logprob": logprob, "entropy": entropy[:, 0]}
    if s["top"]:
        bits = (s["logits"].to(torch.float32) + 0.0).view(torch.int32)
        order = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).to(torch.int64) * (1 << 32)
        order = order + (z.shape[1] - 1 - torch.arange(z.shape[1], device=z.device))
        index = torch.topk(order, s["top"], dim=1).indices
        out["top_index"] = index
        out["top_logprob"] = d.gather(1, index) - log_total
    if s["grad"]:
        one = torch.zeros_like(p).scatter_(1, tokens.clamp(min=0)[:, None], kept.to(torch.float32)[:, None])
        g_logprob = torch.where(kept, s["g_logprob"], torch.zeros_like(s["g_logprob"]))[:, None]
        log_p = torch.where(e > 0, d - log_total, torch.zeros_like(d))
        grad = g_logprob * (one - p) - s["g_entropy"][:, None] * p * (log_p + entropy)
        out["grad"] = (grad * s["temper"]).to(s["logits"].dtype)
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


def _own_quantise(s):
    h = _handle()
    g = h.mx4_tensor_scale(s["x"]) if s["measure"] else s["g"]
    return h.mx4_dequantize(h.mx4_quantize(s["x"], s["fmt"], tensor_scale=g), s["x"].dtype)


def _own_linear(s):
    from paper_2406_11257_b200 import binding
    w = binding.Mx4Matrix(s["w"], s["n"], s["k"], s["fmt"], s["gw"])
    return _handle().mx4_linear(s["x"], w, bias=s["bias"], tensor_scale=s["gx"])


def _own_logprobs(s):
    h = _handle()
    r = h.token_logprobs(s["logits"], s["tokens"], top=s["top"], scale=s["temper"])
    out = {"logprob": r.logprob, "entropy": r.entropy}
    if s["top"]:
        out["top_index"], out["top_logprob"] = r.top_index, r.top_logprob
    if s["grad"]:
        out["grad"] = h.token_logprobs_grad(s["logits"], s["tokens"], r, s["g_logprob"], s["g_entropy"])
    return out


def run(state):
    op = state["op"]
    if own:
        return {"quantise": _own_quantise, "linear": _own_linear, "logprobs": _own_logprobs}[op](state)
    return {"quantise": _plain_quantise, "linear": _plain_linear, "logprobs": _plain_logprobs}[op](state)


# ---- the definitions in 64 bits ---------------------------------------------------

def _round64(x, step_table):
    """Nearest entry of an ascending table of non-negative values, ties to the entry of even place; beyond the last: the last."""
    table = torch.tensor(step_table, dtype=torch.float64, device=x.device)
    a = x.abs()
    at = torch.searchsorted(table, a.contiguous(), right=True).clamp(1, len(step_table) - 1) - 1      # table[at] <= a
    low, high = table[at], table[at + 1]
    up = (a - low > high - a) | ((a - low == high - a) & (at % 2 == 1))
    near = torch.where(up, high, low)
    return torch.where(x < 0, -near, near)


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
_E4M3 = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]


def _quantised64(x, fmt, g, measure=False):
    """The values that x's codes stand for."""
    rows, cols = x.shape
    b = BLOCK[fmt]
    v = torch.zeros(rows, -(-cols // b) * b, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, -1, b)
    top = v.abs().max(2, keepdim=True).values
    if fmt == "e8m0_32":
        unit = torch.exp2((torch.frexp(top.clamp(min=2.0 ** -149)).exponent - 3).clamp(min=-127).double())
        q = _round64(v / unit, _E2M1)
    else:
        if measure:
            m, e = np.frexp(float(x.double().abs().max()) / 2688.0)
            g = torch.tensor(float(np.ldexp(np.ceil(m * 256.0) / 256.0, e)), device=x.device)
        g = g.double()
        unit = _round64(top / (6.0 * g), _E4M3) * g
        q = _round64(torch.where(unit > 0, v / unit.clamp(min=1e-300), torch.zeros_like(v)), _E2M1)
    return (q * unit).view(rows, -1)[:, :cols]


def _weights64(data, rows, cols, fmt, g):
    """The packed matrix read value by value: the place of every code and scale from its row and column."""
    b = BLOCK[fmt]
    kt, scale_bytes = -(-cols // COL_TILE), COL_TILE // b * 128
    at_row = torch.arange(rows, device=data.device)[:, None]
    k = torch.arange(cols, device=data.device)[None, :]
    tile, r = at_row // ROW_TILE, at_row % ROW_TILE
    height = torch.where(tile < rows // ROW_TILE, ROW_TILE, -(-(rows % ROW_TILE) // 8) * 8)
    start = tile * kt * (ROW_TILE * 128 + scale_bytes) + (k // COL_TILE) * (height * 128 + scale_bytes)
    inside = k % COL_TILE
    byte = data[start + r * 128 + ((inside // 32) ^ (r % 8)) * 16 + inside % 32 // 2].to(torch.int64)
    code = torch.where(k % 2 == 0, byte % 16, byte // 16)
    block = inside // b
    scale = data[start + height * 128 + block // 4 * 512 + r % 32 * 16 + r // 32 * 4 + block % 4].to(torch.int64)
    value = torch.tensor(_E2M1, dtype=torch.float64, device=data.device)[code % 8] * torch.where(code >= 8, -1.0, 1.0).double()
    if fmt == "e8m0_32":
        return value * torch.exp2(scale.double() - 127)
    return value * torch.tensor(_E4M3 + [math.nan], dtype=torch.float64, device=data.device)[scale] * g.double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantise":
        return _quantised64(s["x"], s["fmt"], s["g"], s["measure"])
    if case["op"] == "linear":
        a = _quantised64(s["x"], s["fmt"], s["gx"])
        step = 4096            # rows of the weights at a time, for the memory
        kt = -(-case["k"] // COL_TILE)
        tile = kt * (ROW_TILE * 128 + COL_TILE // BLOCK[case["fmt"]] * 128)
        parts = []
        for first in range(0, case["n"], step):
            w = _weights64(s["w"][first // ROW_TILE * tile:], min(case["n"], first + step) - first, case["k"], s["fmt"], s["gw"])
            parts.append(a @ w.T)
        y = torch.cat(parts, 1)
        return y if s["bias"] is None else y + s["bias"].double()
    z = s["logits"].double() * s["temper"]
    log_p = torch.log_softmax(z, 1)
    p = torch.softmax(z, 1)
    at = torch.arange(case["rows"], device=z.device)
    kept = s["tokens"] >= 0
    t = s["tokens"].clamp(min=0)
    h = -torch.special.xlogy(p, p).sum(1)
    out = {"logprob": torch.where(kept, log_p[at, t], 0.0), "entropy": h}
    if case["top"]:
        out["top_index"] = None        # places, which have to be the plain form's
        out["top_logprob"] = torch.sort(log_p, 1, descending=True).values[:, :case["top"]]
    if case["grad"]:
        g = torch.special.xlogy(p, p)
        g.add_(p * h[:, None]).mul_(-s["g_entropy"].double()[:, None])
        gl = s["g_logprob"].double() * kept
        g.sub_(p * gl[:, None])
        g[at, t] += gl
        out["grad"] = g * s["temper"]
    return out
