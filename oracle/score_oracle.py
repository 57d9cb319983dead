"""Plain 64-bit definitions of the operators that score a restored checkpoint (include/excp.h): microscaled
4-bit matrices, their product, log probabilities of tokens and their gradient.  numpy, no GPU, no code in
common with the kernels.  Quantisation takes its divisions in fp32, as its definition says; everything else is
float64."""
from __future__ import annotations

import numpy as np

BLOCK = {"e8m0_32": 32, "e4m3_16": 16}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def _nearest(table: np.ndarray, x: np.ndarray) -> np.ndarray:
    """Index of the table entry nearest to each x >= 0 (ties to the even index; beyond the last: the last)."""
    x = np.asarray(x, np.float64)
    hi = np.clip(np.searchsorted(table, x, side="left"), 1, len(table) - 1)
    lo = hi - 1
    dl, dh = x - table[lo], table[hi] - x
    return np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)


def tensor_scale(x: np.ndarray) -> np.float32:
    a = np.abs(np.asarray(x, np.float32))
    a = a[np.isfinite(a)]
    q = np.float32(a.max() / np.float32(2688.0)) if a.size else np.float32(0)
    if not q > 0:
        return np.float32(1)
    m, e = np.frexp(np.float64(q))
    return np.float32(np.ldexp(np.ceil(m * 256) / 256, e))


def quantize(x: np.ndarray, fmt: str, g=None):
    """(codes uint8 [R, C], scale bytes uint8 [R, blocks])."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    b = BLOCK[fmt]
    nb = -(-cols // b)
    v = np.zeros((rows, nb * b), np.float32)
    v[:, :cols] = x
    v = v.reshape(rows, nb, b)
    bad = ~np.isfinite(v).all(2)
    v = np.where(bad[:, :, None], np.float32(0), v)
    a = np.abs(v).max(2)
    if fmt == "e8m0_32":
        e = np.frexp(a.astype(np.float64))[1] - 1 - 2
        e = np.where(a > 0, np.maximum(e, -127), -127)
        t = v.astype(np.float64) * np.ldexp(1.0, -e)[:, :, None]
        scale = np.where(bad, 255, e + 127).astype(np.uint8)
    else:
        g = np.float32(1 if g is None else g)
        with np.errstate(over="ignore"):
            byte = _nearest(E4M3, (a / (np.float32(6) * g)).astype(np.float32))
            sg = (E4M3[byte].astype(np.float32) * g)[:, :, None]
            t = np.where(sg > 0, v / np.where(sg > 0, sg, np.float32(1)), np.float32(0)).astype(np.float64)
        scale = np.where(bad, 127, byte).astype(np.uint8)
    code = _nearest(E2M1, np.abs(t)).astype(np.uint8) | (np.signbit(t).astype(np.uint8) << 3)
    code = np.where(bad[:, :, None], 0, code).astype(np.uint8)
    return code.reshape(rows, -1)[:, :cols], scale


def scale_values(scale: np.ndarray, fmt: str) -> np.ndarray:
    if fmt == "e8m0_32":
        return np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return np.append(E4M3, np.nan)[scale & 127]


def code_values(code: np.ndarray) -> np.ndarray:
    return E2M1[code & 7] * np.where(code & 8, -1.0, 1.0)


def values(codes: np.ndarray, scales: np.ndarray, fmt: str, g=None) -> np.ndarray:
    """What the codes stand for, in 64 bits (with the tensor scale)."""
    s = np.repeat(scale_values(scales, fmt), BLOCK[fmt], axis=1)[:, :codes.shape[1]]
    return code_values(codes) * s * (1.0 if g is None or fmt == "e8m0_32" else float(np.float32(g)))   # g is an fp32 number


def _place(rows: int, cols: int, fmt: str):
    """Byte offset of every code [R, C] and of every scale [R, blocks]."""
    b = BLOCK[fmt]
    ct, sb = -(-cols // 256), 256 // b * 128

    def tile_start(r, c):
        rt = r // 128
        h = np.where(rt < rows // 128, 128, -(-(rows % 128) // 8) * 8)
        return rt * ct * (128 * 128 + sb) + (c // 256) * (h * 128 + sb), h

    r = np.arange(rows, dtype=np.int64)[:, None]
    c = np.arange(cols, dtype=np.int64)[None, :]
    start, _ = tile_start(r, c)
    code = start + (r % 128) * 128 + (((c % 256) // 32) ^ (r % 8)) * 16 + (c % 32) // 2
    k = np.arange(-(-cols // b), dtype=np.int64)[None, :]
    start, h = tile_start(r, k * b)
    inside = k % (256 // b)
    scale = start + h * 128 + inside // 4 * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + inside % 4
    return code, scale


def packed_bytes(rows: int, cols: int, fmt: str) -> int:
    return -(-cols // 256) * (-(-rows // 8) * 8 * 128 + -(-rows // 128) * (256 // BLOCK[fmt] * 128))


def pack(codes: np.ndarray, scales: np.ndarray, fmt: str) -> np.ndarray:
    rows, cols = codes.shape
    out = np.zeros(packed_bytes(rows, cols, fmt), np.uint8)
    at, sat = _place(rows, cols, fmt)
    np.add.at(out, at, (codes << (4 * (np.arange(cols) % 2)).astype(np.uint8)).astype(np.uint8))
    out[sat] = scales
    return out


def unpack(data: np.ndarray, rows: int, cols: int, fmt: str):
    at, sat = _place(rows, cols, fmt)
    return (data[at] >> (4 * (np.arange(cols) % 2)).astype(np.uint8)) & 15, data[sat]


def logprobs(logits: np.ndarray, tokens: np.ndarray, scale: float = 1.0, top: int = 0):
    """dict of logprob, entropy, top_logprob, top_index and p, log_p (float64)."""
    x = np.asarray(logits, np.float64)
    z = x * scale
    rows, vocab = z.shape
    with np.errstate(all="ignore"):
        m = np.max(z, 1, keepdims=True, initial=-np.inf)       # NaN where the row holds one
        empty = (m == -np.inf)
        d = np.where(empty, -np.inf, z - m)
        s = np.exp(d).sum(1, keepdims=True)
        log_p = d - np.log(np.where(empty, 1.0, s))
        p = np.where(empty, 0.0, np.exp(log_p))
        h = -np.where(p == 0, 0.0, p * log_p).sum(1)
    out = {"p": p, "log_p": log_p, "entropy": h, "empty": empty[:, 0]}
    lp = np.zeros(rows)
    for i, t in enumerate(tokens):
        lp[i] = 0.0 if t < 0 else np.nan if t >= vocab else log_p[i, t]
    out["logprob"] = lp
    key = np.where(np.isnan(x), np.inf, x)
    index = np.zeros((rows, top), np.int64)
    for i in range(rows):
        order = sorted(range(vocab), key=lambda v: (0 if np.isnan(x[i, v]) else 1, -key[i, v], v))
        index[i] = order[:top]
    out["top_index"], out["top_logprob"] = index, np.take_along_axis(log_p, index, 1)
    return out


def logprobs_grad(logits, tokens, scale, g_logprob, g_entropy):
    r = logprobs(logits, tokens, scale)
    rows, vocab = r["p"].shape
    one = np.zeros((rows, vocab))
    keep = np.asarray(tokens) >= 0
    one[np.arange(rows)[keep], np.asarray(tokens)[keep]] = 1.0
    gl = (np.asarray(g_logprob, np.float64) * keep)[:, None]
    log_p = np.where(r["p"] == 0, 0.0, r["log_p"])
    g = gl * (one - r["p"]) - np.asarray(g_entropy, np.float64)[:, None] * r["p"] * (log_p + r["entropy"][:, None])
    return np.where(r["empty"][:, None], 0.0, g * scale)
