"""Plain 64-bit definitions of the layers before the logits and of their gradients (include/excp.h): values in 8 bits,
activations, norms, products with their epilogue.  torch in float64 on whatever device the inputs are, no code in common with
the kernels.  Values in 8 bits take their scale and their quotient in fp32, as their definition says."""
from __future__ import annotations

import math

import torch


# ---- 8 bits ------------------------------------------------------------------------
def act8_codes(x: torch.Tensor):
    """(codes int8 [R, 32 B], scales float32 [R, B]) of x [R, C], B = ceil(C / 32)."""
    rows, cols = x.shape
    b = -(-cols // 32)
    v = torch.zeros(rows, b * 32, dtype=torch.float32, device=x.device)
    v[:, :cols] = x.to(torch.float32)
    v = v.view(rows, b, 32)
    bad = ~torch.isfinite(v).all(2)
    a = torch.where(bad, torch.zeros((), device=x.device), v.abs().amax(2)) / torch.tensor(127.0, device=x.device)
    # up to the next float whose lower 16 bits are zero
    bits = ((a.view(torch.int32) + 0xFFFF) >> 16) << 16
    s = bits.view(torch.float32).clamp(min=2.0 ** -126)
    q = torch.round(torch.where(bad[:, :, None], torch.zeros_like(v), v) * (1.0 / s)[:, :, None])
    return q.to(torch.int8).view(rows, -1), torch.where(bad, torch.full_like(s, math.nan), s)


def act8_pack(codes: torch.Tensor, scales: torch.Tensor) -> torch.Tensor:
    """The packed bytes, without the rounding up to 16."""
    return torch.cat([codes.contiguous().flatten().view(torch.uint8), scales.to(torch.bfloat16).contiguous().flatten().view(torch.uint8)])


def act8_values(codes: torch.Tensor, scales: torch.Tensor, cols: int) -> torch.Tensor:
    rows = codes.shape[0]
    return (codes.view(rows, -1, 32).double() * scales.double()[:, :, None]).reshape(rows, -1)[:, :cols]


def act8_round_trip(x: torch.Tensor) -> torch.Tensor:
    return act8_values(*act8_codes(x), x.shape[1])


# ---- activations -----------------------------------------------------------------------
def act(p: torch.Tensor, name: str) -> torch.Tensor:
    p = p.double()
    if name == "gelu":
        return p * 0.5 * torch.erfc(-p / math.sqrt(2.0))
    if name == "gelu_tanh":
        return 0.5 * p * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (p + 0.044715 * p ** 3)))
    if name == "silu":
        return p / (1.0 + torch.exp(-p))
    return p


def act_slope(p: torch.Tensor, name: str) -> torch.Tensor:
    p = p.double()
    if name == "gelu":
        return 0.5 * torch.erfc(-p / math.sqrt(2.0)) + p * torch.exp(-0.5 * p * p) / math.sqrt(2.0 * math.pi)
    if name == "gelu_tanh":
        k = math.sqrt(2.0 / math.pi)
        t = torch.tanh(k * (p + 0.044715 * p ** 3))
        return 0.5 * (1.0 + t) + 0.5 * p * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * p * p)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-p))
        return s + p * s * (1.0 - s)
    return torch.ones_like(p)


# ---- norms ---------------------------------------------------------------------------------
def norm(x, weight=None, bias=None, eps=1e-5, rms=False):
    """(y, mean [R], rstd [R])."""
    x = x.double()
    mean = torch.zeros_like(x[:, 0]) if rms else x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(1) + eps)
    y = d * rstd[:, None]
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return y, mean, rstd


def norm_grad(dy, x, weight, mean, rstd, rms=False, add=None):
    """(dx, dweight, dbias) with the mean and rstd given."""
    dy, x = dy.double(), x.double()
    xh = (x - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy if weight is None else dy * weight.double()
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if not rms:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * rstd.double()[:, None]
    return (dx if add is None else dx + add.double()), (dy * xh).sum(0), dy.sum(0)


# ---- products ----------------------------------------------------------------------------------
def linear(x, w, bias=None, name="none", residual=None):
    """(y, what goes into the activation)."""
    p = x.double() @ w.double().T
    if bias is not None:
        p = p + bias.double()
    y = act(p, name)
    return (y if residual is None else y + residual.double()), p
