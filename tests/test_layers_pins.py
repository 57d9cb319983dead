"""The 64-bit definitions of the layers (oracle/layers_oracle.py) against hand values and differences, and what the library
answers without a GPU: sizes, refusals of null handles."""
import ctypes as C
import math

import pytest
import torch

from oracle import layers_oracle as lo
from paper_2406_11257_b200 import binding


def test_act8_by_hand():
    # A = 127: the scale is 1, codes are the rounded values, ties to even
    x = torch.tensor([[127.0, -127.0, 0.5, 1.5, -0.5, -2.5, 0.0, 3.25] + [0.0] * 24 + [-0.0, 254.0]])
    codes, scales = lo.act8_codes(x)
    assert scales.tolist() == [[1.0, 2.0]]
    assert codes[0, :8].tolist() == [127, -127, 0, 2, 0, -2, 0, 3]
    assert codes[0, 32:34].tolist() == [0, 127] and codes.shape == (1, 64)
    # 128 / 127 = 1.00787..: up to 8 significant bits, 1 + 2^-7 (steps of 2^-7 in [1, 2)) is not enough
    _, s = lo.act8_codes(torch.tensor([[128.0]]))
    assert s.item() == 1.0 + 2 * 2.0 ** -7 and 128.0 / 127.0 > 1.0 + 2.0 ** -7
    # zeros, tiny values, and what is not finite
    codes, s = lo.act8_codes(torch.tensor([[0.0] * 32 + [1e-42] * 32 + [1.0, math.inf] + [0.0] * 30 + [math.nan] * 32]))
    assert s[0, :2].tolist() == [2.0 ** -126] * 2 and torch.isnan(s[0, 2:]).all() and not codes.any()


def test_act8_is_off_by_half_a_step():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(50, 333, generator=g) * torch.exp(3 * torch.randn(50, 333, generator=g))
    codes, s = lo.act8_codes(x)
    step = s.repeat_interleave(32, 1)[:, :333].double()
    # half a step and the roundings of 1 / s and of the quotient (2^-24 of at most 127 steps each)
    assert ((lo.act8_values(codes, s, 333) - x.double()).abs() <= step * (0.5 + 127 * 2.0 ** -23)).all()
    assert codes.abs().max() == 127


def test_packed_layout():
    assert binding.act8_bytes(3, 33) == -(-3 * 2 * 34 // 16) * 16 and binding.act8_bytes(0, 5) == 0 and binding.act8_bytes(7, 0) == 0
    assert binding.act8_bytes(1 << 31, 1) == 0
    x = torch.arange(66, dtype=torch.float32).view(2, 33)
    b = lo.act8_pack(*lo.act8_codes(x))
    assert b.numel() == 2 * 2 * 34
    # the largest of a block: the scale is above A / 127 by at most 2^-7 of it, so the code is 126 or 127
    assert 126 <= b[31].item() <= 127
    assert 126 <= b[32].item() <= 127 and not b[33:64].any()    # 32 alone in its block, then padding
    scales = b[128:].view(torch.bfloat16).view(2, 2)
    assert (scales.double() * 127 >= torch.tensor([[31.0, 32.0], [64.0, 65.0]]).double()).all()


@pytest.mark.parametrize("name", ["gelu", "gelu_tanh", "silu"])
def test_slopes_against_differences(name):
    p = torch.linspace(-9, 9, 181, dtype=torch.float64)
    d = 1e-5
    want = (lo.act(p + d, name) - lo.act(p - d, name)) / (2 * d)
    assert (lo.act_slope(p, name) - want).abs().max() < 1e-8


@pytest.mark.parametrize("rms", [False, True])
def test_norm_gradient_against_differences(rms):
    g = torch.Generator().manual_seed(2)
    x, dy, w, b = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((3, 7), (3, 7), (7,), (7,)))
    score = lambda x, w, b: (dy * lo.norm(x, w, None if rms else b, 1e-5, rms)[0]).sum()
    _, mean, rstd = lo.norm(x, w, None, 1e-5, rms)
    dx, dw, db = lo.norm_grad(dy, x, w, mean, rstd, rms)
    d = 1e-6
    for t, grad in ((x, dx), (w, dw)) + (() if rms else ((b, db),)):
        for i in range(t.numel()):
            e = torch.zeros_like(t).view(-1)
            e[i] = d
            e = e.view_as(t)
            up, down = ((score(*(u + s * e if u is t else u for u in (x, w, b)))) for s in (1, -1))
            assert abs((up - down) / (2 * d) - grad.view(-1)[i]) < 1e-7


def test_product_gradients_are_the_transposed_products():
    g = torch.Generator().manual_seed(3)
    x, w, dy = (torch.randn(*s, generator=g, dtype=torch.float64).requires_grad_() for s in ((5, 4), (3, 4), (5, 3)))
    y, _ = lo.linear(x, w)
    dx, dw = torch.autograd.grad(y, (x, w), dy)
    assert torch.allclose(dx, dy @ w) and torch.allclose(dw, dy.T @ x)


def test_null_handles_are_refused():
    lib = binding.load_library()
    m = binding.CMatrix(None, 0, 0, 0, 0)
    r = C.byref(m)
    assert lib.excp_act8_quantize(None, r, None, None) == -1
    assert lib.excp_act8_restore(None, None, r, None) == -1
    assert lib.excp_act_grad(None, 1, r, r, None, None, None, None, None) == -1
    assert lib.excp_layer_norm(None, r, None, None, 0, 1e-5, 0, r, None, None, None) == -1
    assert lib.excp_layer_norm_grad(None, r, r, None, 0, 0, None, None, r, None, None, None, None) == -1
    assert lib.excp_linear(None, r, r, None, 0, 0, None, r, None, None, None) == -1
    assert lib.excp_linear_grad_input(None, r, r, None, r, None, None) == -1
    assert lib.excp_linear_grad_weight(None, r, r, None, r, None, None) == -1
    assert lib.excp_act_grad_scratch(None, 5, 5) == 0 and lib.excp_layer_norm_grad_scratch(None, 5, 5) == 0


def test_product_scratch_follows_alignment():
    lib = binding.load_library()
    mat = lambda p, rows, cols, stride, dtype=2: C.byref(binding.CMatrix(p, dtype, rows, cols, stride))
    tidy = mat(1 << 20, 10, 100, 104)
    assert lib.excp_linear_scratch(tidy, tidy) == 0
    assert lib.excp_linear_scratch(tidy, mat(1 << 20, 10, 100, 101)) == 10 * 128 * 2      # rows of 64 values or more
    assert lib.excp_linear_scratch(mat((1 << 20) + 2, 1, 100, 7), tidy) == 128 * 2
    assert lib.excp_linear_scratch(mat(1 << 20, 1, 100, 7), tidy) == 0                    # one row has no stride
    assert lib.excp_linear_scratch(None, tidy) == 0
