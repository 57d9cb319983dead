"""The layers before the logits and their gradients, through the C ABI, against their plain 64-bit definitions.

Tolerances (derived, not fitted), with u = 2^-24:
  8 bits       packed bytes and restored values equal.
  activations  value: |p| 2^-20.  The tail of the normal distribution is within 2^-22 (polynomial) and (4 + p^2) 2^-23 (the exponential and
               its argument) of itself, and its share of |p| is largest, 0.5, at 0, where p^2 adds nothing (p^2 tail < 0.2); 1 - tail is
               rounded by u.  The sigmoids: 2^-22 (exponential), 2 u (sum, reciprocal), argument |z| 3 u times s (1 - s) <= 0.23 / |z|.
               slope: 2^-17.  As above times the slope's other factors: x phi(x) p^2 < 0.5; and x s (1 - s) inner, where 1 - s is off by
               2 u and x inner < 40 as long as s is not 1 (x < 5.2 for gelu_tanh, x < 17 for silu).
  norms        a sum of n values adds at most n / 32 / 8 + 8 + 21 values one after the other (eight of a thread and piece, 5 shuffles, 16
               warps), and at most cols / 4096 + .. of a long row: ADDS u of the sum of magnitudes.
  products     the tensor core adds ceil(K / 16) partial sums to an fp32 accumulator, and up to 8 accumulators are added; each addition is
               off by at most 2^-22 of the sum of magnitudes (truncation included); bias, residual and activation add a rounding each; then one
               rounding to the result's type.
  column sums  rows are added in chains of at most rows / 8 / groups + 8 + 8 + groups / 8 values: (rows / 8 + 40) u of the sum of magnitudes.
"""
import math

import pytest
import torch

from oracle import layers_oracle as lo
from paper_2406_11257_b200 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}      # half a step among fp16's subnormals
U = 2.0 ** -24
ACTS = ["gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(workspace_numel=4096, device=0)
    yield handle
    handle.score_status()
    handle.close()


def make(rows, cols, dtype, seed, slack=0, offset=0, size=1.0):
    """Normals with outliers in a buffer with `slack` more columns, starting `offset` elements in."""
    g = torch.Generator().manual_seed(seed)
    n = rows * (cols + slack) + offset
    x = torch.randn(n, generator=g) * size
    x[torch.rand(n, generator=g) < 0.01] *= 8
    buf = x.to(DT.get(dtype, dtype)).to(DEV)
    return buf[offset:].view(rows, cols + slack)[:, :cols]


def vector(n, dtype, seed, size=1.0, mean=0.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, generator=g) * size + mean).to(DT.get(dtype, dtype)).to(DEV)


def near(got, want, tol, what=""):
    """|got - want| <= tol + a rounding of got's type; NaN where the other has it."""
    g, w = got.double(), want.double()
    assert torch.equal(torch.isnan(g), torch.isnan(w)), what
    t = torch.as_tensor(tol, device=g.device, dtype=torch.float64) + HALF_ULP[got.dtype] * 1.01 * w.abs() + TINY[got.dtype]
    bad = ((g - w).abs() > t) & ~torch.isnan(w)
    if bad.any():
        i = bad.nonzero()[0].tolist()
        at = tuple(i)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {g[at].item()} for {w[at].item()}, allowed "
                             f"{t.expand_as(g)[at].item():.3g}, off {(g - w).abs()[at].item():.3g}")


# ---- 8 bits -------------------------------------------------------------------------
SHAPES = [(1, 1), (1, 4096), (3, 31), (8, 256), (9, 257), (127, 33), (2, 1000), (130, 17), (5, 2049)]


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_act8_and_back(h, rows, cols, dtype):
    for slack, offset in ((0, 0), (5, 0), (8, 8), (0, 1)):
        x = make(rows, cols, dtype, rows * 7 + cols, slack, offset, size=3.0)
        need = binding.act8_bytes(rows, cols)
        room = torch.full((need + 64,), 0xAB, dtype=torch.uint8, device=DEV)
        m = h.act8_quantize(x, out=room)
        want = lo.act8_pack(*lo.act8_codes(x))
        assert torch.equal(m.data[:want.numel()], want)
        assert bool((room[need:] == 0xAB).all())
        values = lo.act8_round_trip(x)
        for out in DT.values():
            assert torch.equal(h.act8_restore(m, out), values.float().to(out))
        wide = torch.full((rows, cols + 3), 7.0, device=DEV)
        h.act8_restore(m, out=wide[:, :cols])
        assert torch.equal(wide[:, :cols].double(), values) and bool((wide[:, cols:] == 7).all())


def test_act8_without_the_bytes_behind_the_last_scale(h):
    """3 * 3 blocks are 306 bytes, of the 320 that a buffer is given: what says all of the values is taken as it is."""
    x = make(3, 70, "bf16", 5)
    data = lo.act8_pack(*lo.act8_codes(x))
    assert data.numel() == 306 and binding.act8_bytes(3, 70) == 320
    m = binding.Act8Matrix(data, 3, 70)
    assert torch.equal(h.act8_restore(m, torch.float32).double(), lo.act8_round_trip(x))
    whole = h.act8_quantize(x)
    dy = make(3, 70, "bf16", 6)
    assert torch.equal(h.act_grad(dy, m, act="gelu").dpre, h.act_grad(dy, whole, act="gelu").dpre)
    with pytest.raises(TypeError):
        h.act8_restore(binding.Act8Matrix(data[:305], 3, 70), torch.float32)


def test_act8_extreme_values(h):
    g = torch.Generator().manual_seed(5)
    x = torch.randn(64, 320, generator=g) * torch.exp(torch.randn(64, 320, generator=g) * 25)
    x[3, 5], x[4, 40], x[5, 319] = math.nan, math.inf, -math.inf
    x[6], x[7], x[8] = 0.0, 3.4e38, 1e-45
    x[9, :32] = torch.tensor([127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 63.5, 126.5] * 4)
    x = x.to(DEV)
    for t in (x, x.to(torch.bfloat16), torch.cat([torch.zeros(64, 1, device=DEV), x], 1)[:, 1:]):
        m = h.act8_quantize(t)
        want = lo.act8_pack(*lo.act8_codes(t))
        # the bits of a NaN scale are not compared
        rows, b = t.shape[0], t.shape[1] // 32
        nan = torch.isnan(want[rows * b * 32:].view(torch.bfloat16).float())
        got = m.data[:want.numel()]
        assert torch.equal(got[:rows * b * 32], want[:rows * b * 32])
        s = got[rows * b * 32:].view(torch.bfloat16)
        assert torch.equal(torch.isnan(s.float()), nan)
        assert torch.equal(s[~nan], want[rows * b * 32:].view(torch.bfloat16)[~nan])
        y, v = h.act8_restore(m), lo.act8_round_trip(t)
        assert torch.equal(torch.isnan(y), torch.isnan(v)) and torch.equal(y[~torch.isnan(v)].double(), v[~torch.isnan(v)])


# ---- the way back through an activation ----------------------------------------------------
@pytest.mark.parametrize("kept", ["plain", "act8"])
@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("act", ACTS)
def test_act_grad(h, act, dtype, kept):
    for rows, cols, slack, offset in ((1, 1, 0, 0), (1, 4096, 0, 0), (3, 31, 5, 0), (70, 257, 0, 1), (333, 1000, 8, 8), (2000, 40, 0, 0), (17, 520, 1, 3)):
        p = make(rows, cols, dtype, rows + cols, slack, offset, size=2.0)
        dy = make(rows, cols, dtype, rows * 3 + cols, 0, offset)
        pre = h.act8_quantize(p) if kept == "act8" else p
        v = lo.act8_round_trip(p) if kept == "act8" else p.double()
        r = h.act_grad(dy, pre, act, again=True)
        want = dy.double() * lo.act_slope(v, act)
        near(r.a, lo.act(v, act), v.abs() * 2.0 ** -20, "again")
        near(r.dpre, want, dy.double().abs() * 2.0 ** -17, "dpre")
        size = (dy.double().abs() * (lo.act_slope(v, act).abs() * (rows / 8 + 40) * U + 2.0 ** -17)).sum(0)
        near(r.dbias, want.sum(0), size, "dbias")
        alone = h.act_grad(dy, pre, act, bias=False)
        assert alone.dbias is None and alone.a is None and torch.equal(alone.dpre, r.dpre)
        in_place = dy.clone()
        assert h.act_grad(in_place, pre, act, out=in_place).dpre is in_place and torch.equal(in_place, r.dpre)


def test_activations_over_their_range(h):
    """Far out, where one factor is 0, and at what the formulas make of infinities and NaN."""
    p = torch.cat([torch.linspace(-30, 30, 6001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e4, -1e4, 1e18, -1e18, 3e38, -3e38])]).to(DEV)[None]
    one = torch.ones_like(p)
    for act in ACTS:
        r = h.act_grad(one, p, act, again=True)
        value = lo.act(p, act)
        near(r.a, value, p.double().abs() * 2.0 ** -20, act)
        fine = p.abs() <= 1e4                      # beyond, the definition's own x^3 and x^2 times 0
        near(r.dpre[fine], lo.act_slope(p, act)[fine], 2.0 ** -17, act)
        assert bool((r.dpre[~fine] == (p[~fine] > 0).float()).all())
        far = torch.tensor([[math.inf, math.nan, 5.0]], device=DEV)
        r = h.act_grad(torch.ones_like(far), far, act, again=True)
        assert r.a[0, 0] == math.inf and torch.isnan(r.a[0, 1]) and torch.isnan(r.dpre[0, 1]) and r.a[0, 2] > 4.9


def test_bias_grad(h):
    for rows, cols, slack in ((0, 5, 0), (1, 1, 0), (7, 333, 3), (4097, 300, 0), (100, 5000, 0)):
        for dtype in sorted(DT):
            dy = make(rows, cols, dtype, rows + cols, slack)
            got = h.bias_grad(dy)
            assert got.dtype == torch.float32
            near(got, dy.double().sum(0), dy.double().abs().sum(0) * (rows / 8 + 40) * U)


# ---- norms -----------------------------------------------------------------------------------------
NORM_SHAPES = [(1, 1), (1, 4096), (3, 31), (5, 256), (9, 257), (130, 1000), (2, 4097), (3, 9000), (2, 16384), (600, 64), (3, 16390), (2, 40001)]


def adds(cols):
    return 8 * max(1, cols / 512 / 8) + 8 + 21


def check_norm(h, x, w, b, rms, eps=1e-5):
    cols = x.shape[1]
    r = h.layer_norm(x, w, b, eps=eps, rms=rms)
    y, mean, rstd = lo.norm(x, w, b, eps, rms)
    a = adds(cols) * U
    d = x.double()
    off_mean = 0.0 * mean if rms else d.abs().mean(1) * (a + 2 * U)
    near(r.row_stats[:, 0], mean, off_mean)
    # (x - mean)^2: twice the error of x - mean, which the sum averages; and the sum's own
    dev = (d - mean[:, None]).abs()
    # an error e of the mean moves every x - mean alike: the sum of squares by cols e^2; the rest are roundings
    rel = a + 8 * U + (off_mean * rstd) ** 2
    near(r.row_stats[:, 1], rstd, rstd * rel)
    xh = dev * rstd[:, None]
    ww = torch.ones(cols, device=x.device).double() if w is None else w.double().abs()
    tol = ww * (xh * (rel[:, None] + 4 * U) + (off_mean * rstd)[:, None] + d.abs() * rstd[:, None] * U) + (0.0 if b is None else b.double().abs() * U)
    near(r.y, y, tol, "y")
    return r, mean, rstd


def check_norm_grad(h, dy, x, v, w, r, add=None):
    """x: what the call takes, v: its values."""
    rows, cols = dy.shape
    mean, rstd = r.row_stats[:, 0].double(), r.row_stats[:, 1].double()
    g = h.layer_norm_grad(dy, x, w, r, add=add)
    dx, dw, db = lo.norm_grad(dy, v, w, mean, rstd, r.rms, add)
    d, v = dy.double().abs(), v.double()
    xh = ((v - mean[:, None]) * rstd[:, None]).abs()
    off_xh = xh * 2 * U + v.abs() * rstd[:, None] * U
    ww = torch.ones(cols, device=dy.device).double() if w is None else w.double().abs()
    gg = d * ww
    a = (adds(cols) + 4) * U
    m1, m2 = gg.mean(1, keepdim=True), (gg * xh).mean(1, keepdim=True)
    off_m2 = (gg * off_xh).mean(1, keepdim=True) + a * m2
    tol = rstd[:, None] * (4 * U * gg + (0.0 if r.rms else a * m1 + 2 * U * m1) + off_xh * m2 + xh * off_m2 + 3 * U * xh * m2)
    if add is not None:
        tol = tol + U * (add.double().abs() + dx.abs())
    near(g.dx, dx, tol, "dx")
    n = (rows + 40) * U
    near(g.dweight, dw, (d * (off_xh + xh * n)).sum(0), "dweight")
    if r.rms:
        assert g.dbias is None
    else:
        near(g.dbias, db, d.sum(0) * n, "dbias")
    return g


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_norm_and_gradient(h, rows, cols, dtype, rms):
    for slack, offset, vt, plain in ((0, 0, dtype, False), (5, 0, "fp32", False), (8, 8, dtype, True), (0, 1, "fp32", True)):
        x = make(rows, cols, dtype, rows * 7 + cols, slack, offset) + 0.25
        if slack:
            x = torch.cat([x, x[:, :1].expand(-1, slack)], 1)[:, :cols]
        w = None if plain else vector(cols, vt, 1, 0.2, 1.0)
        b = None if plain or rms else vector(cols, vt, 2, 0.1)
        r, _, _ = check_norm(h, x, w, b, rms)
        dy = make(rows, cols, dtype, rows + 3 * cols, slack, offset)
        add = make(rows, cols, dtype, 5, 0, offset) if slack else None
        check_norm_grad(h, dy, x, x, w, r, add)
        kept = h.layer_norm(x, w, b, rms=rms, keep=True)
        assert torch.equal(kept.y, r.y) and torch.equal(kept.row_stats, r.row_stats)
        packed = lo.act8_pack(*lo.act8_codes(x))
        assert torch.equal(kept.kept.data[:packed.numel()], packed)
        check_norm_grad(h, dy, kept.kept, lo.act8_round_trip(x), w, r, add)


def test_norm_in_place_and_subsets(h):
    for cols in (300, 4096, 20000):
        x, dy, add = (make(50, cols, "bf16", s) for s in (1, 2, 3))
        w, b = vector(cols, "bf16", 4), vector(cols, "bf16", 5)
        r = h.layer_norm(x, w, b)
        y = x.clone()
        assert h.layer_norm(y, w, b, out=y).y is y and torch.equal(y, r.y)
        g = h.layer_norm_grad(dy, x, w, r, add=add)
        assert torch.equal(h.layer_norm_grad(dy, x, w, r, add=add, vectors=False).dx, g.dx)
        for place in (dy.clone(), add.clone()):
            same = h.layer_norm_grad(place if torch.equal(place, dy) else dy, x, w, r, add=place if torch.equal(place, add) else add, out=place)
            assert same.dx is place and torch.equal(place, g.dx) and torch.equal(same.dweight, g.dweight) and torch.equal(same.dbias, g.dbias)


def test_norm_of_special_rows(h):
    x = make(6, 500, "fp32", 1)
    x[1] = 3.0                                     # no deviation: 1 / sqrt(eps)
    x[2, 7], x[3, 9] = math.nan, math.inf
    x[4] = x[4] * 1e-3 + 4096.0                    # a mean far from 0
    w, b = vector(500, "fp32", 2), vector(500, "fp32", 3)
    r, _, _ = check_norm(h, x[[0, 1, 4, 5]].contiguous(), w, b, False)
    assert r.row_stats[1, 1].item() == pytest.approx(1e5 ** 0.5, rel=1e-6) and torch.equal(r.y[1], b)
    r = h.layer_norm(x, w, b)
    assert torch.isnan(r.y[2:4]).all() and torch.isfinite(r.y[[0, 1, 4, 5]]).all()
    dy = make(6, 500, "fp32", 9)
    g = h.layer_norm_grad(dy, x, w, r)
    assert torch.isnan(g.dx[2:4]).all() and torch.isfinite(g.dx[[0, 1, 4, 5]]).all()
    # no rows: the vectors are 0
    none = h.layer_norm(x[:0], w, b)
    g = h.layer_norm_grad(dy[:0], x[:0], w, none)
    assert g.dx.shape == (0, 500) and not g.dweight.any() and not g.dbias.any()


# ---- products ------------------------------------------------------------------------------------------
PRODUCT_SHAPES = [  # rows, k, n
    (1, 64, 128), (1, 1, 1), (1, 4096, 1000), (3, 100, 33), (16, 512, 300), (17, 65, 129), (64, 1000, 520), (129, 200, 130), (128, 128, 128),
    (200, 64, 70), (300, 1000, 257), (1000, 333, 100), (2304, 72, 2304), (2305, 200, 2049), (40, 8200, 48)]


def magnitude(a, b):
    return a.double().abs() @ b.double().abs().T


def product_tol(a, b):
    return magnitude(a, b) * ((a.shape[1] + 15) // 16 + 12) * 2.0 ** -22


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,k,n", PRODUCT_SHAPES)
def test_linear(h, rows, k, n, dtype):
    for case, (slack, offset, act, bt, rt, out) in enumerate((
            (0, 0, "none", None, None, dtype), (8, 8, "gelu", dtype, dtype, dtype), (5, 0, "silu", "fp32", "fp32", "fp32"), (0, 1, "gelu_tanh", None, dtype, "bf16"))):
        x = make(rows, k, dtype, rows + k, slack, offset)
        w = make(n, k, dtype, n + k + case, slack, offset, size=0.1)
        bias = None if bt is None else vector(n, bt, 3)
        residual = None if rt is None else make(rows, n, rt, 4, slack if rt == dtype else 0)
        y, p = lo.linear(x, w, bias, act, residual)
        got = h.linear(x, w, bias, act=act, residual=residual, dtype=DT[out])
        tol_p = product_tol(x, w) + U * p.abs()
        tol = 1.2 * tol_p + (0.0 if act == "none" else p.abs() * 2.0 ** -20) + (0.0 if residual is None else U * y.abs())
        near(got, y, tol, f"y of case {case}")
        if case == 1:                              # into a part of a wider buffer, which is the residual
            room = torch.full((rows, n + 24), 7.0, dtype=DT[dtype], device=DEV)
            room[:, 8:8 + n] = residual
            h.linear(x, w, bias, act=act, residual=room[:, 8:8 + n], out=room[:, 8:8 + n])
            near(room[:, 8:8 + n], y, tol, "in place")
            assert bool((room[:, :8] == 7).all()) and bool((room[:, 8 + n:] == 7).all())
        for keep in ("act8", torch.float32, torch.bfloat16):
            again, kept = h.linear_kept(x, w, bias, act=act, residual=residual, keep=keep, dtype=DT[out])
            assert torch.equal(again, got)
            if keep != "act8":
                near(kept, p, tol_p, "kept")
                continue
            # off by half a step of its block, and by what the scale moves with A: 2^-7
            top = torch.zeros(rows, -(-n // 32) * 32, device=DEV, dtype=torch.float64)
            top[:, :n] = p.abs()
            step = (top.view(rows, -1, 32).amax(2) / 127 * (1 + 2.0 ** -7)).repeat_interleave(32, 1)[:, :n]
            near(h.act8_restore(kept), p, tol_p * 1.1 + step * 0.501 + 2.0 ** -126, "kept in 8 bits")
            q, s = lo.act8_codes(h.linear_kept(x, w, bias, act=act, residual=residual, keep=torch.float32, dtype=DT[out])[1])
            assert torch.equal(kept.data[:q.numel() + 2 * s.numel()], lo.act8_pack(q, s))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,k,n", PRODUCT_SHAPES)
def test_linear_gradients(h, rows, k, n, dtype):
    for slack, offset in ((0, 0), (8, 8), (5, 0), (0, 1)):
        x = make(rows, k, dtype, rows + k, slack, offset)
        w = make(n, k, dtype, n + k, slack, offset, size=0.1)
        dy = make(rows, n, dtype, rows + n, slack, offset)
        dx, dw = dy.double() @ w.double(), dy.double().T @ x.double()
        tol_x, tol_w = product_tol(dy, w.T), product_tol(dy.T, x.T)
        near(h.linear_grad_input(dy, w), dx, tol_x, "dx")
        got = h.linear_grad_weight(dy, x)
        assert got.dtype == torch.float32
        near(got, dw, tol_w, "dw")
        add = make(rows, k, dtype, 9, slack)
        near(h.linear_grad_input(dy, w, add=add, dtype=torch.float32), dx + add.double(), tol_x + U * add.double().abs(), "dx + add")
        near(h.linear_grad_weight(dy, x, dtype=DT[dtype]), dw, tol_w, "dw in 16 bits")
        h.linear_grad_weight(dy, x, add=got, out=got)                      # a second micro-batch
        near(got, 2 * dw, 2 * tol_w + 2 * U * dw.abs(), "dw twice")


def test_products_of_nothing(h):
    for rows, k, n in ((0, 5, 7), (5, 0, 7), (5, 7, 0), (300, 0, 300)):
        x, w = make(rows, k, "bf16", 1), make(n, k, "bf16", 2)
        bias, residual = vector(n, "fp32", 3), make(rows, n, "bf16", 4)
        y, p = lo.linear(x, w, bias, "gelu", residual)
        near(h.linear(x, w, bias, act="gelu", residual=residual), y, p.abs() * 2.0 ** -20 + U * y.abs())
        dy = make(rows, n, "bf16", 5)
        assert torch.equal(h.linear_grad_input(dy, w).double(), dy.double() @ w.double()) or n
        near(h.linear_grad_weight(dy, x), dy.double().T @ x.double(), product_tol(dy.T, x.T))


def test_infinities_and_nan_stay_in_their_rows(h):
    for rows in (4, 300):
        x, w = make(rows, 200, "bf16", 1), make(400, 200, "bf16", 2)
        clean = h.linear(x, w)
        x[2, 3], x[3, 199] = math.nan, math.inf
        y = h.linear(x, w)
        keep = [i for i in range(rows) if i not in (2, 3)]
        assert torch.equal(y[keep], clean[keep]) and torch.isnan(y[2]).all() and not torch.isfinite(y[3]).any()


# ---- how the calls are made ----------------------------------------------------------------------------------
def mlp_step(h, x, w, b, nw, nb, dy, run=None):
    """A residual MLP block forward and backward as a training step runs it, activations kept in 8 bits."""
    n = h.layer_norm(x, nw, nb, keep=True)
    a, pre = h.linear_kept(n.y, w[0], b[0], act="gelu", keep="act8")
    y = h.linear(a, w[1], b[1], residual=x)
    g = {"y": y, "w1": h.linear_grad_weight(dy, a), "b1": h.bias_grad(dy)}
    r = h.act_grad(h.linear_grad_input(dy, w[1]), pre, "gelu")
    g["b0"], g["w0"] = r.dbias, h.linear_grad_weight(r.dpre, n.y)
    ng = h.layer_norm_grad(h.linear_grad_input(r.dpre, w[0]), n.kept, nw, n, add=dy)
    return {**g, "x": ng.dx, "nw": ng.dweight, "nb": ng.dbias}


def mlp_inputs(tokens, d, f, seed=1, dtype="bf16"):
    return dict(x=make(tokens, d, dtype, seed), w=[make(f, d, dtype, seed + 1, size=0.05), make(d, f, dtype, seed + 2, size=0.05)],
                b=[vector(f, dtype, seed + 3, 0.1), vector(d, dtype, seed + 4, 0.1)], nw=vector(d, dtype, seed + 5, 0.2, 1.0), nb=vector(d, dtype, seed + 6, 0.1),
                dy=make(tokens, d, dtype, seed + 7, size=0.1))


@pytest.mark.parametrize("tokens,d,f", [(1, 64, 256), (200, 256, 1024), (777, 200, 1000)])
def test_an_mlp_block_forward_and_backward(h, tokens, d, f):
    """Against torch's autograd in 64 bits.  Between the operators values are rounded to 16 and 8 bits, so a gradient is compared as a
    whole: the relative error of a sum of products whose factors are each off by at most r is about r.  Three 16-bit roundings
    (2^-8) and two 8-bit ones (half of 1 / 127 of a block's largest magnitude, some three deviations) in the chain make at most
    3 * 2^-8 + 2 * 1.5 / 127 = 0.036; a wrong term makes more than 0.1 of any gradient here."""
    i = mlp_inputs(tokens, d, f)
    got = mlp_step(h, **i)
    leaf = lambda t: t.double().requires_grad_()
    x, w, b, nw, nb = leaf(i["x"]), [leaf(t) for t in i["w"]], [leaf(t) for t in i["b"]], leaf(i["nw"]), leaf(i["nb"])
    n = torch.nn.functional.layer_norm(x, (d,), nw, nb)
    y = torch.nn.functional.gelu(n @ w[0].T + b[0]) @ w[1].T + b[1] + x
    grads = torch.autograd.grad(y, [x, w[0], b[0], w[1], b[1], nw, nb], i["dy"].double())
    for name, want in zip(["y", "x", "w0", "b0", "w1", "b1", "nw", "nb"], [y.detach(), *grads]):
        assert (got[name].double() - want).norm() <= 0.036 * want.norm(), name


def test_captured_and_replayed(h):
    """A graph of a training step: replayed on new contents of the same tensors, it gives what the calls give; two graphs on one
    handle, replayed at once on two streams, do not disturb each other."""
    a, b = mlp_inputs(130, 128, 512, 1), mlp_inputs(700, 1024, 512, 20)
    eager = [mlp_step(h, **a), mlp_step(h, **b)]
    torch.cuda.synchronize()
    graphs, results = [], []
    for i in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(mlp_step(h, **i))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for r, e in zip(results, eager):
        for k in e:
            assert torch.equal(r[k], e[k]), k
    new = mlp_inputs(130, 128, 512, 50)
    want = mlp_step(h, **new)
    for k in ("x", "nw", "nb", "dy"):
        a[k].copy_(new[k])
    for k in ("w", "b"):
        for t, u in zip(a[k], new[k]):
            t.copy_(u)
    graphs[0].replay()
    torch.cuda.synchronize()
    for k in want:
        assert torch.equal(results[0][k], want[k]), k


def test_same_bits_every_time(h):
    i = mlp_inputs(1000, 512, 2048, 3)
    first = mlp_step(h, **i)
    for _ in range(3):
        again = mlp_step(h, **i)
        for k in first:
            assert torch.equal(first[k], again[k]), k


def test_on_another_stream_and_a_fresh_handle():
    other = binding.Handle(workspace_numel=4096, device=0)
    i = mlp_inputs(64, 128, 256, 4)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = mlp_step(other, **i)
    s.synchronize()
    want = mlp_step(other, **i)
    for k in want:
        assert torch.equal(got[k], want[k]), k
    other.score_status()
    other.close()


def test_rows_past_the_last_stay_as_they_are(h):
    """Results into the first rows and columns of a larger buffer."""
    for rows, k, n in ((5, 96, 100), (130, 64, 257), (300, 200, 520)):
        x, w = make(rows, k, "bf16", 1), make(n, k, "bf16", 2)
        room = torch.full((rows + 3, n + 8), 7.0, dtype=torch.bfloat16, device=DEV)
        h.linear(x, w, out=room[:rows, :n])
        assert torch.equal(room[:rows, :n], h.linear(x, w)) and bool((room[rows:] == 7).all()) and bool((room[:, n:] == 7).all())
        t = make(rows, n, "bf16", 3)
        room.fill_(7.0)
        h.layer_norm(t, out=room[:rows, :n])
        assert torch.equal(room[:rows, :n], h.layer_norm(t).y) and bool((room[rows:] == 7).all()) and bool((room[:, n:] == 7).all())
        room.fill_(7.0)
        h.act_grad(t, t, "silu", out=room[:rows, :n])
        assert torch.equal(room[:rows, :n], h.act_grad(t, t, "silu").dpre) and bool((room[rows:] == 7).all()) and bool((room[:, n:] == 7).all())


def test_waits_that_run_out():
    """No time at all: the products report it and the handle stays usable."""
    other = binding.Handle(workspace_numel=4096, device=0)
    shapes = ((4, 512, 300), (64, 4096, 1024), (2304, 256, 2304))
    for rows, k, n in shapes:
        x, w = make(rows, k, "bf16", 1), make(n, k, "bf16", 2)
        want = other.linear(x, w)
        other.score_status()
        other.set_wait_limit(0)
        other.linear(x, w)
        with pytest.raises(binding.ExcpError) as e:
            other.score_status()
        assert e.value.status == -7
        other.set_wait_limit(2_000_000_000)
        assert torch.equal(other.linear(x, w), want)
        other.score_status()
    other.close()


def test_offsets_past_32_bits(h):
    """Rows whose bytes and elements lie past 2^32 and 2^31 of their buffer."""
    cols, rows = 65536 + 64, 33000                 # 2.16e9 elements of 2 bytes
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    last = make(8, cols, "bf16", 1)
    x[-8:] = last
    y = torch.empty_like(x)
    r = h.layer_norm(x, out=y)
    want, mean, rstd = lo.norm(last)
    near(r.y[-8:], want, (last.double().abs() + mean.abs()[:, None]) * rstd[:, None] * adds(cols) * U * 2)
    g = h.layer_norm_grad(x, x, None, r, out=y)
    dx, _, _ = lo.norm_grad(last, last, None, r.row_stats[-8:, 0], r.row_stats[-8:, 1])
    near(g.dx[-8:], dx, rstd[:, None] * last.double().abs().amax(1, keepdim=True) * adds(cols) * U * 8 * (1 + last.double().abs()))
    near(g.dbias, x[-8:].double().sum(0), x[-8:].double().abs().sum(0) * 64 * U)
    m = h.act8_quantize(x)
    codes, scales = lo.act8_codes(last)
    b = cols // 32
    assert torch.equal(m.data[(rows - 8) * cols:rows * cols].view(torch.int8).view(8, -1), codes)
    assert torch.equal(m.data[rows * cols + (rows - 8) * b * 2:rows * cols + rows * b * 2].view(torch.bfloat16).view(8, b).float(), scales)
    h.act8_restore(m, out=y)
    assert torch.equal(y[-8:].double(), lo.act8_round_trip(last).bfloat16().double())
    got = h.act_grad(x, m, "silu", out=y)
    v = lo.act8_round_trip(last)
    near(got.dpre[-8:], last.double() * lo.act_slope(v, "silu"), last.double().abs() * 2.0 ** -17)
    del m, y, g, r, got
    # as an operand: few rows of a long matrix, and its gradients
    w = make(16, cols, "bf16", 2, size=0.1)
    p = h.linear(x, w, dtype=torch.float32)
    near(p[-8:], last.double() @ w.double().T, product_tol(last, w))
    assert not p[:-8].any()
    dw = h.linear_grad_weight(p.bfloat16(), x)
    near(dw, p[-8:].bfloat16().double().T @ last.double(), product_tol(p[-8:].bfloat16().T, last.T) * 4)
    big = h.linear_grad_input(p.bfloat16(), w)
    near(big[-8:], p[-8:].bfloat16().double() @ w.double(), product_tol(p[-8:].bfloat16(), w.T))


def test_refusals(h):
    x, w = make(4, 64, "bf16", 1), make(8, 64, "bf16", 2)
    y = make(4, 8, "bf16", 3)
    r = h.layer_norm(x)
    q = h.act8_quantize(x)
    room = make(8, 100, "bf16", 9)
    other = torch.as_strided(room, (4, 64), (90, 1))
    bad = [
        lambda: h.linear(x.float(), w.float()),                            # operands of 32 bits
        lambda: h.linear(x, w.half()),                                     # two types
        lambda: h.linear(x, make(8, 63, "bf16", 4)),                       # another number of columns
        lambda: h.linear(x, w, torch.zeros(7, device=DEV)),                # a bias of another length
        lambda: h.linear(x, w, torch.zeros(8, device=DEV, dtype=torch.float64)),
        lambda: h.linear(x, w, residual=make(5, 8, "bf16", 5)),
        lambda: h.linear(x, w, out=make(4, 9, "bf16", 6)),
        lambda: h.linear(x.cpu(), w),
        lambda: h.linear(x[0], w),
        lambda: h.linear(x.T, w),
        lambda: h.linear(x, w, dtype=torch.float64),
        lambda: h.linear_grad_input(y, make(7, 64, "bf16", 7)),
        lambda: h.linear_grad_weight(y, make(5, 64, "bf16", 8)),
        lambda: h.linear_grad_weight(y, x, add=torch.zeros(8, 65, device=DEV)),
        lambda: h.layer_norm(x, torch.ones(64, device=DEV, dtype=torch.float16)),      # neither x's type nor 32 bits
        lambda: h.layer_norm(x, torch.ones(64, device=DEV), torch.ones(64, device=DEV, dtype=torch.bfloat16)),
        lambda: h.layer_norm(x, bias=torch.ones(64, device=DEV), rms=True),
        lambda: h.layer_norm(x, eps=-1.0),
        lambda: h.layer_norm(x, eps=math.nan),
        lambda: h.layer_norm(x, out=x.float()),
        lambda: h.layer_norm_grad(x, x.float(), None, r),
        lambda: h.layer_norm_grad(x[:3], x, None, r),
        lambda: h.layer_norm_grad(x[:3], q, None, r),
        lambda: h.layer_norm_grad(x[:3], x[:3], None, r),                  # statistics of other rows
        lambda: h.layer_norm_grad(x, x, None, r, add=x.float()),
        lambda: h.act_grad(x, x.float(), "gelu"),
        lambda: h.act_grad(x, x[:3], "gelu"),
        lambda: h.act_grad(x, binding.Act8Matrix(q.data[:100], 4, 64), "gelu"),
        lambda: h.act8_quantize(x, out=torch.zeros(100, dtype=torch.uint8, device=DEV)),
        lambda: h.act8_quantize(x, out=torch.zeros(1000, dtype=torch.uint8, device=DEV)[1:]),
        lambda: h.act8_quantize(x.double()),
        lambda: h.act8_restore(binding.Act8Matrix(q.data, 8, 64)),
        lambda: h.layer_norm(room[:4, :64], out=other),                    # one place, two strides
        lambda: h.linear(x, w, residual=room[:4, :8], out=torch.as_strided(room, (4, 8), (90, 1))),
        lambda: h.act_grad(room[:4, :64], x, "silu", out=other),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((TypeError, binding.ExcpError)):
            f()
            pytest.fail(f"call {i} was taken")
    for f in (lambda: h.linear(x, w, act="relu"), lambda: h.act_grad(x, x, "relu")):
        with pytest.raises(KeyError):
            f()
    with pytest.raises(ValueError):
        h.linear_kept(x, w, keep="fp8")
    torch.cuda.synchronize()


def test_products_on_several_streams_at_once(h):
    """Products of every kind (split over clusters, many runs of a 32-bit result, pairs of CTAs) and 4-bit ones, enqueued on four streams
    that nothing orders: each gives what it gives alone."""
    calls = []
    for i, (rows, k, n) in enumerate(((4, 4096, 2000), (64, 4096, 1024), (200, 2048, 1024), (2304, 256, 2304), (333, 1000, 515))):
        x, w, dy = make(rows, k, "bf16", i), make(n, k, "bf16", i + 10), make(rows, n, "bf16", i + 20)
        q = h.mx4_quantize(w, "e8m0_32")
        calls += [lambda x=x, w=w: h.linear(x, w, dtype=torch.float32), lambda dy=dy, w=w: h.linear_grad_input(dy, w), lambda dy=dy, x=x: h.linear_grad_weight(dy, x),
                  lambda x=x, q=q: h.mx4_linear(x, q)]
    alone = [f() for f in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    results = []
    for turn in range(6):
        for j, s in enumerate(streams):
            with torch.cuda.stream(s):
                results.append([calls[(i * 7 + 5 * j + turn) % len(calls)]() for i in range(len(calls))])
    torch.cuda.synchronize()
    for t, r in enumerate(results):
        for i, y in enumerate(r):
            assert torch.equal(y, alone[(i * 7 + 5 * (t % 4) + t // 4) % len(calls)])
    h.score_status()


@pytest.mark.parametrize("k", [700, 3000, 9000])
def test_long_sums_of_32_bits(h, k):
    """The tensor core cuts sums off: in runs of 768 columns (and no fewer than 48 additions of 16) a sum loses no more than 48 times half
    a unit of its running value on average, so the norm of the error stays below 2^-20 of the result's whatever the length."""
    for m, n in ((2304, 2400), (300, 200), (8, 2000), (257, 130)):
        dy, x = make(k, m, "bf16", 1), make(k, n, "bf16", 2)
        want = dy.double().T @ x.double()
        assert ((h.linear_grad_weight(dy, x).double() - want).norm() <= 2.0 ** -20 * want.norm())
        a, b = make(m, k, "bf16", 3), make(n, k, "bf16", 4)
        want = a.double() @ b.double().T
        assert ((h.linear(a, b, dtype=torch.float32).double() - want).norm() <= 2.0 ** -20 * want.norm())


@pytest.mark.parametrize("k", [3000, 9000])
def test_long_sums_of_what_is_kept(h, k):
    """Kept in 32 bits or 8 beside a result of 16: runs of 2048 columns, 128 additions of 16, lose 128 / 48 times what those above do.  A
    code is another where its value lies no further from a border than that: at most twice the error over a step (A / 127, and A is
    above the root of the block's mean square) of all codes.  A block's codes are others where its scale is: A that close to where the
    scale takes its next value, 2^-8 further."""
    off = 128 / 48 * 2.0 ** -20
    for m, n in ((2304, 2400), (300, 200), (8, 2000), (257, 130)):
        x, w = make(m, k, "fp16", 3), make(n, k, "fp16", 4, size=0.02)
        want = x.double() @ w.double().T
        y, kept = h.linear_kept(x, w, keep=torch.float32)
        assert ((kept.double() - want).norm() <= off * want.norm())
        again, packed = h.linear_kept(x, w, keep="act8")
        assert torch.equal(y, again)
        near(y, want, product_tol(x, w) * 1.01, "y")
        q, e = lo.act8_codes(want)
        ours = packed.data[:q.numel()].view(torch.int8).view(q.shape)
        assert int((ours.double() != q.double()).sum()) <= 2 * off * (127 + 256) * q.numel()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,n", [(1, 45), (40, 45), (300, 2397), (2500, 2397), (2500, 2400), (33, 8), (130, 4100)])
def test_results_leave_what_lies_beside_them(h, rows, n, dtype):
    """Rows that start on 16 bytes and end anywhere, in a part of a wider buffer, with rows behind the last."""
    x, w = make(rows, 64, "bf16", 1), make(n, 64, "bf16", 2)
    room = torch.full((rows + 3, (n + 31) // 8 * 8), 7.0, dtype=DT[dtype], device=DEV)
    h.linear(x, w, out=room[:rows, 8:8 + n])
    want = x.double() @ w.double().T
    near(room[:rows, 8:8 + n], want, product_tol(x, w) * 1.01, "y")
    assert bool((room[rows:] == 7).all() and (room[:, :8] == 7).all() and (room[:, 8 + n:] == 7).all())
