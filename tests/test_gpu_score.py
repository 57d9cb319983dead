"""The operators that score a restored checkpoint, through the C ABI, against their plain 64-bit definitions.

Tolerances (derived, not fitted):
  packed bytes and dequantised values   equal.
  product      the tensor core adds ceil(C / 64) partial sums to an fp32 accumulator (and up to 16 partial accumulators are
               added where the columns are split); each addition is off by at most 2^-22 of the sum of magnitudes (truncation
               included), the tensor scales and the bias add three roundings; then one rounding to the result's type.
  log probs    z, z - m and the final sums are roundings of 2^-24 of their magnitude, exp of a rounded argument is off by
               2^-23 |z - m|, and a sum in a chain of n additions by n 2^-24: at most vocab / 256 + 64 additions meet one value.
"""
import numpy as np
import pytest
import torch

from oracle import score_oracle as so
from paper_2406_11257_b200 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}
FMTS = ["e8m0_32", "e4m3_16"]


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(workspace_numel=4096, device=0)
    yield handle
    handle.score_status()
    handle.close()


def dense(x: torch.Tensor) -> np.ndarray:
    return x.detach().to(torch.float32).cpu().numpy()


def make(rows, cols, dtype, seed, slack=0, offset=0, spread=3.0):
    """Values over several binades in a buffer with `slack` more columns, starting `offset` elements in."""
    g = torch.Generator().manual_seed(seed)
    n = rows * (cols + slack) + offset
    x = torch.randn(n, generator=g) * torch.exp(torch.randn(n, generator=g) * spread * 0.3)
    buf = x.to(DT[dtype]).to(DEV)
    return buf[offset:].view(rows, cols + slack)[:, :cols]


def device_scale(v):
    return torch.tensor(float(v), dtype=torch.float32, device=DEV)


SHAPES = [(1, 1), (1, 4096), (3, 31), (8, 256), (9, 257), (127, 33), (128, 256), (129, 1000), (130, 17), (260, 700), (1, 65)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_and_back(h, rows, cols, dtype, fmt):
    for slack, offset in ((0, 0), (5, 0), (8, 8), (0, 1)):
        x = make(rows, cols, dtype, rows * 7 + cols, slack, offset)
        g = so.tensor_scale(dense(x)) if fmt == "e4m3_16" else None
        gd = None
        if fmt == "e4m3_16":
            gd = h.mx4_tensor_scale(x)
            assert float(gd) == g
        room = torch.full((binding.mx4_bytes(rows, cols, fmt),), 0xAB, dtype=torch.uint8, device=DEV)
        m = h.mx4_quantize(x, fmt, tensor_scale=gd, out=room)
        codes, scales = so.quantize(dense(x), fmt, g)
        assert np.array_equal(m.data.cpu().numpy(), so.pack(codes, scales, fmt))
        want = torch.from_numpy(so.values(codes, scales, fmt, g).astype(np.float32))
        for out in DT.values():
            y = h.mx4_dequantize(m, out)
            assert torch.equal(y.cpu(), want.to(out))
        wide = torch.full((rows, cols + 3), 7.0, device=DEV)
        h.mx4_dequantize(m, out=wide[:, :cols])
        assert torch.equal(wide[:, :cols].cpu(), want) and bool((wide[:, cols:] == 7).all())


@pytest.mark.parametrize("fmt", FMTS)
def test_quantize_extreme_values(h, fmt):
    rng = np.random.default_rng(5)
    x = (rng.normal(size=(40, 320)) * np.exp2(rng.integers(-140, 120, (40, 1)).astype(np.float64))).astype(np.float32)
    x[0] = 0.0
    x[1] = -0.0
    x[2, 3], x[3, 100], x[4, 319] = np.nan, np.inf, -np.inf
    x[5] = np.float32(3.4e38)
    x[6] = np.float32(2.0 ** -149)
    x[7, :] = np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], 40)       # every tie, both signs below
    x[8, :] = -x[7, :]
    xd = torch.from_numpy(x).to(DEV)
    for g in ([None] if fmt == "e8m0_32" else [None, 2.0 ** -20, 2.0 ** 100, 1.5 * 2.0 ** -110, 0.7]):
        m = h.mx4_quantize(xd, fmt, tensor_scale=None if g is None else device_scale(g))
        codes, scales = so.quantize(x, fmt, g)
        assert np.array_equal(m.data.cpu().numpy(), so.pack(codes, scales, fmt))
        y = h.mx4_dequantize(m)
        with np.errstate(over="ignore"):
            want = so.values(codes, scales, fmt, g).astype(np.float32)
        assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)


def test_tensor_scale_edges(h):
    for x, want in (([[0.0, -0.0]], 1.0), ([[np.nan, np.inf]], 1.0), ([[np.nan, -2688.0 * 0.75]], 0.75)):
        t = torch.tensor(x, dtype=torch.float32, device=DEV)
        assert float(h.mx4_tensor_scale(t)) == want
    assert float(h.mx4_tensor_scale(torch.empty((0, 5), device=DEV))) == 1.0
    assert float(h.mx4_tensor_scale(torch.empty((5, 0), device=DEV))) == 1.0
    big = torch.zeros((3000, 1111), device=DEV)
    big[2999, 1110] = -26.88
    for _ in range(3):
        assert float(h.mx4_tensor_scale(big)) == so.tensor_scale(np.array([26.88], np.float32))


def check_product(y, codes_a, scales_a, ga, codes_b, scales_b, gb, fmt, bias, dtype):
    a, b = so.values(codes_a, scales_a, fmt, ga), so.values(codes_b, scales_b, fmt, gb)
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    steps = -(-a.shape[1] // 64)
    tol = (steps + 16) * 2.0 ** -22 * mag + 3 * 2.0 ** -24 * np.abs(want)
    if bias is not None:
        want = want + bias
        tol += 2.0 ** -24 * np.abs(want)
    tol += HALF_ULP[dtype] * (np.abs(want) + tol) + 2.0 ** -25
    got = y.to(torch.float32).cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    worst = (np.abs(got - want)[ok] / tol[ok]).max(initial=0.0)
    assert worst <= 1.0, worst


PRODUCTS = [(1, 64, 128), (1, 4096, 300), (2, 1, 1), (7, 1000, 513), (8, 256, 128), (16, 2048, 1000), (33, 300, 129), (100, 512, 256),
            (128, 640, 384), (129, 257, 127), (200, 1024, 1000), (256, 256, 256), (300, 4096, 40), (513, 700, 777), (1000, 64, 8), (640, 3000, 512)]
# 256 x 256 tiles enough for the kernel of many rows: aligned rows of the result and others, ragged on every side, several tiles
# to a pair of SMs, both halves of a tile missing rows
PRODUCTS += [(1300, 513, 2048), (1100, 300, 2100), (2100, 260, 2608), (2049, 1500, 2305), (257, 64, 10001), (9000, 100, 260)]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,k,n", PRODUCTS)
def test_matmul(h, rows, k, n, fmt):
    xa, xb = make(rows, k, "fp32", 1 + rows), make(n, k, "fp32", 2 + n)
    ga = so.tensor_scale(dense(xa)) if fmt == "e4m3_16" else None
    gb = so.tensor_scale(dense(xb)) if fmt == "e4m3_16" else None
    qa, qb = so.quantize(dense(xa), fmt, ga), so.quantize(dense(xb), fmt, gb)
    ma = binding.Mx4Matrix(torch.from_numpy(so.pack(*qa, fmt)).to(DEV), rows, k, fmt, None if ga is None else device_scale(ga))
    mb = binding.Mx4Matrix(torch.from_numpy(so.pack(*qb, fmt)).to(DEV), n, k, fmt, None if gb is None else device_scale(gb))
    bias = torch.randn(n, generator=torch.Generator().manual_seed(4)).to(DEV)
    for dtype in sorted(DT):
        for with_bias in (False, True):
            y = h.mx4_matmul(ma, mb, bias=bias if with_bias else None, dtype=DT[dtype])
            check_product(y, *qa, ga, *qb, gb, fmt, dense(bias) if with_bias else None, dtype)
    # into a wider buffer, and twice: the same bits
    wide = torch.full((rows, n + 5), 7.0, device=DEV, dtype=torch.bfloat16)
    h.mx4_matmul(ma, mb, out=wide[:, :n])
    assert bool((wide[:, n:] == 7).all())
    assert torch.equal(wide[:, :n], h.mx4_matmul(ma, mb, dtype=torch.bfloat16))
    h.score_status()


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", ["fp16", "bf16", "fp32"])
@pytest.mark.parametrize("rows,k,n,slack", [(1, 4096, 512, 0), (5, 999, 130, 1), (16, 256, 3000, 8), (150, 1000, 260, 3), (300, 512, 520, 0),
                                             (1100, 600, 2064, 5), (1281, 257, 2047, 0), (17, 11000, 96, 2)])
def test_linear(h, rows, k, n, slack, dtype, fmt):
    x, w = make(rows, k, dtype, 11, slack), make(n, k, "fp32", 12)
    gx = device_scale(so.tensor_scale(dense(x)) * 1.37) if fmt == "e4m3_16" else None
    gw = h.mx4_tensor_scale(w) if fmt == "e4m3_16" else None
    m = h.mx4_quantize(w, fmt, tensor_scale=gw)
    bias = torch.randn(n, generator=torch.Generator().manual_seed(9)).to(DEV)
    gxf, gwf = (float(gx), float(gw)) if gx is not None else (None, None)
    qx, qw = so.quantize(dense(x), fmt, gxf), so.quantize(dense(w), fmt, gwf)
    for b in (None, bias):
        y = h.mx4_linear(x, m, bias=b, tensor_scale=gx)
        assert y.dtype == x.dtype
        check_product(y, *qx, gxf, *qw, gwf, fmt, None if b is None else dense(b), dtype)
    room = torch.empty(binding.mx4_bytes(rows, k, fmt) + 64, dtype=torch.uint8, device=DEV)
    assert torch.equal(h.mx4_linear(x, m, bias=bias, tensor_scale=gx, x_packed=room), y)
    h.score_status()


@pytest.mark.parametrize("n", [33000, 32992])
def test_product_past_32_bit_offsets(h, n):
    # 2.2e9 results: the last rows lie past element 2^31 and byte 2^32 (rows that start on 32 bytes, and others)
    rows, k, fmt = 66000, 64, "e8m0_32"
    x, w = make(rows, k, "bf16", 51), make(n, k, "fp32", 52)
    y = h.mx4_linear(x, h.mx4_quantize(w, fmt))
    qw = so.quantize(dense(w), fmt)
    for part in (slice(0, 2), slice(rows - 3, rows)):
        check_product(y[part], *so.quantize(dense(x[part]), fmt), None, *qw, None, fmt, None, "bf16")
    del y


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows", [3, 200, 9000])
def test_product_of_rows_with_nan_stays_in_its_rows(h, rows, fmt):
    k, n = 320, 300
    x, w = make(rows, k, "fp32", 21), make(n, k, "fp32", 22)
    x, w = x.clone(), w.clone()
    x[1, 77], w[200, 5], w[299, 319] = float("nan"), float("inf"), float("nan")
    mx, mw = h.mx4_quantize(x, fmt), h.mx4_quantize(w, fmt)
    qx, qw = so.quantize(dense(x), fmt, 1), so.quantize(dense(w), fmt, 1)
    check_product(h.mx4_matmul(mx, mw, dtype=torch.float32), *qx, 1, *qw, 1, fmt, None, "fp32")


def test_products_of_nothing(h):
    for fmt in FMTS:
        w = h.mx4_quantize(torch.ones((300, 0), device=DEV), fmt)
        x = h.mx4_quantize(torch.ones((5, 0), device=DEV), fmt)
        bias = torch.arange(300, dtype=torch.float32, device=DEV)
        assert torch.equal(h.mx4_matmul(x, w, bias=bias, dtype=torch.float32), bias.expand(5, 300))
        assert not h.mx4_matmul(x, w, dtype=torch.float16).any()
        assert torch.equal(h.mx4_linear(torch.ones((5, 0), device=DEV), w, bias=bias), bias.expand(5, 300))
        assert torch.equal(h.mx4_linear(torch.ones((500, 0), device=DEV), w, bias=bias), bias.expand(500, 300))
        w = h.mx4_quantize(torch.ones((30, 64), device=DEV), fmt)
        x = torch.ones((0, 64), device=DEV)
        assert h.mx4_linear(x, w).shape == (0, 30)
        none = h.mx4_quantize(x, fmt)
        assert h.mx4_matmul(w, none).shape == (30, 0)


def test_product_on_another_stream_and_in_a_graph(h):
    x, w = make(4, 512, "bf16", 31), make(700, 512, "bf16", 32)
    m = h.mx4_quantize(w, "e8m0_32")
    want = h.mx4_linear(x, m)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = h.mx4_linear(x, m)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    tokens = torch.tensor([1, 2, 3, 4], device=DEV)
    h.token_logprobs(want, tokens, top=3)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = h.mx4_linear(x, m)
        r = h.token_logprobs(y, tokens, top=3)
    for _ in range(3):
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    assert torch.equal(r.top_index, h.token_logprobs(want, tokens, top=3).top_index)


def test_a_wait_that_runs_out_is_reported(h):
    # a token quantised in the product, some packed, split columns, the kernel of many rows
    for rows, n in ((1, 700), (40, 700), (300, 700), (1100, 2100)):
        x, w = make(rows, 2048, "bf16", 41), make(n, 2048, "bf16", 42)
        m = h.mx4_quantize(w, "e8m0_32")
        want = h.mx4_linear(x, m)
        h.set_wait_limit(0)
        try:
            h.mx4_linear(x, m)
            with pytest.raises(binding.ExcpError) as e:
                h.score_status()
            assert e.value.status == -7
        finally:
            h.set_wait_limit(2_000_000_000)
        assert torch.equal(h.mx4_linear(x, m), want)
        h.score_status()


# ---- log probabilities ---------------------------------------------------------------

def make_logits(rows, vocab, dtype, seed, slack=0, offset=0, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    n = rows * (vocab + slack) + offset
    x = torch.randn(n, generator=g) * 4
    if kind == "ties":
        x = torch.round(x)
    elif kind == "equal":
        x = torch.full((n,), 2.5)
    elif kind == "masked":
        x[torch.rand(n, generator=g) < 0.9] = -float("inf")
    elif kind == "lowest":
        x[torch.rand(n, generator=g) < 0.5] = torch.finfo(DT[dtype]).min
    elif kind == "peaked":
        x[::max(1, vocab // 3)] += 60
    elif kind == "rising":
        x = torch.arange(n, dtype=torch.float32) * 0.01
    buf = x.to(DT[dtype]).to(DEV)
    return buf[offset:].view(rows, vocab + slack)[:, :vocab]


def close(got, want, tol):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.isinf(got), np.isinf(want)) and np.array_equal(got[np.isinf(got)], want[np.isinf(want)])
    ok = np.isfinite(want)
    worst = (np.abs(got[ok] - want[ok]) / np.broadcast_to(tol, want.shape)[ok]).max(initial=0.0)
    assert worst <= 1.0, worst


def check_logprobs(h, x, tokens, scale, top, grad=True, seed=1):
    rows, vocab = x.shape
    td = torch.from_numpy(np.asarray(tokens, np.int64)).to(DEV)
    r = h.token_logprobs(x, td, top=top, scale=scale)
    xn = dense(x)
    scale32 = float(np.float32(scale))
    want = so.logprobs(xn, tokens, scale32, top)
    # magnitudes that are rounded: the maximum, and the distances to it, which weigh in by their probability
    reach = np.abs(xn.astype(np.float64).max(1, initial=-np.inf) * scale32)
    reach = np.where(np.isfinite(reach), reach, 0.0) + 1 + 2 * np.log(vocab)
    chain = vocab / 256 + 64
    tol = 2.0 ** -22 * reach + chain * 2.0 ** -24
    close(r.logprob.cpu().numpy(), want["logprob"], tol + 2.0 ** -23 * np.where(np.isfinite(want["logprob"]), np.abs(want["logprob"]), 0) + 1e-30)
    spread = 1 + np.log(max(vocab, 2))                # d p log p adds up to at most the entropy's size times the error of log p
    close(r.entropy.cpu().numpy(), want["entropy"], 2 * spread * tol + 1e-30)
    if top:
        assert np.array_equal(r.top_index.cpu().numpy(), want["top_index"])
        close(r.top_logprob.cpu().numpy(), want["top_logprob"], tol[:, None] + 2.0 ** -23 * np.where(np.isfinite(want["top_logprob"]), np.abs(want["top_logprob"]), 0) + 1e-30)
    if grad:
        rng = np.random.default_rng(seed)
        gl, gh = rng.normal(size=rows).astype(np.float32), rng.normal(size=rows).astype(np.float32)
        dtype = {v: k for k, v in DT.items()}[x.dtype]
        wg = so.logprobs_grad(xn, tokens, scale32, gl, gh)
        lp = np.where(want["p"] == 0, 0, np.abs(want["log_p"])) + np.abs(want["entropy"])[:, None]
        size = np.abs(gl)[:, None] * want["p"] + np.abs(gh)[:, None] * want["p"] * (lp + 1)
        one = np.zeros_like(wg)
        t = np.asarray(tokens)
        one[np.arange(rows)[t >= 0], t[t >= 0]] = np.abs(gl)[t >= 0]
        tg = scale32 * (size * (4 * spread * tol[:, None] + 2.0 ** -20) + one * 2.0 ** -22)
        tg = tg + HALF_ULP[dtype] * (np.abs(wg) + tg) + (2.0 ** -25 if dtype == "fp16" else 1e-37)
        gld, ghd = torch.from_numpy(gl).to(DEV), torch.from_numpy(gh).to(DEV)
        got = h.token_logprobs_grad(x, td, r, gld, ghd)
        close(dense(got), wg, tg)
        assert torch.equal(h.token_logprobs_grad(x, td, r, gld, None), h.token_logprobs_grad(x, td, r, gld, torch.zeros_like(ghd)))
        wide = torch.full((rows, vocab + 3), 7.0, dtype=x.dtype, device=DEV)
        h.token_logprobs_grad(x, td, r, gld, ghd, out=wide[:, :vocab])
        assert torch.equal(wide[:, :vocab], got) and bool((wide[:, vocab:] == 7).all())
        own = x.clone(memory_format=torch.preserve_format) if x.is_contiguous() else x.clone()
        h.token_logprobs_grad(own, td, r, gld, ghd, out=own)
        assert torch.equal(own, got)


LOGITS = [(1, 1, 1), (1, 2, 2), (5, 7, 7), (3, 31, 5), (2, 256, 20), (4, 1000, 64), (7, 4097, 20), (1, 50304, 20), (2, 131072, 3), (300, 513, 4),
          (1, 250001, 5)]


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("rows,vocab,top", LOGITS)
def test_logprobs_sizes(h, rows, vocab, top, dtype):
    rng = np.random.default_rng(rows + vocab)
    tokens = rng.integers(0, vocab, rows)
    for slack, offset, scale in ((0, 0, 1.0), (3, 1, 0.6), (8, 8, 1.7)):
        if rows * vocab > 100000 and slack == 8:
            continue
        check_logprobs(h, make_logits(rows, vocab, dtype, vocab + slack, slack, offset), tokens, scale, top, grad=rows * vocab <= 300000)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("kind", ["ties", "equal", "masked", "lowest", "peaked", "rising"])
def test_logprobs_values(h, kind, dtype):
    for rows, vocab, top in ((3, 40, 9), (4, 5000, 33), (1, 30000, 20)):
        x = make_logits(rows, vocab, dtype, 5, kind=kind)
        tokens = np.arange(rows) * 3 % vocab
        tokens[0] = -1 if rows > 1 else 0
        check_logprobs(h, x, tokens, 1.0, top, grad=kind != "lowest")


@pytest.mark.parametrize("rows", [6, 400])
def test_logprobs_rows_that_hold_nothing_or_nan(h, rows):
    for vocab in (5, 900, 20000 if rows == 6 else 901):
        x = make_logits(rows, vocab, "fp32", 3).clone()
        x[0] = -float("inf")
        x[1, vocab // 2] = float("nan")
        x[2, vocab - 1] = float("inf")
        x[3] = -float("inf")
        x[3, 2] = 1.5                                  # a single word left: probability one
        tokens = np.arange(rows) % vocab
        tokens[3] = 2
        tokens[5] = -7
        td = torch.from_numpy(tokens).to(DEV)
        r = h.token_logprobs(x, td, top=4)
        want = so.logprobs(dense(x)[:6], tokens[:6], 1.0, 4)
        lp = r.logprob.cpu().numpy()
        assert lp[0] == -np.inf and np.isnan(lp[1]) and np.isnan(lp[2]) and lp[3] == 0 and lp[5] == 0
        e = r.entropy.cpu().numpy()
        assert e[0] == 0 and np.isnan(e[1]) and np.isnan(e[2]) and e[3] == 0 and np.isfinite(e[4:]).all()
        assert np.array_equal(r.top_index.cpu().numpy()[:6], want["top_index"])
        assert np.array_equal(r.top_logprob.cpu().numpy()[0], [-np.inf] * 4)
        g = h.token_logprobs_grad(x, td, r, torch.ones(rows, device=DEV), torch.ones(rows, device=DEV))
        assert not g[0].any() and torch.isnan(g[1]).all() and torch.isnan(g[2]).all() and not g[3].any()
        assert torch.isfinite(g[4:]).all()
        # a token past the vocabulary: NaN, nothing read
        td[4] = vocab + 5
        lp2 = h.token_logprobs(x, td).logprob
        assert torch.isnan(lp2[4]) and torch.equal(lp2[5:], r.logprob[5:])


def test_logprobs_are_the_same_twice_and_ignore_neighbours(h):
    x = make_logits(64, 3001, "bf16", 8)
    tokens = torch.arange(64, device=DEV)
    a, b = h.token_logprobs(x, tokens, top=7), h.token_logprobs(x, tokens, top=7)
    one = h.token_logprobs(x[5:6], tokens[5:6], top=7)
    for k in ("logprob", "entropy", "top_logprob", "top_index"):
        assert torch.equal(getattr(a, k), getattr(b, k))
    assert torch.equal(one.top_index[0], a.top_index[5])


def test_logprobs_past_32_bit_offsets(h):
    # 2.2e9 half-precision logits: the last rows lie past element 2^31 and byte 2^32
    rows, vocab = 17000, 131000
    x = torch.zeros((rows, vocab), dtype=torch.float16, device=DEV)
    x[-1] = make_logits(1, vocab, "fp16", 4)[0]
    x[-2, 77] = 3.0
    tokens = torch.full((rows,), 77, device=DEV)
    r = h.token_logprobs(x, tokens, top=2)
    want = so.logprobs(dense(x[-2:]), [77, 77], 1.0, 2)
    close(r.logprob[-2:].cpu().numpy(), want["logprob"], 1e-4)
    assert np.array_equal(r.top_index[-2:].cpu().numpy(), want["top_index"])
    g = h.token_logprobs_grad(x, tokens, r, torch.ones(rows, device=DEV), out=x)
    wg = so.logprobs_grad(np.zeros((1, vocab)), [77], 1.0, [1.0], [0.0])
    close(dense(g[100:101]), wg, np.abs(wg) * 2.0 ** -10 + 2.0 ** -24)
    del x, g


# ---- refusals -----------------------------------------------------------------------------

def test_refusals_of_the_binding(h):
    x = torch.ones((4, 64), device=DEV)
    w = h.mx4_quantize(x, "e8m0_32")
    v = h.mx4_quantize(x, "e4m3_16")
    with pytest.raises(KeyError):
        h.mx4_quantize(x, "e2m3")
    for bad in (x.double(), x.cpu(), x[0], x.t()):
        with pytest.raises(TypeError):
            h.mx4_quantize(bad, "e8m0_32")
    with pytest.raises(TypeError):
        h.mx4_quantize(x, "e8m0_32", out=torch.empty(10, dtype=torch.uint8, device=DEV))
    with pytest.raises(TypeError):
        h.mx4_quantize(x, "e4m3_16", tensor_scale=torch.ones(2, device=DEV))
    with pytest.raises(TypeError):
        h.mx4_matmul(w, v)
    with pytest.raises(TypeError):
        h.mx4_linear(x[:, :32], w)
    with pytest.raises(TypeError):
        h.mx4_linear(x, w, bias=torch.ones(3, device=DEV))
    with pytest.raises(TypeError):
        h.mx4_linear(x, w, out=torch.ones((4, 5), device=DEV))
    tokens = torch.zeros(4, dtype=torch.int64, device=DEV)
    for bad in (tokens.int(), tokens[:3], tokens.cpu()):
        with pytest.raises(TypeError):
            h.token_logprobs(x, bad)
    r = h.token_logprobs(x, tokens)
    with pytest.raises(TypeError):
        h.token_logprobs_grad(x, tokens, r, torch.ones(3, device=DEV))
    with pytest.raises(TypeError):
        h.token_logprobs_grad(x, tokens, r, None, out=x.half())
    for kw in ({"top": 65}, {"top": -1}, {"scale": 0.0}, {"scale": -1.0}, {"scale": float("inf")}, {"scale": float("nan")}):
        with pytest.raises(binding.ExcpError) as e:
            h.token_logprobs(x, tokens, **kw)
        assert e.value.status == -1


def test_refusals_of_the_c_abi(h):
    lib, H = h.lib, h._h
    x = torch.ones((4, 64), device=DEV)
    q = torch.empty(binding.mx4_bytes(4, 64, "e8m0_32") + 16, dtype=torch.uint8, device=DEV)
    f = torch.ones(64, device=DEV)
    t = torch.zeros(4, dtype=torch.int64, device=DEV)
    p, qp, fp, tp = x.data_ptr(), q.data_ptr(), f.data_ptr(), t.data_ptr()
    bad = -1
    assert lib.excp_mx4_quantize(None, p, 0, 4, 64, 64, 1, 0, qp, 0) == bad
    assert lib.excp_mx4_quantize(H, 0, 0, 4, 64, 64, 1, 0, qp, 0) == bad
    assert lib.excp_mx4_quantize(H, p, 3, 4, 64, 64, 1, 0, qp, 0) == bad           # type
    assert lib.excp_mx4_quantize(H, p, 0, 4, 64, 63, 1, 0, qp, 0) == bad           # overlapping rows
    assert lib.excp_mx4_quantize(H, p + 2, 0, 4, 64, 64, 1, 0, qp, 0) == bad       # element alignment
    assert lib.excp_mx4_quantize(H, p, 0, 4, 64, 64, 0, 0, qp, 0) == bad           # format
    assert lib.excp_mx4_quantize(H, p, 0, 4, 64, 64, 1, 0, qp + 8, 0) == bad       # packed alignment
    assert lib.excp_mx4_quantize(H, p, 0, 4, 64, 64, 1, 0, 0, 0) == bad
    assert lib.excp_mx4_quantize(H, p, 0, 1 << 31, 64, 64, 1, 0, qp, 0) == bad     # size
    assert lib.excp_mx4_tensor_scale(H, p, 0, 4, 64, 64, 0, 0) == bad
    assert lib.excp_mx4_dequantize(H, qp, 4, 64, 1, 0, 0, 0, 64, 0) == bad
    assert lib.excp_mx4_matmul(H, qp, 4, 0, qp, 4, 0, 64, 1, 0, 0, 0, 4, 0) == bad
    assert lib.excp_mx4_matmul(H, qp, 4, 0, qp, 4, 0, 64, 1, 0, p, 0, 3, 0) == bad
    assert lib.excp_mx4_matmul(H, qp, 4, fp + 1, qp, 4, 0, 64, 2, 0, p, 0, 4, 0) == bad
    assert lib.excp_mx4_linear(H, p, 0, 17, 64, 0, qp, 4, 0, 64, 1, 0, p, 0, 4, 0, 0) == bad  # no room for the packed x
    assert lib.excp_token_logprobs(H, p, 0, 4, 64, 64, 0, 1.0, 0, fp, fp, 0, 0, 0, 0) == bad
    assert lib.excp_token_logprobs(H, p, 0, 4, 64, 64, tp, 1.0, 0, 0, fp, 0, 0, 0, 0) == bad
    assert lib.excp_token_logprobs(H, p, 0, 4, 64, 64, tp, 1.0, 2, fp, fp, 0, 0, 0, 0) == bad
    assert lib.excp_token_logprobs(H, p, 0, 4, 8, 64, tp, 1.0, 9, fp, fp, 0, fp, tp, 0) == bad  # more alternatives than words
    assert lib.excp_token_logprobs(H, p, 0, 4, 64, 64, tp, 1.0, 0, fp, fp, fp + 4, 0, 0, 0) == bad
    assert lib.excp_token_logprobs_grad(H, p, 0, 4, 64, 64, tp, 1.0, 0, 0, 0, p, 64, 0) == bad
    assert lib.excp_token_logprobs_grad(H, p, 0, 4, 32, 64, tp, 1.0, fp, 0, 0, p, 32, 0) == bad  # in place with another stride
    assert lib.excp_score_status(None, 0) == bad
    assert lib.excp_token_logprobs(H, 0, 0, 0, 64, 64, 0, 1.0, 0, 0, 0, 0, 0, 0, 0) == 0         # no rows: nothing to do


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "masked", "rising"])
def test_logprobs_of_many_rows(h, kind, dtype):
    # more rows than SMs: the persistent blocks, several rows each, short and odd rows among them
    for rows, vocab, top in ((1300, 37, 5), (700, 1030, 64), (1100, 129, 20)):
        for slack, offset in ((0, 0), (1, 1)):
            x = make_logits(rows, vocab, dtype, 77 + vocab, slack, offset, kind)
            check_logprobs(h, x, np.arange(rows) * 7 % vocab, 0.9, top, grad=False)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("vocab", [1, 5, 16, 33, 1001, 20011])
def test_gradient_of_rows_at_every_offset(h, vocab, dtype):
    """A value's gradient does not depend on where its row starts: equal bits, and nothing written beside the rows."""
    rows, gen = 5, torch.Generator(device=DEV).manual_seed(vocab)
    x = (torch.randn((rows, vocab), device=DEV, generator=gen) * 3).to(DT[dtype])
    tokens = torch.randint(0, vocab, (rows,), device=DEV, generator=gen)
    gl, gh = torch.randn(rows, device=DEV, generator=gen), torch.randn(rows, device=DEV, generator=gen)
    r = h.token_logprobs(x, tokens, scale=0.7)
    want = h.token_logprobs_grad(x, tokens, r, gl, gh)
    wg = so.logprobs_grad(dense(x), tokens.cpu().numpy(), 0.7, gl.cpu().numpy(), gh.cpu().numpy())
    ulp = {torch.float32: 2.0 ** -20, torch.float16: 2.0 ** -10, torch.bfloat16: 2.0 ** -7}[DT[dtype]]
    size = float((gl.abs() + gh.abs() * (np.log(vocab) + 20)).max())
    close(dense(want), wg, np.abs(wg) * ulp + size * 2.0 ** -18)
    per16 = 16 // x.element_size()
    for start in range(per16):
        for out_start in (0, 1, per16 - 1):
            for slack, out_slack in ((0, 0), (1, 0), (3, per16)):
                xs = torch.full((start + rows * (vocab + slack) + per16,), float("nan"), dtype=x.dtype, device=DEV)
                ys = torch.full((out_start + rows * (vocab + out_slack) + per16,), 7.0, dtype=x.dtype, device=DEV)
                xv = xs.as_strided((rows, vocab), (vocab + slack, 1), start)
                yv = ys.as_strided((rows, vocab), (vocab + out_slack, 1), out_start)
                xv.copy_(x)
                h.token_logprobs_grad(xv, tokens, r, gl, gh, out=yv)
                assert torch.equal(yv, want)
                yv.fill_(7.0)
                assert bool((ys == 7).all())


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", [1, 7, 40, 511, 513, 1600])
def test_tensor_scale_of_rows_at_every_offset(h, cols, dtype):
    """The largest value is found wherever it lies, and what lies beside the rows is not looked at."""
    per32 = 32 // torch.empty((), dtype=DT[dtype]).element_size()
    for start in range(per32):
        for at in sorted({0, 1 % cols, min(per32 - start, cols - 1), cols // 2, cols - 1}):
            xs = torch.full((start + 3 * (cols + 1) + per32,), 30000.0, dtype=DT[dtype], device=DEV)
            x = xs.as_strided((3, cols), (cols + 1, 1), start)
            x.fill_(0.5)
            x[2, at] = -21.0
            assert float(h.mx4_tensor_scale(x)) == so.tensor_scale(dense(x))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("cols", [1, 7, 33, 255, 256, 257, 530])
def test_quantize_and_back_at_every_offset(h, cols, dtype, fmt):
    """Codes and values do not depend on where a row starts, and nothing beside the rows is read into them or written."""
    rows, gen = 37, torch.Generator(device=DEV).manual_seed(cols)
    x = (torch.randn((rows, cols), device=DEV, generator=gen) * 3).to(DT[dtype])
    g = h.mx4_tensor_scale(x) if fmt == "e4m3_16" else None
    m = h.mx4_quantize(x, fmt, tensor_scale=g)
    codes, scales = so.quantize(dense(x), fmt, None if g is None else float(g))
    assert np.array_equal(m.data.cpu().numpy(), so.pack(codes, scales, fmt))
    back = h.mx4_dequantize(m, DT[dtype])
    want = torch.from_numpy(so.values(codes, scales, fmt, None if g is None else float(g)).astype(np.float32))
    assert torch.equal(back.cpu(), want.to(DT[dtype]))
    per16 = 16 // x.element_size()
    for start in range(per16):
        for slack in (0, 1, per16 - 1, per16):
            xs = torch.full((start + rows * (cols + slack) + per16,), float("nan"), dtype=x.dtype, device=DEV)
            xv = xs.as_strided((rows, cols), (cols + slack, 1), start)
            xv.copy_(x)
            assert torch.equal(h.mx4_quantize(xv, fmt, tensor_scale=g).data, m.data)
            xs.fill_(77.0)
            h.mx4_dequantize(m, out=xv)
            assert torch.equal(xv, back)
            xv.fill_(77.0)
            assert bool((xs == 77).all())


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "masked", "lowest", "peaked"])
def test_logprobs_of_short_rows_by_the_thousand(h, kind, dtype):
    """A warp to a row: below, at and above its words; as many alternatives as lanes; one more goes another way."""
    for rows, vocab, top in ((1500, 3, 3), (1500, 39, 5), (1500, 64, 33), (1300, 301, 32)) + (((1200, 4096, 32),) if kind == "ties" else ()):
        x = make_logits(rows, vocab, dtype, 177 + vocab, vocab % 2, vocab % 3, kind)
        check_logprobs(h, x, np.arange(rows) * 7 % vocab, 0.9, top, grad=vocab < 40)


def test_short_rows_by_the_thousand_that_hold_nothing_or_nan(h):
    rows, vocab = 1500, 700
    x = make_logits(rows, vocab, "bf16", 9).clone()
    x[0] = -float("inf")
    x[1, 5] = float("nan")
    x[2, 699] = float("inf")
    tokens = np.arange(rows) % vocab
    tokens[3] = -1
    r = h.token_logprobs(x, torch.from_numpy(tokens).to(DEV), top=9)
    want = so.logprobs(dense(x)[:8], tokens[:8], 1.0, 9)
    lp = r.logprob.cpu().numpy()
    assert lp[0] == -np.inf and np.isnan(lp[1]) and np.isnan(lp[2]) and lp[3] == 0 and np.isfinite(lp[4:]).all()
    assert np.array_equal(r.top_index.cpu().numpy()[:8], want["top_index"])


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "masked", "lowest", "peaked", "rising"])
def test_logprobs_of_few_long_rows(h, kind, dtype):
    """Rows that several blocks share."""
    for rows, vocab, top in ((1, 20480, 64), (3, 33001, 5)) + (((20, 41003, 20), (40, 90001, 4)) if kind == "normal" else ()):
        x = make_logits(rows, vocab, dtype, 277 + vocab, vocab % 2, vocab % 3, kind)
        check_logprobs(h, x, np.arange(rows) * 7777 % vocab, 0.9, top, grad=rows < 3)
