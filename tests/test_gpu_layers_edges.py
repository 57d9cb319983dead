"""The layers at the edges of what their definitions allow, against their plain 64-bit definitions.  U = 2^-24 as in test_gpu_layers.py."""
import math

import pytest
import torch

from oracle import layers_oracle as lo
from paper_2406_11257_b200 import binding
from test_gpu_layers import DEV, DT, U, make, near, vector

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(workspace_numel=4096, device=0)
    yield handle
    handle.score_status()
    handle.close()


# ---- norms -------------------------------------------------------------------------
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cols,slack", [(1000, 0), (1000, 3), (4096, 0), (300, 1), (8, 0), (17000, 0), (17001, 0)])
@pytest.mark.parametrize("rows", [5, 2000])
def test_gradient_of_equal_values_is_finite(h, rows, cols, slack, dtype, weighted):
    """Rows of one large value (which 8 bits hold exactly) with a small eps: xh is 0 in every column, so dx = rstd (g - mean g).  The mean
    times rstd, 2^91 * 2^49, is past fp32's numbers, and may not be formed where there is no column.  The mean of g is off by u of the mean
    magnitude for each of at most cols / 8 / 32 + 40 additions in a row and a product; four roundings are left."""
    x = torch.full((rows, cols + slack), 127 * 2.0 ** 84, device=DEV).to(DT[dtype])[:, :cols]
    dy = make(rows, cols, dtype, 3, slack)
    w = vector(cols, dtype, 4, 0.2, 1.0) if weighted else None
    r = h.layer_norm(x, w, eps=1e-30, keep=True)
    want, _, db = lo.norm_grad(dy, x, w, r.row_stats[:, 0], r.row_stats[:, 1])
    gg = dy.double().abs() * (1.0 if w is None else w.double().abs())
    tol = r.row_stats[:, 1:].double() * U * (4 * gg + (cols / 256 + 44) * gg.mean(1, keepdim=True))
    for v in (x, r.kept):
        for vectors in (True, False):
            g = h.layer_norm_grad(dy, v, w, r, vectors=vectors)
            near(g.dx, want, tol, "dx")
        g = h.layer_norm_grad(dy, v, w, r)
        assert not g.dweight.any()
        near(g.dbias, db, dy.double().abs().sum(0) * (rows + 40) * U, "dbias")


@pytest.mark.parametrize("rows", [3000, 200])
@pytest.mark.parametrize("cols", [256, 320, 4096, 16384, 20000])
def test_rstd_is_rounded_once(h, rows, cols):
    """Whole numbers, whose squares add up exactly (at most 64 * 20000 < 2^24): what is left is the rounding of the sum over cols (u, which the root
    halves) and of 1 / root (u).  With a power of two for cols the division is exact too."""
    g = torch.Generator().manual_seed(cols + rows)
    x = torch.randint(-8, 9, (rows, cols), generator=g).float().to(DEV)
    r = h.layer_norm(x, eps=0.0, rms=True)
    want = 1.0 / torch.sqrt((x.double() ** 2).mean(1))
    units = 1.0 if cols & (cols - 1) == 0 else 1.5
    assert bool(((r.row_stats[:, 1].double() - want).abs() <= units * U * 1.0001 * want).all())


# ---- products ------------------------------------------------------------------------
@pytest.mark.parametrize("rows,k,n", [(4, 512, 300), (64, 4096, 1024), (1, 11008, 4096)])
def test_waits_that_some_ctas_give_up(rows, k, n):
    """Limits at which some CTAs of a cluster give up and others do not: the product says so or is right, and the next one is right."""
    other = binding.Handle(workspace_numel=4096, device=0)
    x, w = make(rows, k, "bf16", 1), make(n, k, "bf16", 2)
    want = other.linear(x, w)
    other.score_status()
    for limit in (1, 500, 2000, 5000, 10000):
        for _ in range(3):
            other.set_wait_limit(limit)
            got = other.linear(x, w)
            try:
                other.score_status()
            except binding.ExcpError as e:
                assert e.status == -7
            else:
                assert torch.equal(got, want)
            other.set_wait_limit(2_000_000_000)
            assert torch.equal(other.linear(x, w), want)
            other.score_status()
    other.close()


def big(rows, cols, seed, dtype=torch.bfloat16, size=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(rows, cols, generator=g, device=DEV) * size).to(dtype)


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


def test_sums_of_any_length(h):
    """32-bit results of more columns than tensor memory has room for in runs of 768 (few rows on one side, too many tiles to be split; or so
    long that even a part of the columns is): as exact as short ones, 2^-20 of the result's norm."""
    for k, n, m in ((65536, 19100, 16), (131072, 19000, 8), (262144, 100, 3)):
        dy, x = big(k, n, 1), big(k, m, 2)
        want = torch.zeros(n, m, dtype=torch.float64, device=DEV)
        for i in range(0, k, 8192):
            want += dy[i:i + 8192].double().T @ x[i:i + 8192].double()
        assert off(h.linear_grad_weight(dy, x), want) <= 2.0 ** -20, (k, n, m)
        del dy, x
    for rows, k, n in ((64, 50304, 11008), (1, 50304, 4096)):
        x, w = big(rows, k, 3), big(n, k, 4)
        want = torch.cat([x.double() @ w[i:i + 2048].double().T for i in range(0, n, 2048)], 1)
        assert off(h.linear(x, w, dtype=torch.float32), want) <= 2.0 ** -20, (rows, k, n)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,k,n", [(1, 11008, 4096), (40, 8200, 48), (64, 4096, 4096), (300, 3000, 700)])
def test_what_is_kept_does_not_change_results(h, rows, k, n, dtype):
    """The same y whatever is kept beside it, and what is kept in 32 bits as exact as a result of 32 bits (2^-20 of the norm)."""
    x, w = big(rows, k, 1, DT[dtype]), big(n, k, 2, DT[dtype], 0.02)
    bias = vector(n, dtype, 3)
    y = h.linear(x, w, bias, act="gelu")
    for keep in ("act8", torch.float32, torch.float16, torch.bfloat16):
        again, kept = h.linear_kept(x, w, bias, act="gelu", keep=keep)
        assert torch.equal(again, y), keep
        if keep == torch.float32:
            want = x.double() @ w.double().T + bias.double()
            assert off(kept, want) <= 2.0 ** -20
            q, s = lo.act8_codes(kept)
            packed = h.linear_kept(x, w, bias, act="gelu")[1].data
            assert torch.equal(packed[:q.numel() + 2 * s.numel()], lo.act8_pack(q, s))


@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,k,n", [(2304, 3000, 2400), (2304, 9000, 2400)])
def test_kept_in_32_bits_is_as_exact_as_a_result(h, rows, k, n, dtype, act):
    x, w = big(rows, k, 1, DT[dtype]), big(n, k, 2, DT[dtype], 0.02)
    _, kept = h.linear_kept(x, w, act=act, keep=torch.float32)
    assert off(kept, x.double() @ w.double().T) <= 2.0 ** -20


@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_results_of_many_rows_beside_8_bits(h, dtype, act):
    """The forward pass that keeps its activations gives what the one that does not gives."""
    x, w = big(2304, 9000, 1, DT[dtype]), big(2400, 9000, 2, DT[dtype], 0.02)
    y = h.linear(x, w, act=act)
    for keep in ("act8", torch.float16, torch.bfloat16):
        assert torch.equal(h.linear_kept(x, w, act=act, keep=keep)[0], y)


@pytest.mark.parametrize("k", [9000, 50304])
@pytest.mark.parametrize("rows,n", [(2304, 2304), (200, 300), (1, 2304)])
def test_long_sums_of_one_sign_in_16_bits(h, rows, n, k):
    """Terms of one sign: an addition of 16 columns cuts off at most 2^-22 of the running sum, which is half of the last one on average, so a run of
    2048 columns loses at most 64 * 2^-22 of it (and the sum of the runs no more than their share of 2^-24 each); the rounding to fp16 falls on both sides, and of rows * n of them a mean of 5 deviations
    (2^-11 / sqrt(12) each at most) is left."""
    g = torch.Generator(device=DEV).manual_seed(7)
    x, w = ((torch.rand(r, k, generator=g, device=DEV) + 0.5).mul_(s).half() for r, s in ((rows, 1.0), (n, 400.0 / k)))
    y, want = h.linear(x, w).double(), x.double() @ w.double().T
    assert abs(((y - want) / want).mean().item()) <= 64 * 2.0 ** -22 + 25 * U + 5 * 2.0 ** -11 / math.sqrt(12 * rows * n)


# ---- results that the caller gives ------------------------------------------------------
def test_results_move_their_version(h):
    """What a call writes into a tensor of the caller's is a change that autograd sees: saved for a backward pass, it is refused there."""
    x, w, dy = make(4, 64, "bf16", 1), make(8, 64, "bf16", 2), make(4, 8, "bf16", 3)
    n, q = h.layer_norm(x), h.act8_quantize(x)
    z = h.mx4_quantize(w, "e8m0_32")
    logits = make(4, 100, "fp32", 4)
    r = h.token_logprobs(logits, torch.zeros(4, dtype=torch.int64, device=DEV))
    new = lambda like, dtype=torch.bfloat16: torch.empty(like.shape, dtype=dtype, device=DEV)
    calls = [(new(dy), lambda o: h.linear(x, w, out=o)), (new(dy), lambda o: h.linear_kept(x, w, out=o)), (new(x), lambda o: h.linear_grad_input(dy, w, out=o)),
             (new(w, torch.float32), lambda o: h.linear_grad_weight(dy, x, out=o)), (new(x), lambda o: h.layer_norm(x, out=o)),
             (new(x), lambda o: h.layer_norm_grad(x, x, None, n, out=o)), (new(x), lambda o: h.act_grad(x, x, "gelu", out=o)),
             (new(q.data, torch.uint8), lambda o: h.act8_quantize(x, out=o)), (new(x), lambda o: h.act8_restore(q, out=o)),
             (new(dy), lambda o: h.mx4_linear(x, z, out=o)), (new(w), lambda o: h.mx4_dequantize(z, out=o)),
             (new(logits, torch.float32), lambda o: h.token_logprobs_grad(logits, torch.zeros(4, dtype=torch.int64, device=DEV), r, torch.ones(4, device=DEV), out=o))]
    for i, (out, f) in enumerate(calls):
        before, inputs = out._version, [t._version for t in (x, w, dy)]
        f(out)
        assert out._version == before + 1, i
        assert [t._version for t in (x, w, dy)] == inputs, i
    leaf = torch.ones(4, 8, device=DEV, requires_grad=True)
    y = torch.zeros(4, 8, device=DEV)
    product = leaf * y                             # saves y
    h.linear(x, w, out=y)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.sum().backward()
    with torch.inference_mode():
        out = new(dy)
        h.linear(x, w, out=out)                    # has no version
        assert torch.equal(out, h.linear(x, w))


def test_long_products_on_several_streams_at_once(h):
    """Products whose runs are added up in tensor memory (all of an SM's, or a part), ones of many rows and 4-bit ones on four streams that nothing orders,
    and captured in two graphs that are replayed at once: each gives what it gives alone."""
    calls = []
    for i, (rows, k, n) in enumerate(((2, 50304, 1000), (64, 11008, 4096), (500, 9000, 500), (16, 30000, 3000), (2304, 3000, 2304))):
        x, w = big(rows, k, i), big(n, k, i + 10, size=0.1)
        q = h.mx4_quantize(w, "e8m0_32")
        calls += [lambda x=x, w=w: h.linear(x, w, dtype=torch.float32), lambda x=x, w=w: h.linear(x, w, act="gelu"), lambda x=x, q=q: h.mx4_linear(x, q)]
    alone = [f() for f in calls]
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream() for _ in range(4)], []
    for turn in range(4):
        for j, s in enumerate(streams):
            with torch.cuda.stream(s):
                results.append([calls[(i * 7 + 5 * j + turn) % len(calls)]() for i in range(len(calls))])
    torch.cuda.synchronize()
    for t, r in enumerate(results):
        for i, y in enumerate(r):
            assert torch.equal(y, alone[(i * 7 + 5 * (t % 4) + t // 4) % len(calls)])
    graphs, replayed = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            replayed.append([f() for f in calls])
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for r in replayed:
        assert all(torch.equal(y, a) for y, a in zip(r, alone))
    h.score_status()
