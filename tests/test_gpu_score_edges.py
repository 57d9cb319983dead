"""Edges of the scoring operators, through the C ABI, against their 64-bit definitions (oracle/score_oracle.py): where a result
could be wrong at values, sizes or an order of calls that ordinary use seldom meets.

Tolerances (derived, not fitted) are those of test_gpu_score.py unless a test says its own."""
import numpy as np
import pytest
import torch

from oracle import score_oracle as so
from paper_2406_11257_b200 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def h():
    handle = binding.Handle(workspace_numel=4096, device=0)
    yield handle
    handle.score_status()
    handle.close()


def device_scale(v):
    return torch.tensor(float(v), dtype=torch.float32, device=DEV)


def test_first_call_of_a_handle_on_a_stream_of_its_own():
    """The workspace is clear before the first kernel uses it, whatever the default stream is busy with."""
    x = torch.randn((700, 900), device=DEV)
    want = so.tensor_scale(x.cpu().numpy())
    big = torch.empty(1 << 28, dtype=torch.float32, device=DEV)
    side, third = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        handle = binding.Handle(workspace_numel=4096, device=0)
        for _ in range(40):                        # about 20 ms of work on the default stream
            big.zero_()
        with torch.cuda.stream(side):
            first = handle.mx4_tensor_scale(x)
        done = side.record_event()
        with torch.cuda.stream(third):             # the second call on yet another stream, behind the first
            third.wait_event(done)
            second = handle.mx4_tensor_scale(x)
        third.synchronize()
        with torch.cuda.stream(third):
            assert float(first) == float(second) == float(want)
        torch.cuda.synchronize()
        assert float(handle.mx4_tensor_scale(x)) == float(want)
        handle.close()


@pytest.mark.parametrize("fmt", ["e8m0_32", "e4m3_16"])
@pytest.mark.parametrize("rows,k,n", [(40, 4096, 700), (300, 4096, 700), (1100, 4096, 6000)])
def test_waits_that_run_out_in_the_middle(h, rows, k, n, fmt):
    """Limits at which some waits are met and others are not: a result is right or reported, and the calls behind it are right."""
    x = torch.randn((rows, k), generator=torch.Generator().manual_seed(11)).to(torch.bfloat16).to(DEV)
    m = h.mx4_quantize(torch.randn((n, k), generator=torch.Generator().manual_seed(12)).to(DEV), fmt)
    want = h.mx4_linear(x, m)
    try:
        for limit in (1, 2000, 10000, 30000, 100000):
            h.set_wait_limit(limit)
            y = h.mx4_linear(x, m)
            reported = False
            try:
                h.score_status()
            except binding.ExcpError as e:
                assert e.status == -7
                reported = True
            assert reported or torch.equal(y, want)
            h.set_wait_limit(2_000_000_000)
            assert torch.equal(h.mx4_linear(x, m), want)
            h.score_status()
    finally:
        h.set_wait_limit(2_000_000_000)


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("scale", [None, 0.7, 2.0 ** -20, 2.0 ** 90])
def test_zeros_keep_their_sign_among_other_values(h, scale, dtype):
    """Code 8 for -0, also where the block's scale is not 0 (a scale of 2^90 takes the division, the others the reciprocal)."""
    g = torch.Generator().manual_seed(61)
    x = torch.randn((37, 330), generator=g)
    if scale == 2.0 ** 90 and dtype != "fp16":
        x = x * 2.0 ** 90
    x[:, ::3] = -0.0
    x[:, 1::7] = 0.0
    x = x.to(DT[dtype]).to(DEV)
    m = h.mx4_quantize(x, "e4m3_16", tensor_scale=None if scale is None else device_scale(scale))
    codes, scales = so.quantize(x.to(torch.float32).cpu().numpy(), "e4m3_16", scale)
    assert np.array_equal(m.data.cpu().numpy(), so.pack(codes, scales, "e4m3_16"))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("largest", [1e-34, 2688 * 2.0 ** -126, 3e-35, 1e-36, 777.0 * 2.0 ** -126, 1e-40, 2.0 ** -149 * 2688, 2.0 ** -133])
def test_tensor_scale_of_tiny_matrices(h, largest, dtype):
    """The quotient is rounded up to 8 significant bits of its own, subnormal or not; a quotient of 0 gives 1."""
    x = torch.zeros((5, 300))
    x[3, 7], x[4, 299] = -largest, largest / 3
    x = x.to(DT[dtype]).to(DEV)
    want = so.tensor_scale(x.to(torch.float32).cpu().numpy())
    assert float(h.mx4_tensor_scale(x)) == float(want)


SCALES = [(165 / 128 * 2.0 ** -80, 25 / 16 * 2.0 ** -62), (2.0 ** -90, 1.5 * 2.0 ** -62), (1.5 * 2.0 ** -30, 2.0 ** -118), (2.0 ** 70, 1.25 * 2.0 ** 60),
          (1.5 * 2.0 ** 100, 2.0 ** -120)]


@pytest.mark.parametrize("ga,gb", SCALES)
@pytest.mark.parametrize("rows,k,n", [(1, 500, 300), (40, 320, 200), (300, 256, 300), (1100, 256, 2080), (1100, 256, 2085)])
def test_product_of_tensor_scales_out_of_range(h, rows, k, n, ga, gb):
    """The product of the two tensor scales may be subnormal, 0 or infinite in fp32 although the results are not.

    Tolerance: that of the sums (test_gpu_score.py), two roundings by the scales, the last one among subnormals."""
    gen = torch.Generator().manual_seed(71)
    xa, xb = torch.randn((rows, k), generator=gen).numpy() * 64, torch.randn((n, k), generator=gen).numpy() * 64
    xa[rows // 2:rows // 2 + 1, :] = 0 if rows > 1 else xa[0]
    xb[n // 2] = 0
    xa, xb = (xa * np.float64(ga)).astype(np.float32), (xb * np.float64(gb)).astype(np.float32)
    qa, qb = so.quantize(xa, "e4m3_16", ga), so.quantize(xb, "e4m3_16", gb)
    ma = binding.Mx4Matrix(torch.from_numpy(so.pack(*qa, "e4m3_16")).to(DEV), rows, k, "e4m3_16", device_scale(ga))
    mb = binding.Mx4Matrix(torch.from_numpy(so.pack(*qb, "e4m3_16")).to(DEV), n, k, "e4m3_16", device_scale(gb))
    a, b = so.values(*qa, "e4m3_16", ga), so.values(*qb, "e4m3_16", gb)
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    tol = (-(-k // 64) + 16) * 2.0 ** -22 * mag + 3 * 2.0 ** -24 * np.abs(want) + 2.0 ** -148
    most = float(np.finfo(np.float32).max)
    for y in (h.mx4_matmul(ma, mb, dtype=torch.float32), h.mx4_linear(torch.from_numpy(xa).to(DEV), mb, tensor_scale=device_scale(ga))):
        got = y.cpu().numpy().astype(np.float64)
        over = np.abs(want) > 1.01 * most
        assert np.array_equal(got[over], np.copysign(np.inf, want[over]))
        fits = np.abs(want) < 0.99 * most
        assert np.isfinite(got[fits]).all()
        worst = (np.abs(got - want)[fits] / tol[fits]).max(initial=0.0)
        assert worst <= 1.0, worst
    h.score_status()


@pytest.mark.parametrize("dtype", sorted(DT))
def test_gradient_of_a_token_past_the_vocabulary(h, dtype):
    """Its log probability is NaN, and so is the gradient of its row where there is a g_logprob; the entropy does not
    depend on the token."""
    vocab = 903
    x = (torch.randn((5, vocab), generator=torch.Generator().manual_seed(81)) * 3).to(DT[dtype]).to(DEV)
    tokens = torch.tensor([3, vocab, -1, 1 << 40, 7], device=DEV)
    inside = torch.tensor([3, 0, -1, 0, 7], device=DEV)
    gl, gh = torch.randn(5, device=DEV), torch.randn(5, device=DEV)
    r, s = h.token_logprobs(x, tokens), h.token_logprobs(x, inside)
    assert torch.isnan(r.logprob).tolist() == [False, True, False, True, False]
    assert torch.equal(r.entropy, s.entropy)
    assert torch.equal(h.token_logprobs_grad(x, tokens, r, None, gh), h.token_logprobs_grad(x, inside, s, None, gh))
    assert not h.token_logprobs_grad(x, tokens, r, None, None).any()
    got, other = h.token_logprobs_grad(x, tokens, r, gl, gh), h.token_logprobs_grad(x, inside, s, gl, gh)
    assert torch.isnan(got[1]).all() and torch.isnan(got[3]).all()
    for i in (0, 2, 4):
        assert torch.equal(got[i], other[i])


@pytest.mark.parametrize("rows,vocab", [(3, 901), (2, 131072), (1500, 300)])
def test_row_statistics_are_of_the_logits_before_scaling(h, rows, vocab):
    """What a C caller may read: the largest logit itself, the sum of exp(scale (x - largest)), the entropy, 0."""
    x = torch.randn((rows, vocab), generator=torch.Generator().manual_seed(83)).to(DEV) * 4
    r = h.token_logprobs(x, torch.zeros(rows, dtype=torch.int64, device=DEV), scale=0.6)
    stats = r.row_stats.cpu()
    xd = x.double().cpu()
    assert torch.equal(stats[:, 0], x.max(1).values.cpu())
    want = torch.exp(float(np.float32(0.6)) * (xd - xd.max(1, keepdim=True).values)).sum(1)
    # a sum of positive terms: exp of a rounded argument of at most 40, and the chain of additions
    assert ((stats[:, 1].double() - want).abs() <= want * (40 * 2.0 ** -22 + (vocab / 256 + 64) * 2.0 ** -24)).all()
    assert torch.equal(stats[:, 2], r.entropy.cpu()) and not stats[:, 3].any()


@pytest.mark.parametrize("rows,top", [(50, 20), (333, 3), (300, 0)])
def test_results_hold_little_more_memory_than_their_own(h, rows, top):
    """The log probabilities and entropies may lie together, and the alternatives' two halves; the statistics lie alone."""
    r = h.token_logprobs(torch.randn((rows, 700), device=DEV), torch.zeros(rows, dtype=torch.int64, device=DEV), top=top)
    limits = {"logprob": 8, "entropy": 8, "row_stats": 16} | ({"top_logprob": 12 * top, "top_index": 12 * top} if top else {})
    for name, bytes_a_row in limits.items():
        t = getattr(r, name)
        assert t.untyped_storage().nbytes() <= rows * bytes_a_row and t.is_contiguous(), name


@pytest.mark.parametrize("rows,top", [(1, 20), (2, 19), (21, 0), (9, 2)])
def test_results_of_a_few_rows_hold_one_block(h, rows, top):
    """Up to the allocator's smallest block of 512 bytes nothing is gained by taking them apart; they do not overlap."""
    x = torch.randn((rows, 700), device=DEV)
    r = h.token_logprobs(x, torch.zeros(rows, dtype=torch.int64, device=DEV), top=top)
    places = []
    for name in ("logprob", "entropy", "row_stats") + (("top_logprob", "top_index") if top else ()):
        t = getattr(r, name)
        assert t.untyped_storage().nbytes() <= 512
        places.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()))
    places.sort()
    assert all(a[1] <= b[0] for a, b in zip(places, places[1:]))


@pytest.mark.parametrize("top", [1 << 32, (1 << 32) + 3, -(1 << 32), 1 << 40, (1 << 31) + 1])
def test_numbers_of_alternatives_past_32_bits_are_refused(h, top):
    with pytest.raises(binding.ExcpError) as e:
        h.token_logprobs(torch.ones((4, 64), device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV), top=top)
    assert e.value.status == -1


def test_gradient_past_32_bit_offsets(h):
    """2.2e9 half-precision logits: the last rows lie past element 2^31 and byte 2^32 of what is read and of what is written."""
    rows, vocab = 17000, 131000
    x = torch.zeros((rows, vocab), dtype=torch.float16, device=DEV)
    gen = torch.Generator().manual_seed(91)
    x[-2:] = (torch.randn((2, vocab), generator=gen) * 3).to(torch.float16).to(DEV)
    tokens = torch.full((rows,), 77, device=DEV)
    last = x[-2:].to(torch.float32).cpu().numpy()
    r = h.token_logprobs(x, tokens)
    gl, gh = torch.ones(rows, device=DEV), torch.full((rows,), 0.5, device=DEV)
    h.token_logprobs_grad(x, tokens, r, gl, gh, out=x)
    wg = so.logprobs_grad(last, [77, 77], 1.0, [1.0, 1.0], [0.5, 0.5])
    p = so.logprobs(last, [77, 77])["p"]
    # fp32: log p and the entropy are off by (chain + reach) 2^-22, p by as much of itself; then half an ulp of fp16
    tol = np.abs(wg) * 2.0 ** -11 + p * 40 * (vocab / 256 + 100) * 2.0 ** -24 + 2.0 ** -25
    tol[:, 77] += 2.0 ** -22
    got = x[-2:].to(torch.float32).cpu().numpy().astype(np.float64)
    assert (np.abs(got - wg) <= tol).all()
    even = so.logprobs_grad(np.zeros((1, vocab)), [77], 1.0, [1.0], [0.5])
    for i in (0, 100, 16390):                      # 16390: the row that holds element 2^31
        assert (np.abs(x[i:i + 1].to(torch.float32).cpu().numpy() - even) <= np.abs(even) * 2.0 ** -10 + 2.0 ** -24).all()
    del x


@pytest.mark.parametrize("dtype", sorted(DT))
@pytest.mark.parametrize("rows,vocab", [(5, 7), (1500, 40), (300, 901), (3, 60001)])
def test_a_nan_at_either_end_of_a_row_is_its_first_alternative(h, rows, vocab, dtype):
    x = (torch.randn((rows, vocab), generator=torch.Generator().manual_seed(97)) * 3).to(DT[dtype])
    x[0, 0] = x[1, vocab - 1] = x[2, 0] = x[2, 3] = x[2, vocab - 1] = float("nan")
    xn = x.to(torch.float32).numpy()
    r = h.token_logprobs(x.to(DEV), torch.zeros(rows, dtype=torch.int64, device=DEV), top=5)
    assert np.array_equal(r.top_index[:3].cpu().numpy(), so.logprobs(xn[:3], [0, 0, 0], 1.0, 5)["top_index"])
    assert torch.isnan(r.top_logprob[:3]).all() and torch.isfinite(r.top_logprob[3:]).all()


@pytest.mark.parametrize("fmt", ["e8m0_32", "e4m3_16"])
@pytest.mark.parametrize("cols", [33000, 32800])
def test_quantisation_past_32_bit_offsets(h, cols, fmt):
    """2.2e9 values: the last rows lie past element 2^31 and byte 2^32 of the matrix, and past 2^30 bytes of the packed one (rows
    that start on 32 bytes, and others)."""
    rows, tail = 66000, 66000 % 128
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device=DEV)
    x[-tail:] = (torch.randn((tail, cols), generator=torch.Generator().manual_seed(99)) * 3).to(torch.bfloat16).to(DEV)
    last = x[-tail:].to(torch.float32).cpu().numpy()
    g = h.mx4_tensor_scale(x) if fmt == "e4m3_16" else None
    gf = None if g is None else float(g)
    assert g is None or gf == float(so.tensor_scale(last))
    m = h.mx4_quantize(x, fmt, tensor_scale=g)
    codes, scales = so.quantize(last, fmt, gf)
    packed = so.pack(codes, scales, fmt)               # the last row tile alone has the layout of a matrix of its own
    assert np.array_equal(m.data[-packed.size:].cpu().numpy(), packed)
    x.fill_(7.0)
    h.mx4_dequantize(m, out=x)
    want = torch.from_numpy(so.values(codes, scales, fmt, gf).astype(np.float32)).to(torch.bfloat16)
    assert torch.equal(x[-tail:].cpu(), want)
    assert not x[:-tail].any()
    del x, m
