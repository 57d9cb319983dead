"""Pins of the 64-bit definitions that the scoring operators are tested against: hand values of the 4-bit formats,
the packed layout, probabilities from exact sums, the gradient against differences."""
import math

import numpy as np
import pytest

from oracle import score_oracle as so
from paper_2406_11257_b200 import binding


def test_e2m1_rounds_to_nearest_ties_to_even():
    x = np.zeros((1, 32), np.float32)
    x[0, :16] = [0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.0000005, -0.25, -0.75, -5.5, 6.0, 7.9, 4.0, -0.0]
    codes, scale = so.quantize(x, "e8m0_32")          # largest 7.9: floor(log2) = 2, scale 2^0
    assert scale.tolist() == [[127]]
    assert so.code_values(codes)[0, :16].tolist() == [0.0, 0.5, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -0.0, -1.0, -6.0, 6.0, 6.0, 4.0, 0.0]
    assert codes[0, 15] == 8                            # -0 keeps its sign


@pytest.mark.parametrize("largest,byte", [(6.0, 127), (4.0, 127), (3.999, 126), (8.0, 128), (1.0, 125), (0.0, 0), (2.0 ** -126, 0),
                                          (3.4e38, 252), (2.0 ** -149, 0)])
def test_power_of_two_scales(largest, byte):
    codes, scale = so.quantize(np.array([[largest, 0.0]], np.float32), "e8m0_32")
    assert scale[0, 0] == byte


def test_e4m3_table_and_scales():
    assert so.E4M3[:3].tolist() == [0.0, 2.0 ** -9, 2.0 ** -8] and so.E4M3[-1] == 448.0 and len(so.E4M3) == 127
    codes, scale = so.quantize(np.array([[6.0] + [0.0] * 15 + [3.0] + [1.5] * 2], np.float32), "e4m3_16")
    assert so.scale_values(scale, "e4m3_16").tolist() == [[1.0, 0.5]]
    assert so.values(codes, scale, "e4m3_16")[0, 16:].tolist() == [3.0, 1.5, 1.5]
    assert so.tensor_scale(np.array([2688.0 * 0.75], np.float32)) == 0.75
    assert so.tensor_scale(np.array([2688.0 * 0.7501, np.inf], np.float32)) == np.float32(0.75 + 2.0 ** -8)
    assert so.tensor_scale(np.zeros(3, np.float32)) == 1.0


def test_non_finite_blocks_are_nan():
    x = np.ones((1, 64), np.float32)
    x[0, 5], x[0, 40] = np.nan, -np.inf
    for fmt, bad in (("e8m0_32", [True, True]), ("e4m3_16", [True, False, True, False])):
        codes, scale = so.quantize(x, fmt)
        assert np.isnan(so.scale_values(scale, fmt))[0].tolist() == bad


@pytest.mark.parametrize("fmt", ["e8m0_32", "e4m3_16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (7, 255), (8, 256), (127, 257), (128, 64), (129, 512), (300, 700)])
def test_packing_is_a_bijection(fmt, rows, cols):
    rng = np.random.default_rng(rows * 1000 + cols)
    codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    scales = rng.integers(1, 127, (rows, -(-cols // so.BLOCK[fmt]))).astype(np.uint8)
    data = so.pack(codes, scales, fmt)
    c, s = so.unpack(data, rows, cols, fmt)
    assert np.array_equal(c, codes) and np.array_equal(s, scales)
    assert data.size == so.packed_bytes(rows, cols, fmt) == binding.mx4_bytes(rows, cols, fmt)
    # hand places of the first tile: row 9's chunk 2 sits at place 2 ^ 1; its scales follow the codes
    if rows == 300:
        assert data[9 * 128 + 3 * 16] == codes[9, 64] | codes[9, 65] << 4
        assert data[128 * 128 + 16 * 9 + 0] == scales[9, 0] and data[128 * 128 + 16 * 9 + 4 * 2 + 3] == scales[9 + 64, 3]


def test_sizes_of_nothing_and_unknown_formats():
    assert binding.mx4_bytes(0, 100, "e8m0_32") == 0 and binding.mx4_bytes(5, 0, "e4m3_16") == 0
    lib = binding.load_library()
    assert lib.excp_mx4_bytes(4, 4, 3) == 0 and lib.excp_mx4_bytes(1 << 31, 4, 1) == 0


def test_log_probabilities_of_a_hand_row():
    x = np.log(np.array([[0.5, 0.25, 0.125, 0.125]]))
    r = so.logprobs(x, [1], top=4)
    assert math.isclose(r["logprob"][0], math.log(0.25)) and math.isclose(r["entropy"][0], 1.75 * math.log(2))
    assert r["top_index"].tolist() == [[0, 1, 2, 3]]
    r = so.logprobs(np.array([[-np.inf] * 3]), [0], top=2)
    assert r["logprob"][0] == -np.inf and r["entropy"][0] == 0 and r["top_index"].tolist() == [[0, 1]]
    r = so.logprobs(np.array([[1.0, -np.inf, 1.0]]), [-1], top=3)
    assert r["logprob"][0] == 0 and math.isclose(r["entropy"][0], math.log(2)) and r["top_index"].tolist() == [[0, 2, 1]]


def test_gradient_against_differences():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(4, 9)) * 2
    tokens, scale = np.array([0, 8, -1, 3]), 0.7
    gl, gh = rng.normal(size=4), rng.normal(size=4)

    def f(y):
        r = so.logprobs(y, tokens, scale)
        return (gl * r["logprob"] + gh * r["entropy"]).sum()

    g = so.logprobs_grad(x, tokens, scale, gl, gh)
    eps = 1e-5
    for i in range(4):
        for v in range(9):
            y, w = x.copy(), x.copy()
            y[i, v] += eps
            w[i, v] -= eps
            # central difference: eps^2 of the third derivative, and rounding 1e-16 / eps
            assert abs((f(y) - f(w)) / (2 * eps) - g[i, v]) < 1e-8
