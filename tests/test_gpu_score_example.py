"""The example that runs the scoring operators together: a checkpoint compressed, restored, held at 4 bits, scored."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("fmt", ["e8m0_32", "e4m3_16"])
@pytest.mark.parametrize("tokens", [1, 300])
def test_score_checkpoint(fmt, tokens):
    import score_checkpoint
    r = score_checkpoint.score("tiny", tokens, fmt)
    assert r["record_bytes"] < r["weights_bytes"] and r["packed_bytes"] < r["weights_bytes"] / 6
    assert all(math.isfinite(v) for v in r.values())
    # weights of standard deviation 0.02 over 256 columns: logits of standard deviation 0.32, so every log probability is near
    # -log(4096) = -8.32; 4 bits move a logit by about a tenth of its deviation
    assert abs(r["mean_logprob_restored"] + math.log(4096)) < 1.0 + 4 * 0.32 / math.sqrt(tokens)
    assert abs(r["mean_logprob_restored"] - r["mean_logprob_restored_fp32"]) < 0.5
    # the residuals are 200 times smaller than the weights, and a pruned or quantised one is off by less than itself
    assert r["largest_change"] < 0.5
    # the gradient of a row sums to zero up to its bfloat16 rounding: 4096 entries of at most 2 / tokens in all, half an ulp 2^-9 each
    assert abs(r["gradient_sum"]) < 2.0 * 2 ** -8
