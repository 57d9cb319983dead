"""The example's way back: from the score of a text through the restored 16-bit embedding and the final norm."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("tokens", [1, 300])
def test_score_checkpoint_with_16_bit_weights(tokens):
    import score_checkpoint
    r = score_checkpoint.score("tiny", tokens, "e8m0_32")
    # 256 products of weights (0.02, rounded by 2^-9 of themselves) with unit values move a logit by 0.02 * 16 * 2^-9, a log probability by
    # no more than twice the largest of them, and the logit's own rounding by 2^-9 of about 1
    assert abs(r["mean_logprob_restored_16bit"] - r["mean_logprob_restored_fp32"]) < 0.02
    assert r["embedding_gradient_norm"] > 0 and r["norm_gradient_norm"] > 0
    # over the words the gradients of the logits of a token add up to nothing, up to the 16-bit rounding of 4096 of them (2 / tokens in
    # all, 2^-9 each) times a hidden value of at most 5
    assert r["embedding_gradient_column_sum"] < 5 * 2.0 * 2 ** -8
    # moving a row along itself does not change its norm's result (but for eps): what is left is the rounding of dx and of the
    # states kept in 8 bits, 2^-6 of |dx| |state| per row; |dx| is at most |dlogits| |w| = 2 / tokens * 0.02 * 64
    assert r["state_gradient_along_states"] < 2.0 ** -6 * (2.0 / tokens) * 0.02 * 64 * 16 * 1.5
