"""Scores a text with a checkpoint's final norm and output embedding before and after it went through the compressor, the
restored one held in 16 bits and at 4 bits, and takes the gradient of the score: with respect to the logits, and through the
16-bit weights to the embedding, the norm and the hidden states.

    python examples/score_checkpoint.py [--shape tiny|pythia-410m|pythia-1.4b|llama-7b] [--tokens N] [--format e8m0_32|e4m3_16]

The weights, the moments and the hidden states are synthetic (seeded); there is no trained model here, so the
numbers say how far compression and 4 bits move the log probabilities, not how good a model is.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2406_11257_b200 import binding, synth  # noqa: E402


def score(shape: str = "tiny", tokens: int = 256, fmt: str = "e4m3_16", seed: int = 1) -> dict:
    cfg = synth.CONFIG_SHAPES[shape]
    n, d, v = cfg.vocab * cfg.d_model, cfg.d_model, cfg.vocab
    w_t, w_prev, ea, eas = synth.make_quad(n, seed, 0, device="cuda")
    h = binding.Handle(workspace_numel=n)

    # the checkpoint's step: compress W_t against the last reconstruction, restore W^_t
    blob = torch.empty(binding.compress_bound(n), dtype=torch.uint8, device="cuda")
    nbytes, _ = h.compress_tensor(binding.Params(median_source=binding.MEDIAN_ABS_RESIDUAL), w_t, w_prev, ea, eas, blob)
    restored = torch.empty_like(w_t)
    h.decompress_tensor(blob, nbytes, w_prev, restored, ea, eas)

    gen = torch.Generator(device="cuda").manual_seed(seed)
    hidden = torch.randn(tokens, d, generator=gen, device="cuda").to(torch.bfloat16)
    text = torch.randint(0, v, (tokens,), generator=gen, device="cuda")
    # the final norm: with mean and bias for the neox shapes, without for the llama ones; the input is kept in 8 bits for its gradient
    rms = cfg.family == "llama"
    norm_w = torch.ones(d, device="cuda")
    norm = h.layer_norm(hidden, norm_w, None if rms else torch.zeros(d, device="cuda"), rms=rms, keep=True)
    hidden, states = norm.y, hidden
    scale_x = h.mx4_tensor_scale(hidden) if fmt == "e4m3_16" else None

    def run(weights: torch.Tensor):
        weights = weights.view(v, d)
        packed = h.mx4_quantize(weights, fmt, h.mx4_tensor_scale(weights) if fmt == "e4m3_16" else None)
        logits = h.mx4_linear(hidden, packed, tensor_scale=scale_x)
        return logits, h.token_logprobs(logits, text, top=5)

    _, before = run(w_t)
    logits, after = run(restored)
    grad = h.token_logprobs_grad(logits, text, after, torch.full((tokens,), -1.0 / tokens, device="cuda"))
    # the same with the restored weights themselves, in 16 bits, and the way back to them
    w16 = restored.view(v, d).to(torch.bfloat16)
    logits16 = h.linear(hidden, w16)
    exact = h.token_logprobs(logits16, text)
    dlogits = h.token_logprobs_grad(logits16, text, exact, torch.full((tokens,), -1.0 / tokens, device="cuda"))
    dw = h.linear_grad_weight(dlogits, hidden)
    back = h.layer_norm_grad(h.linear_grad_input(dlogits, w16), norm.kept, norm_w, norm)
    plain = torch.log_softmax(hidden.float() @ restored.view(v, d).T, 1).gather(1, text[:, None])[:, 0]
    h.score_status()
    out = {"record_bytes": nbytes, "weights_bytes": 4 * n, "packed_bytes": binding.mx4_bytes(v, d, fmt),
           "mean_logprob_original": before.logprob.mean().item(), "mean_logprob_restored": after.logprob.mean().item(),
           "mean_logprob_restored_16bit": exact.logprob.mean().item(), "mean_logprob_restored_fp32": plain.mean().item(), "mean_entropy": after.entropy.mean().item(),
           "largest_change": (before.logprob - after.logprob).abs().max().item(),
           "same_first_choice": (before.top_index[:, 0] == after.top_index[:, 0]).float().mean().item(),
           "gradient_sum": grad.float().sum().item(), "embedding_gradient_norm": dw.norm().item(), "embedding_gradient_column_sum": dw.sum(0).abs().max().item(),
           "norm_gradient_norm": back.dweight.norm().item(), "state_gradient_along_states": (back.dx.float() * states.float()).sum(1).abs().max().item()}
    h.close()
    return out


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--shape", default="pythia-410m", choices=sorted(synth.CONFIG_SHAPES))
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--format", default="e4m3_16", choices=sorted(binding.MX4_FORMAT))
    a = ap.parse_args()
    for k, x in score(a.shape, a.tokens, a.format).items():
        print(f"{k:28s} {x}")
