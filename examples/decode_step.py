"""One watermarked decode step from hidden states to tokens with their log probabilities, and one
training step on them, with the operators of this library alone.

    python examples/decode_step.py [rows] [vocabulary] [hidden size]

decode   head_logits (4-bit head) -> top_candidates -> watermark_candidates (the top-k scheme) ->
         watermark_sample without a bias of its own -> token_logprobs of the sampled tokens
detect   the same window and key on the tokens
train    token_logprobs of a target with its gradient: cross entropy, an entropy bonus and a penalty
         on the log sum
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_03844_amd as sbw  # noqa: E402

KEY, GAMMA, DELTA, TOP = 15485863, 0.25, 2.0, 40


def decode_step(hidden, codes, scales, window, seeds, inv_temperature=1.25):
    """(tokens [B], TokenLogprobs of the watermarked distribution, candidates [B, TOP])."""
    logits = sbw.head_logits(hidden, codes, scales)
    candidates, _ = sbw.top_candidates(logits, TOP)
    sbw.watermark_candidates(logits, window, candidates, KEY, GAMMA, DELTA)
    # the logits carry their bias now: gamma = 0 samples without another
    tokens, _ = sbw.watermark_sample(logits, window, KEY, 0.0, 0.0, seeds,
                                     inv_temperature=inv_temperature, with_scores=False)
    return tokens, sbw.token_logprobs(logits, tokens, inv_temperature, top=5), candidates


def training_step(logits, targets, entropy_bonus=0.01, log_sum_penalty=1e-4):
    """(loss, its gradient with respect to the logits)."""
    logits = logits.requires_grad_()
    r = sbw.token_logprobs(logits, targets)
    loss = -r.logprobs.mean() - entropy_bonus * r.entropy.mean() + log_sum_penalty * r.lse.square().mean()
    loss.backward()
    return loss.detach(), logits.grad


def main(rows=8, vocabulary=32000, hidden_size=2048):
    g = torch.Generator(device="cuda").manual_seed(7)
    codes = torch.randint(0, 256, (vocabulary, hidden_size // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.empty((vocabulary, hidden_size // 128), device="cuda").uniform_(0.5, 1.5, generator=g)
    scales *= 0.65 / hidden_size ** 0.5
    window = torch.randint(0, vocabulary, (rows, 4), generator=g, device="cuda", dtype=torch.int32)
    text = [window]
    for step in range(16):
        hidden = torch.randn((rows, hidden_size), generator=g, device="cuda").to(torch.bfloat16)
        seeds = torch.randint(0, 1 << 62, (rows,), generator=g, device="cuda")
        tokens, answer, candidates = decode_step(hidden, codes, scales, window, seeds)
        text.append(tokens[:, None])
        window = torch.cat([window[:, 1:], tokens[:, None]], dim=1).contiguous()
    print(f"last step: log probabilities {answer.logprobs.mean().item():.3f}, entropy "
          f"{answer.entropy.mean().item():.3f} nats, likeliest {answer.top_logprobs[:, 0].mean().item():.3f}")
    counts, scored, z = sbw.detect_ex(torch.cat(text, dim=1).contiguous(), KEY, GAMMA, "self_salt", width=4)
    print(f"green {counts.sum().item()} of {scored.sum().item()}, mean z {z.mean().item():.2f}")
    loss, grad = training_step(sbw.head_logits(hidden, codes, scales), tokens)
    print(f"loss {loss.item():.3f}, gradient norm {grad.norm().item():.4f}")


if __name__ == "__main__":
    main(*map(int, sys.argv[1:]))
