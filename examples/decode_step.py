"""One watermarked decode step from hidden states to tokens with their log probabilities, and one
training step on them, with the operators of this library alone.

    python examples/decode_step.py [rows] [vocabulary] [hidden size]

decode   head_logits (4-bit head) -> top_candidates -> watermark_candidates (the top-k scheme) ->
         watermark_sample without a bias of its own -> token_logprobs of the sampled tokens
requests quantize_fp8 and matmul_fp8 (an 8-bit head) -> watermark -> sample_tokens, each request with a
         temperature, top-k, top-p and min-p of its own
detect   the same window and key on the tokens
train    token_logprobs of a target with its gradient: cross entropy, an entropy bonus and a penalty
         on the log sum; then the same through linear_fp8, down to the head's weights
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


def requests_step(hidden, head, window, seeds, inv_temperatures, top_ks, top_ps, min_ps):
    """(tokens [B], their log probabilities among what each request's filters keep); head: codes and scales."""
    logits = sbw.matmul_fp8(*sbw.quantize_fp8(hidden), *head)
    sbw.watermark(logits, window, KEY, GAMMA, DELTA)
    return sbw.sample_tokens(logits, seeds, inv_temperatures, top_ks, top_ps, min_ps)


def head_training_step(hidden, weight, targets):
    """(loss, gradient of the hidden states, gradient of the head's weights) by 8-bit products."""
    hidden, weight = hidden.detach().requires_grad_(), weight.detach().requires_grad_()
    loss = -sbw.token_logprobs(sbw.linear_fp8(hidden, weight), targets).logprobs.mean()
    return loss.detach(), *torch.autograd.grad(loss, (hidden, weight))


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

    weight = torch.randn((vocabulary, hidden_size), generator=g, device="cuda") * (3 / hidden_size ** 0.5)
    head = sbw.quantize_fp8(weight, 128)
    inv_temperatures = torch.empty(rows, device="cuda").uniform_(0.7, 1.4, generator=g)
    top_ks = torch.arange(rows, device="cuda", dtype=torch.int32) % 3 * 20          # none, 20, 40
    top_ps = torch.empty(rows, device="cuda").uniform_(0.8, 1.0, generator=g)
    min_ps = torch.full((rows,), 0.01, device="cuda")
    tokens, logprobs = requests_step(hidden, head, window, seeds, inv_temperatures, top_ks, top_ps, min_ps)
    print(f"filtered: tokens {tokens.tolist()}, mean log probability {logprobs.mean().item():.3f}")
    loss, of_hidden, of_weight = head_training_step(hidden, weight, tokens)
    print(f"8-bit head: loss {loss.item():.3f}, gradient norms {of_hidden.norm().item():.4f} and {of_weight.norm().item():.4f}")


if __name__ == "__main__":
    main(*map(int, sys.argv[1:]))
