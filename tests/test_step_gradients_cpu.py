"""What carries no gradient refuses an input that asks for one (before any look at the device)."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def head():
    return (torch.zeros((2, 128), dtype=torch.bfloat16), torch.zeros((5, 64), dtype=torch.uint8),
            torch.zeros((5, 1)))


def test_head_refuses_inputs_that_require_a_gradient(sbw):
    hidden, codes, scales = head()
    for which in (hidden, scales):
        which.requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            sbw.head_logits(hidden, codes, scales)
        with torch.no_grad(), pytest.raises(ValueError, match="device"):   # the next check
            sbw.head_logits(hidden, codes, scales)
        which.requires_grad_(False)
    with pytest.raises(ValueError, match="device"):
        sbw.head_logits(hidden.requires_grad_().detach(), codes, scales)


def test_candidates_values_refuse_logits_that_require_a_gradient(sbw):
    logits = torch.zeros((2, 9), requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        sbw.top_candidates(logits, 3)
    with pytest.raises(ValueError, match="gradient"):
        sbw.top_candidates(logits, 3, values=torch.zeros((2, 3)), with_values=False)
    with pytest.raises(ValueError, match="device"):            # ids alone have none to lose
        sbw.top_candidates(logits, 3, with_values=False)
    with pytest.raises(ValueError, match="device"):
        sbw.top_candidates(logits.detach(), 3)
    with torch.no_grad(), pytest.raises(ValueError, match="device"):
        sbw.top_candidates(logits, 3)


def test_tangents_are_refused(sbw):
    hidden, codes, scales = head()
    logits, ids = torch.zeros((2, 9)), torch.zeros(2, dtype=torch.int32)
    stats, g = torch.zeros((2, 2)), torch.zeros(2)
    calls = [(lambda a: sbw.token_logprobs(a, ids), logits), (lambda a: sbw.top_candidates(a, 3), logits),
             (lambda a: sbw.head_logits(a, codes, scales), hidden), (lambda a: sbw.head_logits(hidden, codes, a), scales),
             (lambda a: sbw.token_logprobs_grad(a, ids, stats, None, g), logits),
             (lambda a: sbw.token_logprobs_grad(logits, ids, a, None, g), stats),
             (lambda a: sbw.token_logprobs_grad(logits, ids, stats, None, a), g)]
    with forward_ad.dual_level():
        for call, t in calls:
            with pytest.raises(ValueError, match="device"):
                call(t)
            with pytest.raises(ValueError, match="tangent"):
                call(forward_ad.make_dual(t, torch.ones_like(t)))
