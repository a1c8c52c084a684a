"""Filtered sampling says so where a gradient would be dropped (the Python path, before the device is looked at)."""
import pytest
import torch


def test_a_temperature_that_requires_a_gradient():
    import paper_2609_03844_amd as sbw
    x, seeds, each = torch.zeros((3, 8)), torch.zeros(3, dtype=torch.int64), torch.ones(3, requires_grad=True)
    with pytest.raises(ValueError, match="no gradient to inv_temperature"):
        sbw.sample_tokens(x, seeds, each)
    with torch.no_grad(), pytest.raises(ValueError, match="current HIP device"):
        sbw.sample_tokens(x, seeds, each)
    with pytest.raises(ValueError, match="current HIP device"):
        sbw.sample_tokens(x, seeds, each, with_logprobs=False)
    # filters have no derivative but zero
    with pytest.raises(ValueError, match="current HIP device"):
        sbw.sample_tokens(x, seeds, top_p=each, min_p=each)
