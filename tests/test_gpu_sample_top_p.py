"""Filtered sampling with a top-p of 0 and less."""
import numpy as np
import pytest
import torch

import step_reference
from test_gpu_step import logits, placed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def say(text):
    print(text, flush=True)


KINDS = {"small": dict(top_k=40), "thousand": dict(top_k=1000), "wide": dict(), "floor": dict(min_p=0.001),
         "counted": dict(top_k=3000), "low": dict(inv_t=2e38)}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 7, 4001, 32001, 128259])
def test_top_p_of_zero_and_less_keeps_the_first(sbw, V, dtype):
    """By whichever step a row takes, as a number and of each row."""
    rng = np.random.default_rng(V)
    x = logits(rng, 6, V)
    x[1] *= np.float32(0.1)                    # flat: much would be kept by mistake
    x[2] = np.round(x[2])                      # ties: the first column of the largest
    x[3] = 0.0
    t, exact = placed(x, dtype)
    seeds = torch.from_numpy(rng.integers(0, 2 ** 63, 6, dtype=np.int64)).cuda()
    first = np.array([step_reference.order(r)[0] for r in exact])
    for name, f in KINDS.items():
        for top_p in (0.0, -0.0, -1e-9, -0.1, -1.0, -3e38, -np.inf):
            say(f"top-p {top_p} {name} {dtype} {V}")
            for given in (top_p, torch.full((6,), top_p, device="cuda")):
                tokens, logprobs = sbw.sample_tokens(t, seeds, f.get("inv_t", 1.0), f.get("top_k", 0), given, f.get("min_p", 0.0))
                assert np.array_equal(tokens.cpu().numpy(), first), (name, top_p)
                assert not logprobs.any(), (name, top_p)
