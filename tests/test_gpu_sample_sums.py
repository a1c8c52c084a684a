"""Filtered sampling where the sums of weights decide: tails far below the largest weight."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def say(text):
    print(text, flush=True)


def adds(V):
    """Roundings in a row's sum of weights: a lane's vectors, a wave, the parts one after another (two products, an exponential and
    an addition each) and the wave that joined them."""
    return 32 + 6 * (V / 2 ** 15 + 1)


def cut_range(row, top_p):
    """(sum kept at least, at most) of weights relative to the largest, 1 / T = 1.

    The steps for wide rows hold weights in fp32.  A score is off by 4 u of itself (the difference, its factor's two roundings, the
    product), so a weight by u (4 |y| + 2) of itself, the exponential's own unit in the last place among it.  The sum of all is
    off by `adds` roundings besides, what it is compared with by whole numbers of 2^-61 of it each: together
    u (adds + 8 E|y| + 5).  A logit whose place is within that of where top-p ends may be kept or not."""
    x = np.sort(row.astype(np.float64))[::-1]
    y = x - x[0]
    e = np.exp(y)
    S = e.sum()
    off = U * (adds(row.size) + 8 * (e * np.abs(y)).sum() / S + 5)
    before = np.cumsum(e) - e
    return [max(e[0], e[before < float(np.float32(top_p)) * (1 + sign * off) * S].sum()) for sign in (-1, 1)]


def check_tail(sbw, rows, top_ps):
    """Rows whose first column is drawn but for a chance that the tail's sum is: its log probability shows what was kept."""
    x = np.stack(rows).astype(np.float32)
    t = torch.from_numpy(x).cuda()
    rng = np.random.default_rng(5)
    for top_p in top_ps:
        seeds = torch.from_numpy(rng.integers(0, 2 ** 63, len(rows), dtype=np.int64)).cuda()
        tokens, logprobs = (v.cpu().numpy() for v in sbw.sample_tokens(t, seeds, top_p=top_p))
        for b, row in enumerate(x):
            if tokens[b] != row.argmax():
                continue
            low, high = cut_range(row, top_p)
            kept = np.exp(-float(logprobs[b]))
            # the sum of what is kept: at most 64 weights a lane and a wave's lanes in fp32, weights as above, the logarithm and its rounding
            slack = U * (72 + 8 * 21 * (high - 1) + 8)
            say(f"tail row {b} top_p {top_p} kept 1 + {kept - 1:.6e}, definition 1 + {low - 1:.6e} to 1 + {high - 1:.6e}")
            assert low * (1 - slack) <= kept <= high * (1 + slack), (b, top_p)
        assert (tokens == x.argmax(1)).sum() >= len(rows) - 1


@pytest.mark.parametrize("V", [128256, 152064, 1000003])
def test_tails_of_weights_near_a_billionth(sbw, V):
    """One likely token and a tail that holds a small part of the sum, weights between 2^-31 and 2^-29 of the largest: what is
    kept of it goes by sums that must not round such weights to a common unit."""
    rng = np.random.default_rng(V)

    def row(weights):
        r = np.log(rng.permutation(weights)).astype(np.float32)
        at = rng.integers(0, V)
        r[at] = 0.0
        return r
    unit = 2.0 ** -30
    spread = row(np.linspace(1.02, 1.48, V) * unit)
    small = row(np.linspace(0.3, 0.49, V) * unit)
    tied = row(np.concatenate([np.full(V // 2, 2.49), np.linspace(1.02, 1.45, V - V // 2)]) * unit)
    for r in (spread, small, tied):
        tail = (np.exp(r.astype(np.float64))).sum() - 1
        check_tail(sbw, [r] * 4, [1 - tail * part for part in (0.15, 0.4, 0.8)])
