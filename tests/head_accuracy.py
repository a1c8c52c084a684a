"""The arithmetic of a head with 4-bit weights in numpy, with the weights held as offset + q.

A group's sum starts at -(offset + 8) times the sum of its hidden values, so the larger the offset, the larger the
sums that are rounded on the way to a result that does not depend on it.  Products are exact, every 32 of them and
the sum so far are rounded once, a group's sum is scaled into its wave's (256 columns), and the waves' are added.
"""
import numpy as np

import step_reference as ref


def off(got, want):
    return np.sqrt(np.mean((got - want) ** 2) / np.mean(want ** 2))


def simulated(hidden, codes, scales, offset):
    q = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1).astype(np.float64)
    B, K = hidden.shape
    group = K // scales.shape[1]
    h = hidden.astype(np.float64)
    waves = []
    for k in range(0, K, 256):
        total = np.zeros((B, q.shape[0]), np.float32)
        for at in range(k, k + 256, group):
            s = np.zeros_like(total)
            for w in (np.full_like(q, -offset - 8.0), q + offset):
                for i in range(at, at + group, 32):
                    s = (s + h[:, i:i + 32] @ w[:, i:i + 32].T).astype(np.float32)
            total = (total + s.astype(np.float64) * scales[:, at // group]).astype(np.float32)
        waves.append(total)
    out = waves[0]
    for w in waves[1:]:
        out = out + w
    return out.astype(np.float64)
