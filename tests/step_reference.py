"""Plain 64-bit definitions of the operators of include/sbw_step.h, on the CPU, with the
tolerances that the kernels' 32-bit arithmetic allows.

Tolerances.  u = 2^-24 is the rounding error of one fp32 operation.
* A score y = (x - m) * inv_t carries at most four roundings, so 4 u |y|; its exponential is
  that much off, relatively, plus two units for the exponential itself.  A sum of N positive terms
  is off by at most u times the additions between a term and the sum: a lane's own (N / 1024 or 64),
  and at most 64 more in the trees.  Hence log S is off by ADDS u + 4 u E|y| at most, E|y| the mean
  of |y| under p.
* A gradient's p = exp((x - m) inv_t - log S) is off by 4 u (|log p| + log S) + 4 u relatively, the
  products behind it by a few roundings more.
* Outputs are fp32: a value beyond its range is an infinity.
* A head's group sum adds at most 136 |h| s per weight (weights offset by up to 128 on the way) in at
  most ADDS sequential additions.
"""
import numpy as np

U = 2.0 ** -24


def adds(N):
    return 64 + max(64, N / 1024)


def order(row):
    """Columns of a row, larger logits first, equal ones by column, NaN in front."""
    x = row.astype(np.float64) + 0.0
    rank = np.where(np.isnan(x), -np.inf, -x)
    return np.lexsort((np.arange(x.size), rank, ~np.isnan(x)))


def logprobs(x, tokens, inv_t, top=0):
    """(logprobs, lse, entropy, top_ids, top_logprobs) and the tolerance of each, float64."""
    B, V = x.shape
    n = tokens.shape[1]
    inv_t = np.float64(np.float32(inv_t))
    lp, lse, H = np.zeros((B, n)), np.zeros(B), np.zeros(B)
    ids, tl = np.full((B, top), -1, np.int64), np.full((B, top), -np.inf)
    t_lp, t_lse, t_H, t_tl = np.zeros((B, n)), np.zeros(B), np.zeros(B), np.zeros((B, top))
    for b in range(B):
        row = x[b].astype(np.float64)
        m = np.max(row)
        bad = np.isnan(row).any() or m == np.inf
        real = (tokens[b] >= 0) & (tokens[b] < V)
        k = min(top, V)
        ids[b, :k] = order(x[b])[:k]
        if bad:
            lse[b] = H[b] = np.nan
            lp[b] = np.where(real, np.nan, 0.0)
            tl[b, :k] = np.nan
            continue
        if m == -np.inf:
            lse[b], H[b] = -np.inf, 0.0
            lp[b] = np.where(real, -np.inf, 0.0)
            continue
        y = (row - m) * inv_t
        e = np.exp(y)
        S = e.sum()
        kept = e > 0
        mean = (e[kept] * y[kept]).sum() / S
        logp = y - np.log(S)
        lse[b], H[b] = m * inv_t + np.log(S), np.log(S) - mean
        lp[b] = np.where(real, logp[np.where(real, tokens[b], 0)], 0.0)
        tl[b, :k] = logp[ids[b, :k]]
        of_sum = U * (adds(V) + 4 * abs(mean) + 4 * np.log(S))
        with np.errstate(invalid="ignore"):
            t_lp[b] = of_sum + 6 * U * np.abs(lp[b])
            t_tl[b] = of_sum + 6 * U * np.abs(tl[b])
        t_lse[b] = of_sum + 4 * U * (abs(lse[b]) + abs(m * inv_t))
        second = (e[kept] * y[kept] ** 2).sum() / S
        t_H[b] = 2 * of_sum + U * (2 * adds(V) * abs(mean) + 8 * second + 8 * abs(H[b]))
    limit = np.float64(np.finfo(np.float32).max)
    lp, lse, tl = (np.where(v > limit, np.inf, np.where(v < -limit, -np.inf, v)) for v in (lp, lse, tl))
    return (lp, lse, H, ids, tl), (t_lp, t_lse, t_H, None, t_tl)


def gradient(x, tokens, inv_t, stats, H, g, g_lse, g_H, bf16=False):
    """The gradient and its tolerance, float64; stats (largest logit, log S) and H as given."""
    B, V = x.shape
    inv_t = np.float64(np.float32(inv_t))
    d, tol = np.zeros((B, V)), np.zeros((B, V))
    for b in range(B):
        row = x[b].astype(np.float64)
        m, ln_s = np.float64(stats[b, 0]), np.float64(stats[b, 1])
        if m == -np.inf:
            continue
        if np.isnan(m) or np.isnan(ln_s):
            d[b] = np.nan
            continue
        y = (row - m) * inv_t - ln_s
        p = np.exp(y)
        yp = np.where(p > 0, y, 0.0)
        real = (tokens[b] >= 0) & (tokens[b] < V)
        gj = np.where(real, g[b].astype(np.float64), 0.0)
        share = np.float64(g_lse[b]) - gj.sum()
        inner = share - np.float64(g_H[b]) * (yp + np.float64(H[b]))
        size = abs(np.float64(g_lse[b])) + np.abs(gj).sum() + abs(np.float64(g_H[b])) * (np.abs(yp) + abs(H[b]))
        d[b] = p * inner
        tol[b] = p * size * U * (8 * np.abs(yp) + 4 * ln_s + 16 + gj.size)
        np.add.at(d[b], tokens[b][real], gj[real])
        np.add.at(tol[b], tokens[b][real], (4 + gj.size) * U * np.abs(gj[real]))
        d[b] *= inv_t
        tol[b] *= inv_t
        tol[b] += 2 * U * np.abs(d[b]) + 2.0 ** -126   # results below the normal range may vanish
        if bf16:
            tol[b] = tol[b] * 1.01 + 2.0 ** -8 * np.abs(d[b]) + 2.0 ** -126
    return d, tol


def weights(codes, scales):
    """float64 weights [V, K] of packed codes and scales."""
    q = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1).astype(np.float64) - 8.0
    return q * np.repeat(scales.astype(np.float64), q.shape[1] // scales.shape[1], axis=1)


def head(hidden, codes, scales, bf16=False):
    h = hidden.astype(np.float64)
    out = h @ weights(codes, scales).T
    K = h.shape[1]
    size = np.abs(h) @ np.repeat(np.abs(scales.astype(np.float64)), K // scales.shape[1], axis=1).T
    tol = U * 136 * size
    if bf16:
        tol = tol + 2.0 ** -8 * np.abs(out)
    return out, tol
