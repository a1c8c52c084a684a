"""The plain 64-bit definition of sbw_sample_tokens, on the CPU; the noise is the oracle's, which other tests pin.

The token is exact: scores are two fp32 operations.  Where the rounding of sums decides whether a logit is kept either answer
is right: rows are taken with top_p a little smaller and a little larger.  How little: the kernel's sum of all weights is
made as that of the log probabilities is, so off by u (adds + 4 E|y|) of itself, and the sums it is compared with are of V
whole numbers of 2^-30 at most, each off by half of one.  A log probability is off by 4 u |y| from its score, a rounding of
itself, and the weights' sum."""
import numpy as np

import oracle
import step_reference as ref

U = 2.0 ** -24


def noise(V, seed):
    return oracle.gumbel_many(np.arange(V, dtype=np.uint32), np.full(V, seed, np.uint64))


def kept_columns(row, inv_t, top_k, top_p, min_p):
    """Columns that the filters keep, in order."""
    columns = ref.order(row)
    x = row.astype(np.float64)[columns]
    e = np.exp((x - x[0]) * inv_t)
    if 0 < top_k < row.size:
        columns, e = columns[:top_k], e[:top_k]
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(e)[:-1]])
        n = max(1, int((before < top_p * e.sum()).sum()))
        columns, e = columns[:n], e[:n]
    if min_p > 0:
        # x itself at or above the largest plus log(min_p) T
        n = int((x[:columns.size] >= x[0] + np.log(min(min_p, 1.0)) / inv_t).sum())
        columns, e = columns[:max(n, 1)], e[:max(n, 1)]
    return columns, e


def sample(row, seed, inv_t, top_k=0, top_p=1.0, min_p=0.0):
    """[(token, log probability, tolerance)]: one, or two where the sums' rounding decides."""
    inv32 = np.float32(inv_t)
    inv_t, top_p, min_p = float(inv32), float(np.float32(top_p)), float(np.float32(min_p))
    if not (inv_t > 0 and np.isfinite(inv_t)):
        return [(-1, np.nan, 0.0)]
    first = ref.order(row)[0]
    if not np.isfinite(row[first]):
        return [(int(first), -np.inf if row[first] == -np.inf else np.nan, 0.0)]
    with np.errstate(over="ignore", invalid="ignore"):      # -inf times 0 where a weight is 0
        scores = (row * inv32).astype(np.float32) + noise(row.size, seed)
    answers = []
    y_all = (row.astype(np.float64) - float(row[first])) * inv_t
    e_all = np.exp(y_all)
    S = e_all.sum()
    off = U * (ref.adds(row.size) + 4 * (e_all * np.abs(y_all))[e_all > 0].sum() / S) + row.size * 2.0 ** -31 / S
    for p in sorted({top_p, top_p * (1 - off), min(top_p * (1 + off), 1.0)} if 0 < top_p < 1 else {top_p}):
        columns, e = kept_columns(row, inv_t, top_k, p, min_p)
        best = scores[columns].max()
        token = int(columns[scores[columns] == best].min())
        y = (float(row[token]) - float(row[first])) * inv_t
        total = e.sum()
        mean = (e * np.abs((row[columns].astype(np.float64) - float(row[first])) * inv_t))[e > 0].sum() / total
        lp = y - np.log(total)
        answers.append((token, lp, U * (ref.adds(row.size) + 4 * mean + 4 * abs(y) + 4 * np.log(total) + 6 * abs(lp))))
    return answers
