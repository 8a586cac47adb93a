"""The operators that make a retained set, in 64 bits from their definitions: attention over
prompts, its weights per key, eviction by accumulated weight.  Plain numpy, none of the package's
code."""
import numpy as np


def sees(n, m, window=0, n_sink=0):
    """[n, m]: which keys each token sees."""
    at = (m - n + np.arange(n))[:, None]
    j = np.arange(m)[None, :]
    yes = j <= at
    if window > 0:
        yes &= (at - j < window) | (j < n_sink)
    return yes


def score_error(q, k, scale):
    """How far a float32 score scale q . k may be off [n, m]: d additions and a product, each within
    2^-24 of terms that sum to |q| . |k|, and as much again where a tensor core truncates."""
    d = q.shape[-1]
    return (d + 4) * 2.0 ** -23 * scale * (np.abs(q) @ np.abs(k).T) + 2.0 ** -21


def attend(q, k, v, scale, window=0, n_sink=0):
    """One sequence, one query head: q [n, d], k and v [m, d].  Returns out, lse and how far each may
    be off:
      2^-8 p |v|     a probability is rounded to bf16 (8 bits) for its product
      2^-8 |out|     so is the output
      2 e p |v|      scores off by e change a probability and the denominator by that much each
      m 2^-22 p |v|  float32 sums over m keys, twice (numerator, denominator), 2^-23 a step, and
                     as many steps again for the factors of running maxima
    and for lse e, the sum's m 2^-23 and its own rounding."""
    n, d = q.shape
    m = k.shape[0]
    out, lse = np.zeros((n, d)), np.full(n, -np.inf)
    off, off_lse = np.zeros((n, d)), np.zeros(n)
    if n == 0 or m == 0:
        return out, lse, off, off_lse
    see = sees(n, m, window, n_sink)
    err = score_error(q, k, scale)
    for i in range(n):
        on = see[i]
        if not on.any():
            continue
        x = k[on] @ q[i] * scale
        top = x.max()
        p = np.exp(x - top)
        lse[i] = top + np.log(p.sum())
        p /= p.sum()
        e = err[i, on].max()
        out[i] = p @ v[on]
        size = p @ np.abs(v[on])
        off[i] = (2.0 ** -8 * (size + np.abs(out[i])) + (2 * e + (m + 8) * 2.0 ** -22) * size
                  + 1e-30)
        off_lse[i] = e + (m + 8) * 2.0 ** -23 + np.abs(lse[i]) * 2.0 ** -23
    return out, lse, off, off_lse


def weights(q, k, lse, scale, window=0, n_sink=0, last=0):
    """Sums at the keys of one sequence over one query head's tokens, and how far they may be off: a
    weight by its score's error and the rounding of the difference, the sum by 2^-24 a step."""
    n, m = q.shape[0], k.shape[0]
    if n == 0 or m == 0:
        return np.zeros(m), np.zeros(m)
    see = sees(n, m, window, n_sink)
    if last > 0:
        see[:max(0, n - last)] = False
    x = q @ k.T * scale
    w = np.where(see, np.exp(np.where(see, x - lse[:, None], 0.0)), 0.0)
    e = (score_error(q, k, scale) + 2.0 ** -22 * (np.abs(x) + np.abs(np.where(see, lse[:, None], 0))))
    return w.sum(0), (w * e).sum(0) + (n + 2) * 2.0 ** -23 * w.sum(0)


def policy(score, length, budget, n_sink, n_recent):
    """Mask and kept scores of one unit."""
    N = len(score)
    mask, kept = np.zeros(N, np.uint8), np.zeros(N, np.float32)
    if not (0 <= budget <= N and 0 <= length <= N):
        return mask, kept, 1
    at = np.arange(length)
    free = (at >= n_sink) & (at < length - n_recent)
    x = score[:length].astype(np.float64)
    nan = np.isnan(x)
    rank = np.where(~free, 0, np.where(nan, 2, 1))
    order = np.lexsort((at, np.where(rank == 1, -np.where(nan, 0, x), 0.0), rank))
    chosen = np.sort(order[:budget])
    mask[chosen] = 1
    kept[:len(chosen)] = score[chosen]
    return mask, kept, 0
