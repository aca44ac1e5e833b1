"""The key/value cache in 64 bits, from its definition: sequences as lists of rows.

Blocks, tables, rings and codes exist here only as what they mean: a complete block
stands for its rows rounded to 127ths of its largest element, an incomplete one for
its rows."""
import numpy as np


def rotate(x, place, cos, sin, interleaved):
    """x (..., dim) float32 at a place, rotated in 64 bits and rounded to FP32."""
    if cos is None or not 0 <= place < len(cos):
        return x.copy()
    r = 2 * cos.shape[1]
    y = x.astype(np.float64)
    c, s = cos[place].astype(np.float64), sin[place].astype(np.float64)
    a = slice(0, r, 2) if interleaved else slice(0, r // 2)
    b = slice(1, r, 2) if interleaved else slice(r // 2, r)
    u, w = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = u * c - w * s, w * c + u * s
    return y.astype(np.float32)


def codes(rows):
    """Round(127 x / m) of one head's rows, ties to even, and m."""
    m = np.abs(rows).max() if rows.size else np.float32(0)
    if not m > 0:
        return np.zeros(rows.shape), np.float64(m)
    return np.rint(127.0 * rows.astype(np.float64) / np.float64(m)), np.float64(m)


class Sequence:
    """Rows (tokens, heads, dim) of keys and values, FP32."""

    def __init__(self, heads, dim, block):
        self.block = block
        self.k = np.zeros((0, heads, dim), np.float32)
        self.v = np.zeros((0, heads, dim), np.float32)

    def append(self, k, v, cos=None, sin=None, interleaved=False):
        n = len(self.k)
        k = [rotate(x, n + i, cos, sin, interleaved) for i, x in enumerate(k)]
        self.k = np.concatenate([self.k, np.stack(k)]) if k else self.k
        self.v = np.concatenate([self.v, v])

    def cut(self, n):
        self.k, self.v = self.k[:n], self.v[:n]

    def block_codes(self, b, which):
        """(codes, m) of complete block b: (block, heads, dim) and (heads)."""
        x = getattr(self, which)[b * self.block:(b + 1) * self.block]
        out = [codes(x[:, h]) for h in range(x.shape[1])]
        return np.stack([c for c, _ in out], 1), np.array([m for _, m in out])

    def values(self, which):
        """What the cache stands for: (tokens, heads, dim) float64."""
        x = getattr(self, which).astype(np.float64)
        for b in range(len(x) // self.block):
            c, m = self.block_codes(b, which)
            x[b * self.block:(b + 1) * self.block] = c * m[None, :, None] / 127.0
        return x

    def means(self):
        n = -(-len(self.k) // self.block)
        return np.stack([self.k[b * self.block:(b + 1) * self.block].astype(np.float64).mean(0) for b in range(n)])


def attention(q, K, V, scale, seen):
    """One query head: q (dim), K, V (tokens, dim) float64, seen: how often each token
    counts.  Returns (o, lse, S, A): S bounds the scores' terms, A the output's:
    max over the tokens seen of scale sum |q||k|, and sum p |v|."""
    at = np.nonzero(seen)[0]
    if not len(at):
        return np.zeros(V.shape[1]), -np.inf, 0.0, np.zeros(V.shape[1])
    q = q.astype(np.float64)
    s = scale * (K[at] @ q)
    m = s.max()
    e = np.exp(s - m) * seen[at]
    p = e / e.sum()
    S = abs(scale) * (np.abs(K[at]) @ np.abs(q)).max()
    return p @ V[at], m + np.log(e.sum()), S, p @ np.abs(V[at])


def bound(S, n, dim, q=0.0, k=0.0, v=0.0):
    """(relative to A, absolute of o, absolute of lse): how far FP32 sums of FP16 pairs
    may be off.

    A score's terms are off by 2^-22 (the pair of q) and, in an FP32 row, 2^-22 and
    2^-22 more (its pair, the residuals' product); its sum of 3 dim terms by
    4 sqrt(3 dim) 2^-24 of the terms (roundings as random as their operands, four
    deviations), the scale and the log2 units by 3 * 2^-24 of the score, exp2's
    argument by 2^-24 of it and its result by 2^-23.  A weight's relative error is the
    score's absolute one, twice (numerator and sum); the weights' pairs are off by
    2^-22 and the sums of 3 n terms by 4 sqrt(3 n) 2^-24, at most 32 factors exp2(m - m')
    of 2^-23 each on the way.

    FP16 steps do not go below 2^-24, half of one being 2^-25.  q and k: |scale| max|q|
    sum|k| and its like, the terms that floors meet: rows of q and k are scaled below
    2^14 with their largest element at 2^13 or more, so an element is off by 2^-25 of
    2^13, 2^-38 of the largest.  v: the largest value that is seen.  A weight times a
    block's maximum is below 2^14 where 2^ref <= 2 v meets a weight of 1, and off by
    2^-25 or more: 2^-39 2 v of the product with m, and 2^-38 v for each token; a value
    of an FP32 row is scaled below 2^7 and off by 2^-25, 2^-32 2 v of it.  Below 2^-126
    every rounding to FP32 is off by up to 2^-150: two for each of four waves' sums, their
    join and the division, less than 16 in all."""
    score = S * (3 * 2.0 ** -22 + (4 * np.sqrt(3 * dim) + 8) * 2.0 ** -24) + 2.0 ** -38 * (q + k)
    rel = 2 * score + 2.0 ** -22 + 4 * np.sqrt(3 * n) * 2.0 ** -24 + 40 * 2.0 ** -23
    return rel, (n * 2.0 ** -38 + 2.0 ** -31) * v + 2.0 ** -146, score + 4 * np.sqrt(n) * 2.0 ** -24 + 40 * 2.0 ** -23


def select(q, means, place, block, n_sel, keep_first, keep_last):
    """One token and head: q (queries, dim), means (blocks, dim) float64."""
    nb = place // block + 1 if place >= 0 else 0
    if nb <= n_sel:
        pick = list(range(nb))
    else:
        score = (q.astype(np.float64) @ means[:nb].T).max(0)
        score = np.where(np.isnan(score), -np.inf, score)
        forced = list(range(keep_first)) + list(range(nb - keep_last, nb))
        others = sorted(range(keep_first, nb - keep_last), key=lambda b: (-score[b], b))
        pick = sorted(forced + others[:n_sel - keep_first - keep_last])
    return pick + [-1] * (n_sel - len(pick))
