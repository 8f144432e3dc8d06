"""Random numbers next to the borders between two tokens' shares of a row: what weights that are a little off would draw otherwise.

The library's weights are good to 2^-32 of their value (dark.h), and sums of what is not negative to no more than that, beside some 2^-48 for the roundings of sums in 64 bits.  A
border is a quotient of two such sums: it is off by 2^-31 of itself at most.  So a random number that is farther than 2^-30 from every border draws the oracle's token, without an
exception; and the logarithm of the token's share is off by 2^-31 beside its rounding to 32 bits, 2^-24 of its value.
"""
import numpy as np

from oracle import sample_oracle as S

NEAR = 2.0 ** -30


def log_tolerance(log):
    return 2.0 ** -30 + 2.0 ** -24 * np.abs(log)


def next_to_borders(x, n, **kw):
    """For a row x in fp64 and its settings: the n numbers of 32 bits that lie closest to a border, but farther than NEAR from it; the tokens that they draw, and the
    logarithms of their shares."""
    w = S.kept(x, **{**dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0), **kw})
    at = np.nonzero(w)[0]
    sums = np.cumsum(w[at]) / w[at].sum()
    borders = sums[:-1][(sums[:-1] > 2.0 ** -6) & (sums[:-1] < 1.0 - 2.0 ** -20)]
    near = borders.astype(np.float32)
    u = np.unique(np.concatenate([near, np.nextafter(near, np.float32(0)), np.nextafter(near, np.float32(1))]))
    i = np.searchsorted(sums, u.astype(np.float64))
    gap = np.minimum(np.abs(sums[np.minimum(i, sums.size - 1)] - u), np.abs(sums[np.maximum(i - 1, 0)] - u))
    u = u[gap > NEAR][np.argsort(gap[gap > NEAR])[:n]]
    i = np.searchsorted(sums, u.astype(np.float64), side="right")
    return u, at[i], np.log(w[at[i]] / w[at].sum()), np.sort(gap[gap > NEAR])[:n]
