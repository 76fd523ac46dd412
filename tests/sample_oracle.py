"""Plain 64-bit forms of drawing a token and of clipping gradients, for the tests.  Nothing of the library is used."""
import math

import numpy as np


def sample_row(x, scale, closed, u, top_k=0, top_p=1.0, min_p=0.0):
    """(token, ln p, ln p under what was kept, entries kept) of one row; x: float64 values, scale and u as the device holds them."""
    if not 0.0 <= u < 1.0:
        return -1, 0.0, 0.0, 0
    at = np.flatnonzero(~closed)
    if np.any(np.isnan(x[at])) or np.any(x[at] == np.inf):
        return -1, math.nan, math.nan, 0
    at = at[x[at] > -np.inf]
    if len(at) == 0:
        return -1, -math.inf, -math.inf, 0
    M = x[at].max()
    z = (x[at] - M) * scale
    w = np.exp(z)
    order = np.lexsort((at, -x[at]))                # largest first, the lowest number first among equals
    ws = w[order]
    n = len(at)
    if top_k:
        n = min(n, top_k)
    if top_p < 1.0:
        sums = np.cumsum(ws[:n])
        n = min(n, int(np.argmax(sums >= top_p * sums[-1])) + 1)
    if min_p > 0.0:
        n = min(n, int((ws >= min_p).sum()))
    kept = np.sort(order[:n])                       # places in `at`, which ascends
    sums = np.cumsum(w[kept])
    T = sums[-1]
    past = sums > u * T
    j = kept[int(np.argmax(past)) if past.any() else int(np.flatnonzero(w[kept] > 0)[-1])]
    return int(at[j]), z[j] - math.log(w.sum()), z[j] - math.log(T), n


def norm(arrays, scale):
    """scale times the root of the sum of squares; arrays: float64."""
    return scale * math.sqrt(math.fsum(float(np.sum(np.square(a), dtype=np.longdouble)) for a in arrays))


def factor(n, max_norm):
    if not math.isfinite(n):
        return 0.0
    return max_norm / n if n > max_norm else 1.0
