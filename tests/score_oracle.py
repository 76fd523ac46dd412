"""Plain 64-bit forms of the operators over logits and verdicts, row by row, for the tests.  Nothing of the library is used."""
import numpy as np


def closed_entries(V, words=None, width=1):
    """Truth values [V]: entry i is closed if one of i .. i + width - 1 is occupied or not below V."""
    taken = [False] * V
    if words is not None:
        taken = [bool((int(words[i >> 5]) >> (i & 31)) & 1) for i in range(V)]
    w = max(1, int(width))
    return np.array([i + w > V or any(taken[i:i + w]) for i in range(V)])


def score_row(x, scale, closed, token, top):
    """(ln p of the token, entropy, M, L, ids, ln p of them) of one row in 64 bits; token None: no token; x: float64 values."""
    V = len(x)
    none = ([-1] * top, [-np.inf] * top)
    if token is not None and not 0 <= token < V:
        return (0.0, 0.0, 0.0, 0.0) + none
    at = np.flatnonzero(~closed)
    z = x[at]
    if len(z) == 0 or np.all(z == -np.inf):
        return (-np.inf, 0.0, -np.inf, -np.inf) + none
    M = z.max()
    d = (z - M) * scale
    e = np.exp(d)
    s = e.sum()
    L = np.log(s)
    p = e / s
    with np.errstate(invalid="ignore"):
        H = -np.sum(np.where(p > 0, p * (d - L), 0.0))
    lp = -np.inf if token is None or closed[token] else (x[token] - M) * scale - L
    order = sorted((i for i in at if x[i] > -np.inf), key=lambda i: (-x[i], i))[:top]
    ids = list(order) + [-1] * (top - len(order))
    lps = [(x[i] - M) * scale - L for i in order] + [-np.inf] * (top - len(order))
    return lp, H, M, L, ids, lps


def grad_row(x, scale, closed, token, g, h):
    """Gradient of g ln p[token] + h entropy to the row, in 64 bits."""
    V = len(x)
    out = np.zeros(V)
    if token is not None and not 0 <= token < V:
        return out
    _, H, M, L, _, _ = score_row(x, scale, closed, token, 0)
    if L == -np.inf:
        return out
    if token is None or closed[token]:
        g = 0.0
    l = np.where(closed | (x == -np.inf), -np.inf, (np.where(closed, 0.0, x) - M) * scale - L)
    p = np.exp(l)
    with np.errstate(invalid="ignore"):
        out = -np.where(p > 0, p * (g + h * (l + H)), 0.0)
    if token is not None:
        out[token] += g
    return out * scale


def advantages(verdicts, pair_cost, bank_cost, normalise, eps):
    """verdicts: one int array [samples, 4] per program."""
    out = []
    for v in verdicts:
        r = np.array([float(int(f) & 1) - pair_cost * (int(c) & 0xFFFFFFFF) - bank_cost * (int(b) & 0xFFFFFFFF) for f, _, c, b in v])
        if len(r):
            c = r - r.mean()
            if r.max() == r.min():
                c = np.zeros_like(c)
            out.append(c / (np.sqrt(np.mean(c * c)) + eps) if normalise else c)
    return np.concatenate(out) if out else np.zeros(0)


def policy(verdicts, off, lp, old=None, ref=None, pair_cost=0.0, bank_cost=0.0, normalise=True, eps=1e-6, clip_lo=0.2, clip_hi=0.2,
           kl=0.0, per_token=False):
    """(loss, advantages, derivative to lp, sum of the absolute values of the loss's terms), token by token."""
    adv = advantages(verdicts, pair_cost, bank_cost, normalise, eps)
    N, T = len(adv), len(lp)
    g, terms = np.zeros(T), []
    old = lp if old is None else old
    for c in range(N):
        for t in range(int(off[c]), int(off[c + 1])):
            w = 1.0 / (off[N] - off[0]) if per_token else 1.0 / (N * (off[c + 1] - off[c]))
            if -np.inf in (lp[t], old[t]) or (kl and ref[t] == -np.inf):
                continue
            r, A = np.exp(lp[t] - old[t]), adv[c]
            lo, hi = 1.0 - clip_lo, 1.0 + clip_hi
            cut = min(max(r, lo), hi)
            term = -min(r * A, cut * A)
            slope = 0.0 if (A > 0 and r > hi) or (A < 0 and r < lo) else -r * A
            if kl:
                q = ref[t] - lp[t]
                term += kl * (np.expm1(q) - q)
                slope -= kl * np.expm1(q)
            terms.append(w * term)
            g[t] = w * slope
    return float(np.sum(terms)), adv, g, float(np.sum(np.abs(terms)))
