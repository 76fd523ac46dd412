"""The loss over verdicts where ratios, sizes and offsets reach their limits, against the plain 64-bit form.

Tolerances.  u = 2^-24, d = lp - old.  Where |d| >= 0.35 the kernel's rho is exp d itself: d is rounded (|d| u of rho), so are its product with
log2 e and that constant (1.3 |d| u together), and the exponential is within 2^-22 = 4 u; the derivative rounds the weight and the product:
(6 + 3 |d|) u of its value in all.  Nearer to 0 exp d - 1 comes from a series in multiply-adds, within 4 u of its value, which is below 0.42, and rho
is rounded once more: less than the same.  A sum of four terms of one sign adds 3 u, the loss is rounded once.
"""
import numpy as np
import pytest

from tests import score_oracle as ref
from tests.test_gpu_policy import U, B, _dev  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,n", [(2, 65), (2, 3000), (400, 90)])
@pytest.mark.parametrize("span", [(-40.0, -8.0), (-17.5, -16.0), (-3.0, -0.2)])
def test_small_ratios_keep_their_digits(B, N, n, span):
    """Under a positive advantage small ratios are not clipped: the derivative is as exact relative to its own value, and the loss too, where
    only such tokens add to it (the candidates of a negative one own none)."""
    rng = np.random.default_rng(n)
    v = np.zeros((N, 4), dtype=np.int64)
    v[:, 0] = np.where(np.arange(N) % 2 == 0, 1, 2)
    off = np.concatenate([[0], np.cumsum(np.where(np.arange(N) % 2 == 0, n, 0))])
    T = int(off[-1])
    old = np.full(T, -0.5, dtype=np.float32)
    lp = (old + rng.uniform(*span, T)).astype(np.float32)
    outs, o, l, ol = _dev([v], off, lp, old)
    d = np.abs(lp.astype(float) - old)
    for per_token in (False, True):
        loss, _, g = B.vl_policy_loss(outs, o, l, ol, per_token=per_token)
        want_loss, _, want, _ = ref.policy([v], off, lp.astype(float), old.astype(float), per_token=per_token)
        bad = np.flatnonzero(~(np.abs(g.double().cpu().numpy() - want) <= (6 + 3 * d) * U * np.abs(want)))
        assert len(bad) == 0, (d[bad[:5]], g[bad[:5].tolist()], want[bad[:5]])
        assert abs(float(loss) - want_loss) <= ((6 + 3 * d) * U * np.abs(want)).sum() + 4 * U * abs(want_loss)


@pytest.mark.parametrize("kw", [dict(eps=1e-100), dict(eps=1e-100, pair_cost=1e-200), dict(pair_cost=1e20, bank_cost=-1e20), dict(pair_cost=1e20, normalise=False),
                                dict(eps=1e300)], ids=str)
def test_rules_at_the_ends_of_their_range(B, kw):
    """Equal rewards leave exactly nothing, others what the formula says, in numbers.  (Below 2^-126 a 32-bit number is a multiple of 2^-149: a
    rounding there, of an advantage, of a weight or of its product, is off by up to 2^-150 whatever the value.)"""
    import torch
    v = np.array([[1, -1, 0, 0]] * 5 + [[8, 3, 7, 13]] * 5)
    off, lp = np.arange(11) * 3, np.full(30, -1.0, dtype=np.float32)
    lp[::2] = -1.125
    old = np.full(30, -1.0, dtype=np.float32)
    outs, o, l, ol = _dev([v[:5], v[5:]], off, lp, old)
    loss, adv, g = B.vl_policy_loss(outs, o, l, ol, ref_logprob=ol, kl=1e30, **kw)
    assert bool((adv == 0).all()) and bool((g[1::2] == 0).all()) and bool(torch.isfinite(g).all()) and bool(torch.isfinite(loss))
    outs, o, l, ol = _dev([v], off, lp, old)
    loss, adv, g = B.vl_policy_loss(outs, o, l, ol, **kw)
    want_loss, want_adv, want, _ = ref.policy([v], off, lp.astype(float), old.astype(float), **kw)
    assert np.all(np.abs(adv.double().cpu().numpy() - want_adv) <= 2 * U * np.abs(want_adv) + 2.0 ** -150)
    assert np.all(np.abs(g.double().cpu().numpy() - want) <= (6 + 3 * 0.125) * U * np.abs(want) + 2.0 ** -148) and bool(torch.isfinite(loss))
