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


def test_nothing_else_is_written(B):
    """Through the C entry point, with guards around the loss, the advantages, the derivative and the working memory, each in memory of its own:
    offsets that are none lead nowhere, and what is asked for is written whole."""
    import ctypes as C
    import torch
    rng = np.random.default_rng(6)
    lib, mark, G = B._lib, -7.25e33, 64
    for sizes, n in [([30], 20), ([300], 40), ([70, 1, 0, 40], 90), ([3000], 3), ([100, 5], 700)]:
        N = sum(sizes)
        good = np.concatenate([[0], np.cumsum(rng.poisson(n, N))]).astype(np.int64)
        T = int(good[-1]) + 5
        lp, old, rf = (torch.from_numpy((-rng.random(T)).astype(np.float32)).cuda() for _ in range(3))
        v = np.zeros((N, 4), dtype=np.int32)
        v[:, 0] = rng.integers(1, 3, N)
        v[:, 3] = rng.integers(0, 9, N)
        outs = [o.contiguous() for o in torch.from_numpy(v).cuda().split(sizes)]
        ptrs = (C.c_void_p * len(sizes))(*[o.data_ptr() if o.numel() else None for o in outs])
        K = (C.c_uint64 * len(sizes))(*sizes)
        size = lib.vl_policy_work(N, T)
        rules = B.vl_policy_rules(eps=1e-6, clip_lo=0.2, clip_hi=0.2, normalise=1, kl=0.1, bank_cost=0.01)
        bad = [good[::-1].copy(), good - 10 ** 12, good + 10 ** 12, rng.integers(-2 ** 62, 2 ** 62, N + 1), np.full(N + 1, T), np.zeros(N + 1, np.int64)]
        for off in [good] + bad:
            o = torch.from_numpy(off).cuda()
            for want in ((1, 1), (0, 1), (1, 0)):
                bufs = [torch.full((k + 2 * G,), mark, device="cuda") for k in (1, N, T, (size + 3) // 4)]
                p = [b.data_ptr() + 4 * G for b in bufs]
                torch.cuda.synchronize()
                assert lib.vl_policy_loss(0, len(sizes), ptrs, K, o.data_ptr(), T, lp.data_ptr(), old.data_ptr(), rf.data_ptr(), C.byref(rules), p[0],
                                          p[1] if want[0] else None, p[2] if want[1] else None, p[3], size, None) == 0
                torch.cuda.synchronize()
                for b, asked in zip(bufs, (1,) + want + (1,)):
                    assert bool((b[:G] == mark).all()) and bool((b[-G:] == mark).all())
                    assert asked or bool((b == mark).all())
                for b, asked in zip(bufs[:3], (1,) + want):
                    assert not asked or not bool((b[G:-G] == mark).any())
                if off is good and want == (1, 1):
                    first = [b.clone() for b in bufs[:3]]
                    loss, adv, g = B.vl_policy_loss(outs, o, lp, old, ref_logprob=rf, kl=0.1, bank_cost=0.01)
                    assert torch.equal(first[0][G], loss) and torch.equal(first[1][G:-G], adv) and torch.equal(first[2][G:-G], g)
