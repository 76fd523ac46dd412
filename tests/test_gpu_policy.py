"""The loss over verdicts and its derivative: CUDA path against the plain 64-bit form, and the whole training step.

Tolerances.  u = 2^-24.  An advantage is computed in 64 bits and rounded once: u of its value.  A token's term takes exp(d) - 1 in 32
bits (expm1f: at most two steps, and d rounded to 32 bits: |d| u): an error of (4 + 2 |d|) u |rho - 1| + ... <= (6 + 2 |d|) u (1 + rho) |A| w,
the same for the reference's term; sums are in 64 bits.  The loss is within these summed, and u of itself.
"""
import numpy as np
import pytest

from paper_2506_17506_b200 import synth
from tests import score_oracle as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2506_17506_b200 import binding
    return binding


def _verdicts(rng, K, fails=0.3):
    v = np.zeros((K, 4), dtype=np.int64)
    bad = rng.random(K) < fails
    v[:, 0] = np.where(bad, rng.choice([2, 4, 8, 14], K), 1)
    v[:, 1] = np.where(bad, rng.integers(0, 1000, K), -1)
    v[:, 2] = np.where(bad, rng.integers(0, 500, K), 0)
    v[:, 3] = rng.integers(0, 900, K)
    return v


def _case(rng, sizes, mean, lead=0, tail=0):
    N = sum(sizes)
    lens = rng.poisson(mean, N)
    lens[rng.random(N) < 0.1] = 0
    off = lead + np.concatenate([[0], np.cumsum(lens)])
    T = int(off[-1]) + tail
    lp = -rng.exponential(1.5, T).astype(np.float32)
    old = (lp + rng.normal(0, 0.2, T)).astype(np.float32)
    return [_verdicts(rng, k) for k in sizes], off, lp, old, (lp + rng.normal(0, 0.3, T)).astype(np.float32)


def _dev(verdicts, off, lp, *more):
    import torch
    outs = [torch.from_numpy((v & 0xFFFFFFFF).astype(np.uint32).view(np.int32)).cuda() for v in verdicts]
    return (outs, torch.from_numpy(off.astype(np.int64)).cuda(), torch.from_numpy(lp).cuda()) + tuple(
        None if m is None else torch.from_numpy(m).cuda() for m in more)


def _check(got, verdicts, off, lp, old=None, rf=None, **kw):
    f64 = lambda a: None if a is None else a.astype(np.float64)
    loss, adv, g, total = ref.policy(verdicts, off, f64(lp), f64(old), f64(rf), **kw)
    gl, ga, gg = (t.double().cpu().numpy() for t in got)
    eps = kw.get("eps", 1e-6)
    scale = np.abs(adv).max() if len(adv) else 0.0
    assert np.all(np.abs(ga - adv) <= U * np.abs(adv) * 1.01 + 1e-11 * (scale + 1.0) / min(1.0, eps * 1e6))
    with np.errstate(invalid="ignore"):
        d = np.zeros(len(lp)) if old is None else np.where(np.isfinite(lp) & np.isfinite(old), lp.astype(float) - old, 0.0)
        q = np.zeros(len(lp)) if rf is None else np.where(np.isfinite(lp) & np.isfinite(rf), rf.astype(float) - lp, 0.0)
    N = len(adv)
    w, A = np.zeros(len(lp)), np.zeros(len(lp))
    for c in range(N):
        s = slice(int(off[c]), int(off[c + 1]))
        w[s] = 1.0 / (off[N] - off[0]) if kw.get("per_token") else 1.0 / (N * max(1, off[c + 1] - off[c]))
        A[s] = np.abs(adv[c])
    kl = abs(kw.get("kl", 0.0))
    tol = w * ((6 + 2 * np.abs(d)) * U * (1 + np.exp(d)) * A + kl * (6 + 2 * np.abs(q)) * U * (1 + np.exp(q)))
    assert np.all(np.abs(gg - g) <= 1.01 * tol + 2 * U * np.abs(g)), np.flatnonzero(~(np.abs(gg - g) <= tol + 2 * U * np.abs(g)))[:5]
    assert abs(float(gl) - loss) <= tol.sum() + U * abs(loss) + 1e-13 * total


@pytest.mark.parametrize("sizes,mean", [([1], 5), ([2], 1), ([100], 113), ([7, 1, 300], 40), ([33] * 230, 3), ([5000], 2), ([1200, 900], 9),
                                        ([3], 9000), ([1, 1, 1], 700), ([100] * 20, 60), ([40], 0.3), ([500, 0, 1, 523], 31), ([1023, 1], 20)])
@pytest.mark.parametrize("kw", [dict(), dict(normalise=False, pair_cost=0.01, bank_cost=0.001, per_token=True),
                                dict(pair_cost=0.002, kl=0.1, clip_lo=0.1, clip_hi=0.4), dict(per_token=True, kl=-0.05, clip_lo=1.5, clip_hi=float("inf"))],
                         ids=["plain", "costs", "reference", "unclipped"])
def test_loss_and_derivative(B, sizes, mean, kw):
    rng = np.random.default_rng(sum(sizes) + int(mean * 10))
    v, off, lp, old, rf = _case(rng, sizes, mean, lead=int(rng.integers(0, 9)), tail=int(rng.integers(0, 2100)))
    outs, o, l, ol, r = _dev(v, off, lp, old, rf)
    got = B.vl_policy_loss(outs, o, l, ol, ref_logprob=r, **kw)
    _check(got, v, off, lp, old, rf, **kw)
    again = B.vl_policy_loss(outs, o, l, ol, ref_logprob=r, **kw)
    assert all(bool((a == b).all()) for a, b in zip(got, again))


def test_first_step_has_no_old_scores(B):
    rng = np.random.default_rng(1)
    v, off, lp, _, _ = _case(rng, [50, 20], 30)
    outs, o, l = _dev(v, off, lp)
    _check(B.vl_policy_loss(outs, o, l, bank_cost=0.01), v, off, lp, bank_cost=0.01)


def test_programs_without_samples_and_nothing_at_all(B):
    import torch
    rng = np.random.default_rng(2)
    v, off, lp, old, _ = _case(rng, [4, 0, 3, 0], 6)
    outs, o, l, ol = _dev(v, off, lp, old)
    _check(B.vl_policy_loss(outs, o, l, ol), v, off, lp, old)
    loss, adv, g = B.vl_policy_loss([], torch.zeros(1, dtype=torch.int64, device="cuda"), l)
    assert loss.item() == 0.0 and adv.numel() == 0 and bool((g == 0).all())
    loss, adv, g = B.vl_policy_loss(outs, torch.zeros(8, dtype=torch.int64, device="cuda"), l[:0])
    assert loss.item() == 0.0 and adv.numel() == 7 and g.numel() == 0


@pytest.mark.parametrize("K", [1, 3, 10, 1000, 3001])
def test_equal_rewards_give_no_signal(B, K):
    """Costs whose products are no exact numbers: rewards that are equal leave advantages of exactly 0."""
    v = np.tile(np.array([[8, 3, 7, 13]]), (K, 1))
    off = np.arange(K + 1) * 2
    lp = np.full(2 * K, -0.7, dtype=np.float32)
    outs, o, l = _dev([v], off, lp)
    loss, adv, g = B.vl_policy_loss(outs, o, l, pair_cost=0.1, bank_cost=0.3)
    assert loss.item() == 0.0 and bool((adv == 0).all()) and bool((g == 0).all())


def test_ratios_beyond_the_range_of_numbers(B):
    """They are cut for a positive advantage, large for a negative one, and nothing for none."""
    import torch
    v = np.array([[1, -1, 0, 0], [2, 0, 0, 0]])
    off, lp, old = np.array([0, 2, 4]), np.full(4, -1.0, dtype=np.float32), np.array([-300, -1, -300, -1], dtype=np.float32)
    outs, o, l, ol = _dev([v], off, lp, old)
    loss, adv, g = B.vl_policy_loss(outs, o, l, ol)
    assert adv[0] > 0 and g[0] == 0 and g[2] > 1e34 and bool(torch.isfinite(g).all()) and bool(torch.isfinite(loss))
    outs, o, l, ol = _dev([v[:1], v[:1]], off, lp, old)       # programs of one sample each
    loss, adv, g = B.vl_policy_loss(outs, o, l, ol, ref_logprob=l, kl=0.1)
    assert bool((adv == 0).all()) and bool((g == 0).all()) and loss.item() == 0.0


def test_counts_of_32_bits(B):
    rng = np.random.default_rng(4)
    v = _verdicts(rng, 40)
    v[:, 2] = rng.integers(0, 2 ** 32, 40)
    v[:, 3] = rng.integers(0, 2 ** 32, 40)
    off = np.arange(41) * 3
    lp = -rng.random(120).astype(np.float32)
    outs, o, l = _dev([v], off, lp)
    _check(B.vl_policy_loss(outs, o, l, pair_cost=1e-9, bank_cost=1e-9), [v], off, lp, pair_cost=1e-9, bank_cost=1e-9)


def test_impossible_tokens_and_no_numbers(B):
    import torch
    rng = np.random.default_rng(5)
    v, off, lp, old, rf = _case(rng, [30], 50)
    lp[::7] = -np.inf
    old[::5] = -np.inf
    rf[::11] = -np.inf
    outs, o, l, ol, r = _dev(v, off, lp, old, rf)
    _check(B.vl_policy_loss(outs, o, l, ol, ref_logprob=r, kl=0.1), v, off, lp, old, rf, kl=0.1)
    l2 = l.clone()
    l2[3] = float("nan")
    loss, _, g = B.vl_policy_loss(outs, o, l2, ol)
    assert torch.isnan(loss) and torch.isnan(g[3]) and int(torch.isnan(g).sum()) == 1


def test_ratios_next_to_the_clip(B):
    """Steps of one unit in the last place around the borders: the side is the 64-bit one's."""
    n = 400
    v = np.array([[1, -1, 0, 0], [2, 0, 0, 0]])
    off = np.array([0, 2 * n, 4 * n])
    lp = np.zeros(4 * n, dtype=np.float32)
    lp[:] = -1.0
    hi, lo = np.float32(-1.0 - np.log(1.2)), np.float32(-1.0 - np.log(0.8))
    steps = np.arange(-n // 2, n - n // 2)
    near = np.concatenate([hi + steps * np.spacing(hi), lo + steps * np.spacing(lo)]).astype(np.float32)
    old = np.concatenate([near, near])
    outs, o, l, ol = _dev([v], off, lp, old)
    _, _, g = B.vl_policy_loss(outs, o, l, ol)
    _, _, want, _ = ref.policy([v], off, lp.astype(float), old.astype(float))
    assert np.array_equal(g.cpu().numpy() != 0, want != 0)


def test_offsets_that_are_no_ranges(B):
    """Offsets that fall, or leave the tokens, are followed nowhere: every read and write stays inside."""
    import torch
    rng = np.random.default_rng(6)
    v, off, lp, old, _ = _case(rng, [30], 20)
    for bad in (off[::-1].copy(), off - 10 ** 12, off + 10 ** 12, rng.integers(-2 ** 62, 2 ** 62, 31)):
        outs, o, l, ol = _dev(v, bad, lp, old)
        loss, adv, g = B.vl_policy_loss(outs, o, l, ol)
        torch.cuda.synchronize()
        assert g.numel() == len(lp)


def test_derivative_against_differences(B):
    rng = np.random.default_rng(7)
    kw = dict(pair_cost=0.01, bank_cost=0.002, kl=0.2)
    v, off, lp, old, rf = _case(rng, [6, 5], 7)
    outs, o, l, ol, r = _dev(v, off, lp, old, rf)
    _, _, g = B.vl_policy_loss(outs, o, l, ol, ref_logprob=r, **kw)
    g = g.double().cpu().numpy()
    f64 = [a.astype(np.float64) for a in (lp, old, rf)]
    for t in range(len(lp)):
        if min(abs(f64[0][t] - f64[1][t] - np.log(b)) for b in (0.8, 1.2)) < 1e-5:
            continue
        at = []
        for s in (1e-6, -1e-6):
            p = f64[0].copy()
            p[t] += s
            at.append(ref.policy(v, off, p, f64[1], f64[2], **kw)[0])
        # third derivatives times 1e-12 / 6, and the rounding of sums of about one: 1e-15 / 1e-6; the kernel's own: 32 u
        want = (at[0] - at[1]) / 2e-6
        assert abs(g[t] - want) <= 1e-8 + 32 * U * abs(want), (t, g[t], want)


@pytest.mark.parametrize("mean", [20, 300])
def test_streams_graphs_and_two_calls_at_once(B, mean):
    import torch
    rng = np.random.default_rng(8)
    v, off, lp, old, rf = _case(rng, [100, 50], mean)
    outs, o, l, ol, r = _dev(v, off, lp, old, rf)
    l2 = ol.clone()
    want = [B.vl_policy_loss(outs, o, x, ol, ref_logprob=r, kl=0.1) for x in (l, l2)]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        got = [B.vl_policy_loss(outs, o, x, ol, ref_logprob=r, kl=0.1, stream=s) for x, s in ((l, s1), (l2, s2))]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for p, q in zip(want, got) for a, b in zip(p, q))
    x = l.clone()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s1):
            out = B.vl_policy_loss(outs, o, x, ol, ref_logprob=r, kl=0.1)
        graphs.append((graph, out))
    for src, w in ((l2, want[1]), (l, want[0])):
        x.copy_(src)
        torch.cuda.synchronize()
        for (graph, _), s in zip(graphs, (s1, s2)):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(w, out))


def test_training_step_over_verified_candidates(B, oracle_mod):
    """Candidates of a program through the verifier, scores of their registers under a model of one logit row per definition with the
    occupied registers masked out, the loss, and its gradient to the logits: against the oracle's verdicts and masks and the 64-bit forms
    throughout, and against differences of the whole chain."""
    import torch
    prog = synth.build_program(synth.shape_tiny(), 0)
    K = 12
    rows, _ = synth.candidate_rows(prog, K, 0.4, 3)
    gp = B.Program(prog)
    gp.vl_liveness()
    cand = torch.from_numpy(rows.view(np.int16)).cuda().view(torch.uint16)
    out = gp.vl_verify(cand)
    op = oracle_mod.OracleProgram(prog)
    lv = op.liveness()
    verdicts = op.verify(lv, rows)
    v64 = np.stack([verdicts[f].astype(np.int64) for f in ("flags", "first_violation_instr", "conflict_pairs", "bank_conflicts")], axis=1)
    assert np.array_equal(B.verdicts_to_numpy(out)["flags"], verdicts["flags"])
    # one row of logits per definition and candidate; the mask of its instruction in the first candidate
    instr = np.repeat(np.arange(prog.n_instrs), prog.instr_n_defs)
    col = np.concatenate([np.arange(prog.instr_op_off[i], prog.instr_op_off[i] + prog.instr_n_defs[i]) for i in range(prog.n_instrs)]).astype(int)
    width = prog.vreg_width[prog.op_vreg[col]]
    D, P = len(col), prog.P
    words = gp.vl_occupied_masks(cand[0], P, words=True)
    occ = op.occupied(lv, rows[0])
    rng = np.random.default_rng(9)
    x = torch.from_numpy(rng.normal(0, 2, (K * D, P)).astype(np.float32)).cuda()
    tokens = torch.from_numpy(np.ascontiguousarray(rows[:, col]).reshape(-1)).cuda()
    which = torch.from_numpy(np.tile(instr, K).astype(np.int32)).cuda()
    widths = torch.from_numpy(np.tile(width, K).astype(np.uint8)).cuda()
    args = dict(occupied=words, mask_rows=which, widths=widths, scale=0.8)
    sc = B.vl_token_logprobs(x, tokens, top=2, **args)
    off = torch.arange(0, K * D + 1, D, device="cuda")
    old = (sc.logprob + 0.05 * torch.randn(K * D, device="cuda")).contiguous()
    kw = dict(bank_cost=0.05, pair_cost=0.01)
    loss, adv, g = B.vl_policy_loss([out], off, sc.logprob, old, **kw)
    h = torch.full((K * D,), -0.01 / (K * D), device="cuda")
    dx = B.vl_token_logprobs_backward(x, tokens, sc.row_stats, g, entropy=sc.entropy, g_entropy=h, **args)
    gp.close()

    x64, old64 = x.double().cpu().numpy(), old.double().cpu().numpy()
    tok = rows[:, col].reshape(-1).astype(int)
    occw = np.zeros((prog.n_instrs, (P + 31) // 32), dtype=np.uint32)
    for i in range(prog.n_instrs):
        for p in np.flatnonzero(occ[i]):
            occw[i, p >> 5] |= np.uint32(1 << (p & 31))
    closed = np.array([ref.closed_entries(P, occw[instr[r % D]], width[r % D]) for r in range(K * D)])
    scale = float(np.float32(0.8))

    def chain(x):
        s = [ref.score_row(x[r], scale, closed[r], tok[r], 0)[:2] for r in range(K * D)]
        l = np.array([a for a, _ in s])
        return ref.policy([v64], off.cpu().numpy(), l, old64, **kw)[0] + float(np.sum([b for _, b in s])) * float(h[0]), l

    total, l64 = chain(x64)
    lp = sc.logprob.double().cpu().numpy()
    real = np.isfinite(l64)
    assert np.array_equal(np.isinf(lp), np.isinf(l64)) and np.all(np.abs(lp[real] - l64[real]) <= 1e-5)
    assert abs(loss.item() + float(h[0]) * sc.entropy.double().sum().item() - total) <= 1e-5 * (1 + abs(total))
    got = dx.double().cpu().numpy()
    assert np.all(got[closed] == 0) and np.abs(got).max() > 0
    for r in rng.integers(0, K * D, 12):
        i = int(rng.integers(0, P)) if tok[r] >= P or not np.isfinite(l64[r]) else tok[r]
        up, down = x64.copy(), x64.copy()
        up[r, i] += 1e-5
        down[r, i] -= 1e-5
        want = (chain(up)[0] - chain(down)[0]) / 2e-5
        # the terms weigh 1 / (K D) ~ 1e-3: the differences' rounding 1e-15 / 1e-5, the kernels' some 100 u of a weight
        if closed[r, i]:
            want = 0.0
        assert abs(got[r, i] - want) <= 1e-8 + 1e-5 * abs(want), (r, i, got[r, i], want)
