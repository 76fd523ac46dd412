"""Log probabilities of tokens with entropy and alternatives, and their gradient: CUDA path against plain 64-bit forms.

Tolerances.  u = 2^-24 is half a step of a 32-bit number.  A row's sums add at most V / 32 terms one after another and a few
more across threads (the smallest kernel gives a row to one warp), each term being within (6 + 2 |d|) u of its value (two roundings
in d = scale (x - M), at most two steps in the exponential): relative error of a sum at most S = (V / 32 + 40 + 2 D) u, where D bounds
|d| of the terms that matter (a term below exp(-D) V counts as nothing: D = 20 + ln V).  Then |L - exact| <= S + 2 u L, the
entropy L - T / s is within 3 S (1 + H), and ln p within S + 3 u (|d| + L).  A gradient's p = exp(l) is within (6 + 2 (|d| + L)) u of
its value relatively, the sum of its two terms within a few u of their size, and the result is rounded once to its type.  A p below
2^-126, the smallest normal number, counts as 0: what it would be multiplied with, times 2^-126, comes on top.
"""
import numpy as np
import pytest

from tests import score_oracle as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = ["f32", "f16", "bf16"]


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2506_17506_b200 import binding
    return binding


def _type(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _rows(values, dtype, pad=0, shift=0):
    """A CUDA matrix view of the given values with rows `pad` entries further apart, starting `shift` entries into its memory; what
    lies between the rows is no number."""
    import torch
    R, V = values.shape
    store = torch.full((shift + R * (V + pad),), float("nan"), dtype=_type(dtype), device="cuda")
    x = store[shift:].view(R, V + pad)[:, :V]
    x.copy_(torch.from_numpy(np.ascontiguousarray(values)))
    return x


def _make(rng, R, V, kind="plain"):
    if kind == "plain":
        x = rng.normal(0, 2.5, (R, V))
        x[np.arange(R), rng.integers(0, V, R)] += rng.uniform(0, 12, R)
    elif kind == "levels":          # many equal logits
        x = rng.integers(-3, 4, (R, V)).astype(float)
        x[x == 0] *= rng.choice([-1.0, 1.0], (x == 0).sum())
    elif kind == "flat":
        x = np.full((R, V), 1.5)
    elif kind == "holes":           # impossible tokens
        x = rng.normal(0, 2.5, (R, V))
        x[rng.random((R, V)) < 0.5] = -np.inf
        x[0] = -np.inf
    elif kind == "rising":          # every entry is better than all in front of it
        x = np.tile(np.linspace(-8, 8, V), (R, 1))
    return x


def _masks(rng, n, V, share):
    W = (V + 31) // 32
    m = np.zeros((n, W), dtype=np.uint32)
    for b in range(32):
        m |= (rng.random((n, W)) < share).astype(np.uint32) << np.uint32(b)
    return m


def _sum_error(V):
    return (V / 32 + 40 + 2 * (20 + np.log(V))) * U


def _check_scores(got, x64, scale, closed, tokens, top):
    """got: TokenLogprobs; x64: [R, V] as the device holds them; closed: [R] of truth values; tokens: list or None."""
    R, V = x64.shape
    S = _sum_error(V)
    ent, stats = got.entropy.cpu().numpy(), got.row_stats.cpu().numpy()
    lp = got.logprob.cpu().numpy() if tokens is not None else None
    for r in range(R):
        want = ref.score_row(x64[r], scale, closed[r], None if tokens is None else int(tokens[r]), top)
        wlp, H, M, L, ids, lps = want
        assert stats[r, 0] == np.float32(M), (r, stats[r], M)
        if np.isfinite(L):
            assert abs(stats[r, 1] - L) <= S + 2 * U * abs(L), (r, stats[r, 1], L)
        else:
            assert stats[r, 1] == L
        assert abs(ent[r] - H) <= 3 * S * (1 + H) and ent[r] >= 0, (r, ent[r], H)
        if tokens is not None:
            if np.isfinite(wlp):
                assert abs(lp[r] - wlp) <= S + 3 * U * (abs(wlp) + 2 * abs(L)) and lp[r] <= 0, (r, lp[r], wlp)
            else:
                assert lp[r] == wlp
        if top:
            assert got.top_ids[r].tolist() == [int(i) for i in ids], r
            for a, b in zip(got.top_logprobs[r].tolist(), lps):
                assert a == b or abs(a - b) <= S + 3 * U * (abs(b) + 2 * abs(L)), (r, a, b)


SIZES = [(3, 1), (5, 2), (4, 7), (33, 16), (9, 31), (6, 32), (7, 33), (5, 63), (5, 64), (4, 100), (9, 128), (3, 255), (17, 256), (5, 257),
         (8, 512), (3, 1000), (2, 1023), (3, 1024), (3, 1025), (2, 2048), (3, 4097), (2, 8191), (1, 20011), (2, 50021), (1, 131075)]


@pytest.mark.parametrize("R,V", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_scores_of_many_sizes(B, dtype, R, V):
    import torch
    rng = np.random.default_rng(V * 3 + R)
    for top, pad, shift, scale, tok in [(0, 0, 0, 1.0, torch.int64), (min(5, V + 1), 3, 1, 0.7, torch.int32), (32, 8, 8, 1.3, torch.int64)]:
        x = _rows(_make(rng, R, V), dtype, pad, shift)
        t = rng.integers(0, V, R)
        got = B.vl_token_logprobs(x, torch.from_numpy(t).to(tok).cuda(), scale=scale, top=top)
        _check_scores(got, x.double().cpu().numpy(), np.float32(scale).astype(float), np.zeros((R, V), bool), t, top)


@pytest.mark.parametrize("kind", ["levels", "flat", "holes", "rising"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_scores_of_equal_impossible_and_sorted_entries(B, dtype, kind):
    import torch
    rng = np.random.default_rng(5)
    for R, V in [(3, 9), (4, 200), (3, 777), (2, 3000), (2, 40013)]:
        x = _rows(_make(rng, R, V, kind), dtype)
        t = rng.integers(0, V, R)
        got = B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), top=32)
        _check_scores(got, x.double().cpu().numpy(), 1.0, np.zeros((R, V), bool), t, 32)


@pytest.mark.parametrize("R,V", [(1, 131075), (3, 70000), (700, 40000), (40, 9000), (5, 1000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_alternatives_crowded_into_few_places(B, dtype, R, V):
    """The best entries are all a power of two apart, or in one run, or all alike: whatever the entries are handed out by, some thread has
    many of the best."""
    import torch
    rng = np.random.default_rng(V)
    t = np.full(R, -1)
    t[:3] = rng.integers(0, V, min(R, 3))
    for period, run in [(4096, 24), (1024, 8), (512, 4), (16384, 64), (V, 400)]:
        vals = rng.normal(-5, 1, (R, V)).astype(np.float32)
        high = np.arange(V) % period < run
        vals[:, high] = rng.normal(5, 1, (R, int(high.sum())))
        if period == V:
            vals[0] = 0.0
        x = _rows(vals, dtype)
        got = B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), top=32)
        head = B.TokenLogprobs(*[v[:3] for v in got])
        n = min(R, 3)
        _check_scores(head, x[:3].double().cpu().numpy(), 1.0, np.zeros((n, V), bool), t[:3], 32)
        assert bool((got.top_ids[3:] == -1).all()) and bool((got.logprob[3:] == 0).all())


@pytest.mark.parametrize("V", [5, 16, 31, 64, 200, 256, 300, 512, 1024, 1500, 9001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_scores_under_masks_and_widths(B, dtype, V):
    """Closed logits hold infinities, no numbers and the type's largest value; some rows have nothing left; some are under no
    mask; widths up to the widest tuple."""
    import torch
    rng = np.random.default_rng(V)
    R, n = 24, 7
    for share, widths, top in [(0.5, None, 4), (0.15, [0, 1, 2, 4, 5, 31], 3), (0.004, [32, 33, 64, 65, 200, 255], 20), (None, [1, 3, 40], 2)]:
        m = None if share is None else _masks(rng, n, V, share)
        if m is not None:
            m[3] = 0xFFFFFFFF
            m[4] = 0
        which = rng.integers(-1, n + 1, R).astype(np.int32)
        which[:3] = [3, 4, -2 ** 31]
        w = None if widths is None else rng.choice(widths, R).astype(np.uint8)
        closed = np.array([ref.closed_entries(V, m[which[r]] if m is not None and 0 <= which[r] < n else None, 1 if w is None else w[r])
                           for r in range(R)])
        vals = _make(rng, R, V)
        fill = rng.choice([np.nan, np.inf, -np.inf, {"f32": 3.4e38, "f16": 65504.0, "bf16": 3.3e38}[dtype]], (R, V))
        x = _rows(np.where(closed, fill, vals), dtype, pad=int(rng.integers(0, 9)))
        t = rng.integers(0, V, R)
        t[5] = 65535
        got = B.vl_token_logprobs(x, torch.from_numpy(t.astype(np.uint16)).cuda(),
                                  occupied=None if m is None else torch.from_numpy(m.view(np.int32)).cuda(),
                                  mask_rows=None if m is None else torch.from_numpy(which).cuda(),
                                  widths=None if w is None else torch.from_numpy(w).cuda(), top=top)
        _check_scores(got, x.double().cpu().numpy(), 1.0, closed, t, top)


def test_masks_by_row_and_without_tokens(B):
    import torch
    rng = np.random.default_rng(2)
    R, V = 10, 130
    m = _masks(rng, R + 2, V, 0.4)
    x = _rows(_make(rng, R, V), "f32")
    got = B.vl_token_logprobs(x, occupied=torch.from_numpy(m.view(np.int32)).cuda(), top=3)
    assert got.logprob is None
    _check_scores(got, x.double().cpu().numpy(), 1.0, np.array([ref.closed_entries(V, m[r]) for r in range(R)]), None, 3)


@pytest.mark.parametrize("V", [40, 3000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_the_lowest_value_and_of_no_numbers(B, dtype, V):
    import torch
    low = {"f32": -3.4028234663852886e38, "f16": -65504.0, "bf16": -3.3895313892515355e38}[dtype]
    vals = np.full((6, V), low)
    vals[1, 7] = 3.0              # one real entry among the type's lowest value
    vals[2, ::2] = -np.inf        # the lowest value among impossible ones
    vals[3] = -np.inf
    vals[4] = np.linspace(-1, 1, V); vals[4, 11] = np.nan
    vals[5] = np.linspace(-1, 1, V); vals[5, 12] = np.inf
    x = _rows(vals, dtype)
    t = np.array([1, 7, 1, 0, 5, 5])
    got = B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), top=2)
    _check_scores(B.TokenLogprobs(got.logprob[:4], got.entropy[:4], got.row_stats[:4], got.top_ids[:4], got.top_logprobs[:4]),
                  x.double().cpu().numpy()[:4], 1.0, np.zeros((4, V), bool), t[:4], 2)
    assert torch.isnan(got.logprob[4]) and torch.isnan(got.entropy[4]) and torch.isnan(got.row_stats[4, 1])
    assert torch.isnan(got.entropy[5]) and got.row_stats[5, 0].item() == np.inf
    dx = B.vl_token_logprobs_backward(x[:4], torch.from_numpy(t[:4]).cuda(), got.row_stats[:4].contiguous(),
                                      torch.ones(4, device="cuda"), entropy=got.entropy[:4].contiguous(), g_entropy=torch.ones(4, device="cuda"))
    assert bool(torch.isfinite(dx.float()).all())
    # the token has all of the probability: g (1 - p) with p = 1 within 6 u, and a few u of the two terms' size in their sum
    assert bool((dx[3] == 0).all()) and float(dx[1].float().abs().max()) <= 16 * U
    assert bool((dx[2, ::2] == 0).all())


def test_logits_far_from_zero(B):
    import torch
    rng = np.random.default_rng(8)
    x = _rows(_make(rng, 4, 5000) + 30000.0, "f32")
    t = rng.integers(0, 5000, 4)
    got = B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), scale=0.25, top=4)
    _check_scores(got, x.double().cpu().numpy(), 0.25, np.zeros((4, 5000), bool), t, 4)


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 50.0, 1e6])
def test_scales_at_the_ends_of_their_range(B, scale):
    import torch
    rng = np.random.default_rng(9)
    scale = float(np.float32(scale))
    for R, V in [(3, 40), (4, 1500), (2, 30011)]:
        vals = _make(rng, R, V)
        vals[0, 3] = -np.inf
        vals[1] = rng.choice([1e30, -1e30, 3e38, -3e38, 2e29], V)      # products with the scale leave the range of numbers
        x = _rows(vals, "f32")
        x64, closed, t = x.double().cpu().numpy(), np.zeros((R, V), bool), rng.integers(0, V, R)
        got = B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), scale=scale, top=3)
        real = [r for r in range(R) if r != 1]
        pick = lambda v: None if v is None else v[real]
        _check_scores(B.TokenLogprobs(*[pick(v) for v in got]), x64[real], scale, closed[real], t[real], 3)
        lp, H, M, L, ids, _ = ref.score_row(x64[1], scale, closed[1], int(t[1]), 3)
        assert got.row_stats[1, 0].item() == np.float32(M) and got.top_ids[1].tolist() == [int(i) for i in ids]
        assert abs(got.row_stats[1, 1].item() - L) <= _sum_error(V) + 2 * U * L and abs(got.entropy[1].item() - H) <= 3 * _sum_error(V) * (1 + H)
        stats, H = _oracle_stats(x64, scale, closed, t)
        g, h = rng.normal(0, 8, R).astype(np.float32), rng.normal(0, 2, R).astype(np.float32)
        dx = B.vl_token_logprobs_backward(x, torch.from_numpy(t).cuda(), stats, torch.from_numpy(g).cuda(), entropy=H,
                                          g_entropy=torch.from_numpy(h).cuda(), scale=scale)
        _check_grad(dx, x64, scale, closed, t, g.astype(float), h.astype(float), "f32")


def test_tokens_that_leave_their_row_out(B):
    import torch
    rng = np.random.default_rng(3)
    V = 70
    t = np.array([0, -1, V - 1, V, 2 ** 31 + 5, -2 ** 40, 2 ** 32])
    x = _rows(_make(rng, len(t), V), "f16")
    got = B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), top=3)
    _check_scores(got, x.double().cpu().numpy(), 1.0, np.zeros((len(t), V), bool), t, 3)


def _grad_tolerance(x64, scale, closed, token, g, h, dtype):
    """Per entry, from the module's comment."""
    lp, H, M, L, _, _ = ref.score_row(x64, scale, closed, token, 0)
    want = ref.grad_row(x64, scale, closed, token, g, h)
    if not np.isfinite(L) or (token is not None and not 0 <= token < len(x64)):
        return want, np.zeros_like(want)
    d = np.where(closed | (x64 == -np.inf), 0.0, (np.where(closed, 0.0, x64) - M) * scale)
    l = d - L
    p = np.where(closed | (x64 == -np.inf), 0.0, np.exp(l))
    size = p * (abs(g) + abs(h) * (np.abs(l) + H))
    tol = size * (12 + 4 * (np.abs(d) + L + H)) * U + p * abs(h) * 4 * U * (np.abs(d) + L + H)
    if token is not None:
        tol[token] += 4 * U * abs(g)
    half = {"f32": U, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
    floor = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}[dtype]
    tiny = 2.0 ** -126 * scale * (abs(g) + abs(h) * (np.abs(l) + H))
    return want, scale * tol * 1.01 + np.abs(want) * half * 1.01 + floor + tiny


def _check_grad(dx, x64, scale, closed, tokens, g, h, dtype):
    got = dx.double().cpu().numpy()
    for r in range(x64.shape[0]):
        want, tol = _grad_tolerance(x64[r], scale, closed[r], None if tokens is None else int(tokens[r]), g[r], h[r], dtype)
        bad = np.flatnonzero(~(np.abs(got[r] - want) <= tol))
        assert len(bad) == 0, (r, bad[:5], got[r][bad[:5]], want[bad[:5]], tol[bad[:5]])
        assert np.all(got[r][closed[r]] == 0)


def _oracle_stats(x64, scale, closed, tokens):
    """Statistics and entropies as a forward call leaves them, rounded from 64 bits."""
    import torch
    rows = [ref.score_row(x64[r], scale, closed[r], None if tokens is None else int(tokens[r]), 0) for r in range(x64.shape[0])]
    stats = torch.tensor([[M, L] for _, _, M, L, _, _ in rows], dtype=torch.float64).float().cuda()
    return stats, torch.tensor([w[1] for w in rows], dtype=torch.float64).float().cuda()


@pytest.mark.parametrize("R,V", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_of_many_sizes(B, dtype, R, V):
    import torch
    rng = np.random.default_rng(V * 5 + R)
    for pad, shift, out_pad, out_shift, scale, ent in [(0, 0, 0, 0, 1.0, False), (3, 1, 3, 1, 0.7, True), (8, 8, 1, 0, 1.3, True)]:
        x = _rows(_make(rng, R, V), dtype, pad, shift)
        x64, closed = x.double().cpu().numpy(), np.zeros((R, V), bool)
        t = rng.integers(0, V, R)
        t[0] = -1 if R > 2 else t[0]
        scale = float(np.float32(scale))
        stats, H = _oracle_stats(x64, scale, closed, t)
        g, h = rng.normal(0, 8, R).astype(np.float32), rng.normal(0, 2, R).astype(np.float32) * ent
        out = _rows(np.full((R, V), 7.0), dtype, out_pad, out_shift)
        dx = B.vl_token_logprobs_backward(x, torch.from_numpy(t).cuda(), stats, torch.from_numpy(g).cuda(), entropy=H if ent else None,
                                          g_entropy=torch.from_numpy(h).cuda() if ent else None, scale=scale, out=out)
        _check_grad(dx, x64, scale, closed, t, g.astype(float), h.astype(float), dtype)
        if out_pad and R > 1:           # what lies between the rows is left as it was
            gap = out.as_strided((R - 1, out_pad), (V + out_pad, 1), out.storage_offset() + V)
            assert bool(torch.isnan(gap.float()).all())


@pytest.mark.parametrize("V", [5, 31, 64, 256, 300, 512, 1024, 1500, 9001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_under_masks_and_widths(B, dtype, V):
    import torch
    rng = np.random.default_rng(V + 1)
    R, n = 16, 5
    for share, widths in [(0.5, None), (0.1, [0, 1, 2, 4, 31]), (0.004, [33, 64, 255])]:
        m = _masks(rng, n, V, share)
        m[3] = 0xFFFFFFFF
        which = rng.integers(-1, n + 1, R).astype(np.int32)
        which[0] = 3
        w = None if widths is None else rng.choice(widths, R).astype(np.uint8)
        closed = np.array([ref.closed_entries(V, m[which[r]] if 0 <= which[r] < n else None, 1 if w is None else w[r]) for r in range(R)])
        x = _rows(np.where(closed, rng.choice([np.nan, np.inf, -np.inf], (R, V)), _make(rng, R, V)), dtype)
        x64 = x.double().cpu().numpy()
        t = rng.integers(0, V, R)
        t[2] = 65535
        stats, H = _oracle_stats(x64, 1.0, closed, t)
        g, h = rng.normal(0, 8, R).astype(np.float32), rng.normal(0, 2, R).astype(np.float32)
        dx = B.vl_token_logprobs_backward(x, torch.from_numpy(t.astype(np.uint16)).cuda(), stats, torch.from_numpy(g).cuda(), entropy=H,
                                          g_entropy=torch.from_numpy(h).cuda(), occupied=torch.from_numpy(m.view(np.int32)).cuda(),
                                          mask_rows=torch.from_numpy(which).cuda(), widths=None if w is None else torch.from_numpy(w).cuda())
        _check_grad(dx, x64, 1.0, closed, t, g.astype(float), h.astype(float), dtype)


@pytest.mark.parametrize("V", [12, 300, 2500])
def test_gradient_against_differences(B, V):
    """Central differences of the 64-bit scores: with steps of 1e-4 their own error is below 1e-7 of the values here (third
    derivatives of ln p and entropy times scale^3, at most ~ 10 ln V, times 1e-8 / 6, and 1e-16 |f| / 1e-4)."""
    import torch
    rng = np.random.default_rng(V)
    m = _masks(rng, 1, V, 0.3 if V > 100 else 0.1)
    closed = ref.closed_entries(V, m[0], 2)
    x = _rows(_make(rng, 1, V), "f32")
    x64 = x.double().cpu().numpy()[0]
    tok = int(np.flatnonzero(~closed)[1])
    g, h, scale = 1.5, -0.75, 1.25
    args = dict(occupied=torch.from_numpy(m.view(np.int32)).cuda(), widths=torch.tensor([2], dtype=torch.uint8, device="cuda"), scale=scale)
    t = torch.tensor([tok], device="cuda")
    fwd = B.vl_token_logprobs(x, t, **args)
    dx = B.vl_token_logprobs_backward(x, t, fwd.row_stats, torch.tensor([g], device="cuda"), entropy=fwd.entropy,
                                      g_entropy=torch.tensor([h], device="cuda"), **args)[0].double().cpu().numpy()

    def f(v):
        lp, H, *_ = ref.score_row(v, scale, closed, tok, 0)
        return g * lp + h * H
    S = _sum_error(V)
    for i in np.unique(np.concatenate([rng.integers(0, V, 20), [tok, int(np.argmax(np.where(closed, -np.inf, x64)))]])):
        up, down = x64.copy(), x64.copy()
        up[i] += 1e-4
        down[i] -= 1e-4
        want = (f(up) - f(down)) / 2e-4
        # p is off by the forward call's S as well here
        assert abs(dx[i] - want) <= 2e-7 * np.log(V) + 8 * scale * S * (abs(g) + abs(h) * (np.log(V) + 4)), (i, dx[i], want)


def test_gradient_in_place_and_only_of_the_entropy(B):
    import torch
    rng = np.random.default_rng(4)
    for V in (50, 1030, 20001):
        x = _rows(_make(rng, 5, V), "bf16", pad=5)
        t = torch.from_numpy(rng.integers(0, V, 5)).cuda()
        fwd = B.vl_token_logprobs(x, t)
        g = torch.randn(5, device="cuda")
        want = B.vl_token_logprobs_backward(x, t, fwd.row_stats, g, entropy=fwd.entropy, g_entropy=g)
        only = B.vl_token_logprobs_backward(x, None, fwd.row_stats, entropy=fwd.entropy, g_entropy=g)
        x64 = x.double().cpu().numpy()
        got = B.vl_token_logprobs_backward(x, t, fwd.row_stats, g, entropy=fwd.entropy, g_entropy=g, out=x)
        assert got.data_ptr() == x.data_ptr() and torch.equal(got, want)
        of_entropy, tol = _grad_tolerance(x64[0], 1.0, np.zeros(V, bool), None, 0.0, float(g[0]), "bf16")
        # with the forward call's own statistics: p is off by S more
        more = 4 * _sum_error(V) * abs(float(g[0])) * (4 + np.log(V)) * np.exp(x64[0] - x64[0].max())
        assert np.all(np.abs(only[0].double().cpu().numpy() - of_entropy) <= tol + more)


def test_rows_beyond_32_bits_of_entries(B):
    """The last rows of a matrix of more than 2^32 entries."""
    import torch
    R, V = 33000, 131072
    x = torch.zeros((R, V), dtype=torch.bfloat16, device="cuda")
    x[-1, 5] = 9.0
    x[-2, V - 1] = 4.0
    t = torch.full((R,), -1, dtype=torch.int64, device="cuda")
    t[-2:] = torch.tensor([V - 1, 5], device="cuda")
    got = B.vl_token_logprobs(x, t, top=2)
    tail = B.TokenLogprobs(*[v[-2:] for v in got])
    _check_scores(tail, x[-2:].double().cpu().numpy(), 1.0, np.zeros((2, V), bool), [V - 1, 5], 2)
    assert bool((got.logprob[:-2] == 0).all()) and bool((got.top_ids[:-2] == -1).all())
    g = torch.ones(R, device="cuda")
    B.vl_token_logprobs_backward(x, t, got.row_stats, g, out=x)
    x64 = np.zeros((2, V)); x64[1, 5] = 9.0; x64[0, V - 1] = 4.0
    stats, _ = _oracle_stats(x64, 1.0, np.zeros((2, V), bool), [V - 1, 5])
    for r in range(2):
        want, tol = _grad_tolerance(x64[r], 1.0, np.zeros(V, bool), [V - 1, 5][r], 1.0, 0.0, "bf16")
        p = np.exp(x64[r] - x64[r].max())
        assert np.all(np.abs(x[r - 2].double().cpu().numpy() - want) <= tol + 2 * _sum_error(V) * p)
    assert bool((x[:100] == 0).all())


def test_many_rows_of_which_most_are_left_out(B):
    """More rows than blocks run at once, so that a block goes from row to row: all of them, every third, the last, none."""
    import torch
    rng = np.random.default_rng(12)
    for R, V in [(5000, 2500), (3000, 9000), (2600, 1100)]:
        x = torch.randn(R, V, device="cuda", dtype=torch.bfloat16) * 2
        t = torch.randint(0, V, (R,), device="cuda")
        want = torch.log_softmax(x.double(), dim=1)
        for keep in (slice(None), slice(0, None, 3), slice(R - 1, R), slice(0, 0)):
            u = torch.full((R,), -1, device="cuda")
            u[keep] = t[keep]
            for top in (0, 3):
                got = B.vl_token_logprobs(x, u, top=top)
                lp = want.gather(1, t[:, None])[:, 0]
                S = _sum_error(V)
                assert bool(((got.logprob[keep].double() - lp[keep]).abs() <= S + 8 * U * (lp[keep].abs() + 20)).all())
                rest = u < 0
                assert bool((got.logprob[rest] == 0).all()) and bool((got.row_stats[rest] == 0).all())
                if top:
                    assert bool((got.top_ids[rest] == -1).all())
                    best = torch.sort(x.float(), dim=1, descending=True, stable=True).indices[:, :top]
                    assert torch.equal(got.top_ids[keep].long(), best[keep])


@pytest.mark.parametrize("R,V,top", [(3, 200, 4), (2, 9000, 8), (1, 131072, 20), (300, 1024, 0)])
def test_streams_graphs_and_repeats(B, R, V, top):
    """On a side stream, twice at once, captured and replayed with other inputs: bit for bit what a plain call gives."""
    import torch
    rng = np.random.default_rng(R + V)
    a, b = _rows(_make(rng, R, V), "bf16"), _rows(_make(rng, R, V), "bf16")
    t = torch.from_numpy(rng.integers(0, V, R)).cuda()
    g = torch.randn(R, device="cuda")

    def call(x, stream=None):
        o = B.vl_token_logprobs(x, t, top=top, stream=stream)
        dx = B.vl_token_logprobs_backward(x, t, o.row_stats, g, entropy=o.entropy, g_entropy=g, stream=stream)
        return [v for v in o if v is not None] + [dx]

    want = [call(a), call(b)]
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        got = [call(a, s1), call(b, s2)]
        torch.cuda.synchronize()
        for u, v in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(u, v))
    x = a.clone()
    graphs = []
    with torch.cuda.stream(s1):
        for _ in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s1):
                out = call(x)
            graphs.append((graph, out))
    for src, u in ((b, want[1]), (a, want[0])):
        x.copy_(src)
        torch.cuda.synchronize()
        for (graph, out), st in zip(graphs, (s1, s2)):
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for graph, out in graphs:
            assert all(torch.equal(p, q) for p, q in zip(u, out))


def test_nothing_else_is_written(B):
    """Outputs of the C entry point between guards, and outputs that are not asked for."""
    import ctypes as C
    import torch
    rng = np.random.default_rng(6)
    lib = B._lib
    for R, V, top in [(3, 40, 5), (2, 3001, 32), (65, 300, 1)]:
        x = _rows(_make(rng, R, V), "f32")
        t = torch.from_numpy(rng.integers(0, V, R)).cuda()
        want = B.vl_token_logprobs(x, t, top=top)
        d = B.vl_logits(x.data_ptr(), B.VL_F32, R, V, V, t.data_ptr(), 8, None, 0, None, None, 1.0)
        sizes = [R, R, 2 * R, R * top, R * top]
        bufs = [torch.full((n + 16,), 12345.0, device="cuda") for n in sizes]
        ptrs = [b.data_ptr() + 32 for b in bufs]
        for skip in (None, 0, 1, 2):
            for b in bufs:
                b.fill_(12345.0)
            p = [None if skip == j else q for j, q in enumerate(ptrs)]
            torch.cuda.synchronize()
            assert lib.vl_token_logprobs(0, C.byref(d), p[0], p[1], p[2], top, p[3], p[4], None) == 0
            torch.cuda.synchronize()
            for j, (b, n) in enumerate(zip(bufs, sizes)):
                assert bool((b[:8] == 12345.0).all()) and bool((b[8 + n:] == 12345.0).all())
                if skip == j:
                    assert bool((b == 12345.0).all())
            assert torch.equal(bufs[3][8:8 + R * top].view(torch.int32).view(R, top), want.top_ids)
            if skip != 0:
                assert torch.equal(bufs[0][8:8 + R], want.logprob)
