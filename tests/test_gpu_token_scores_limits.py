"""Scores of tokens and their gradient where sizes, values and streams reach their limits; tolerances as in tests/test_gpu_token_scores.py."""
import numpy as np
import pytest

from paper_2506_17506_b200 import synth
from tests import score_oracle as ref
from tests.test_gpu_token_scores import U, B, _check_grad, _check_scores, _make, _masks, _oracle_stats, _rows, _type  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,V", [(1, 131072), (1, 40000), (7, 131072), (100, 131072), (300, 32768), (149, 40000)])
@pytest.mark.parametrize("kind", ["plain", "flat"])
def test_rows_split_over_blocks_again_and_again(B, R, V, kind):
    """Rows that two, four or eight blocks share, with alternatives: the blocks read each other's counts up to the last row, and one call
    ends while others begin.  Every call gives the first one's results, and these are right."""
    import torch
    rng = np.random.default_rng(R + V)
    x = _rows(_make(rng, min(R, 4), V, kind), "bf16")
    x = x.repeat((R + 3) // 4, 1)[:R].contiguous() if R > 4 else x
    t = torch.from_numpy(rng.integers(0, V, R)).cuda()
    t[R // 2::5] = -1 if R > 1 else int(t[0])
    want = B.vl_token_logprobs(x, t, top=20)
    n = min(R, 2)
    _check_scores(B.TokenLogprobs(*[v[:n] for v in want]), x[:n].double().cpu().numpy(), 1.0, np.zeros((n, V), bool), t[:n].tolist(), 20)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(40):
        got = [B.vl_token_logprobs(x, t, top=20), B.vl_token_logprobs(x, t, top=20, stream=side)]
        torch.cuda.synchronize()
        for g in got:
            assert all(torch.equal(a, b) for a, b in zip(g, want))


@pytest.mark.parametrize("V", [264, 512, 520, 1000, 1024])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_alternatives_of_aligned_rows_under_masks(B, dtype, V):
    """Rows that start and end on vectors, the whole warp at a row: the last vectors of a lane lie behind the row, and behind its mask."""
    import torch
    rng = np.random.default_rng(V)
    R = 9
    m, w = _masks(rng, R, V, 0.3), rng.choice([1, 2, 4, 40], R).astype(np.uint8)
    closed = np.array([ref.closed_entries(V, m[r], w[r]) for r in range(R)])
    x = _rows(np.where(closed, np.nan, _make(rng, R, V)), dtype)
    t = rng.integers(0, V, R)
    got = B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), occupied=torch.from_numpy(m.view(np.int32)).cuda(),
                              widths=torch.from_numpy(w).cuda(), top=5)
    _check_scores(got, x.double().cpu().numpy(), 1.0, closed, t, 5)


# (type, logits' middle, their step, scale): products of logits and scale from 2^20 to beyond 2^100, where a product's own rounding
# is up to many powers of two.  Steps are the type's own at that value, or larger.
LARGE = [("f32", -1e10, 1024.0, 1.0), ("f32", 1e10, 1024.0, 1.0), ("f32", 1e10, 1024.0, 1e-3), ("f32", -1e10, 1024.0, 1e-3),
         ("f32", 1e12, 65536.0, 1e-5), ("f32", -1e12, 65536.0, 1e-5), ("f32", 1e20, 2.0 ** 43, 1.0), ("f32", -1e20, 2.0 ** 43, 1e-6),
         ("f32", 5000.0, 2.0 ** -11, 1e6), ("f32", -5000.0, 2.0 ** -11, 1e3), ("f32", 2907270.4, 0.25, 1.0), ("f32", -2907270.4, 0.25, 1.0),
         ("f32", -1e9, 64.0, 1.0), ("f32", 9e28, 2.0 ** 73, 1e-6),
         ("f16", 65504.0, 32.0, 1e5), ("f16", -65504.0, 32.0, 1e5), ("f16", -65504.0, 32.0, 3e5), ("f16", 65504.0, 32.0, 1e6),
         ("f16", 60000.0, 32.0, 50.0), ("f16", -3000.0, 2.0, 1000.0),
         ("bf16", 1e10, 2.0 ** 26, 1e-6), ("bf16", -1e10, 2.0 ** 26, 1.0), ("bf16", 1e20, 2.0 ** 59, 1.0), ("bf16", -9e28, 2.0 ** 89, 1e-3)]


def _large(rng, R, V, dtype, middle, step):
    """Values around `middle`, a few dozen steps wide, below the type's largest; one row rises, one holds impossible entries."""
    k = rng.integers(-24, 25, (R, V)).astype(float)
    k[0] = np.round(np.linspace(-24, 24, V))
    x = middle + step * k
    most = {"f32": 3.4e38, "f16": 65504.0, "bf16": 3.3e38}[dtype]
    x = np.clip(x, -most, most)
    if V > 4:
        x[-1, ::3] = -np.inf
    return x


@pytest.mark.parametrize("dtype,middle,step,scale", LARGE)
@pytest.mark.parametrize("R,V", [(5, 40), (3, 300), (3, 2041), (3, 9001), (2, 131072), (700, 4200)])
def test_products_of_logits_and_scale_that_are_large(B, dtype, middle, step, scale, R, V):
    import torch
    rng = np.random.default_rng(V)
    x = _rows(_large(rng, R, V, dtype, middle, step), dtype, pad=V % 3)
    scale = float(np.float32(scale))
    t = rng.integers(0, V, R)
    n = min(R, 4)
    pick = np.r_[0:n - 1, R - 1]
    x64 = x[torch.from_numpy(pick).cuda()].double().cpu().numpy()
    for top in (0, 3):
        got = B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), scale=scale, top=top)
        head = B.TokenLogprobs(*[None if v is None else v[torch.from_numpy(pick).cuda()] for v in got])
        _check_scores(head, x64, scale, np.zeros((n, V), bool), t[pick], top)


@pytest.mark.parametrize("dtype,middle,step,scale", LARGE)
@pytest.mark.parametrize("R,V", [(5, 40), (3, 300), (3, 9001), (2, 50000)])
def test_gradients_at_products_that_are_large(B, dtype, middle, step, scale, R, V):
    import torch
    rng = np.random.default_rng(V + 1)
    x = _rows(_large(rng, R, V, dtype, middle, step), dtype, pad=V % 3)
    x64, closed, t, scale = x.double().cpu().numpy(), np.zeros((R, V), bool), rng.integers(0, V, R), float(np.float32(scale))
    stats, H = _oracle_stats(x64, scale, closed, t)
    by = 1e-3 / scale if dtype == "f16" else 1.0          # within the range of halves
    g, h = (rng.normal(0, 8, R) * by).astype(np.float32), (rng.normal(0, 2, R) * by).astype(np.float32)
    for ent in (False, True):
        dx = B.vl_token_logprobs_backward(x, torch.from_numpy(t).cuda(), stats, torch.from_numpy(g).cuda(), entropy=H if ent else None,
                                          g_entropy=torch.from_numpy(h).cuda() if ent else None, scale=scale)
        _check_grad(dx, x64, scale, closed, t, g.astype(float), h.astype(float) * ent, dtype)


@pytest.mark.parametrize("V", [16, 61, 300, 1500, 9001])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_closed_entries_have_no_gradient_whatever_the_others_hold(B, dtype, V):
    """Derivatives that overflowed or are no numbers, rows whose open logits hold an infinity or no number, statistics that are no numbers:
    the gradient of a closed entry is 0."""
    import torch
    rng = np.random.default_rng(V)
    R = 12
    m = _masks(rng, R, V, 0.4)
    m[:, 0] = (m[:, 0] | 1) & ~np.uint32(2)
    closed = np.array([ref.closed_entries(V, m[r]) for r in range(R)])
    vals = np.where(closed, rng.choice([np.nan, np.inf, -np.inf, 7.0], (R, V)), _make(rng, R, V))
    vals[0, 1], vals[1, 1] = np.nan, np.inf
    x = _rows(vals, dtype, pad=V % 2)
    t = torch.full((R,), 1, device="cuda")
    occ = torch.from_numpy(m.view(np.int32)).cuda()
    fwd = B.vl_token_logprobs(x, t, occupied=occ)
    stats, ent = fwd.row_stats.clone(), fwd.entropy.clone()
    stats[2, 1], stats[3, 0], stats[4] = float("nan"), float("nan"), float("inf")
    g, h = torch.ones(R, device="cuda"), torch.ones(R, device="cuda")
    g[5], g[6], h[7], h[8], g[9] = float("inf"), float("nan"), float("inf"), float("nan"), -float("inf")
    ent[10] = float("nan")
    for out in (None, x.clone()):
        for more in (dict(), dict(entropy=ent, g_entropy=h)):
            if out is not None:
                out.copy_(x)
            dx = B.vl_token_logprobs_backward(x if out is None else out, t, stats, g, occupied=occ, out=out, **more).float().cpu().numpy()
            assert np.all(dx[closed] == 0)
            assert not any(np.all(np.isfinite(dx[r])) for r in (0, 1, 5, 6, 9)) and np.all(np.isfinite(dx[11]))


@pytest.mark.parametrize("V", [40, 1500, 9001])
def test_derivatives_that_overflow_with_the_scale(B, V):
    """scale g is beyond the range of numbers: what p = 0 leaves of it is 0, and small p leave numbers."""
    import torch
    rng = np.random.default_rng(V)
    vals = np.full((2, V), -8e-5)
    vals[:, ::4] = -1.0           # exp(-1e6) = 0
    vals[0, 1] = 0.0
    x = _rows(vals, "f32")
    x64, closed, t, scale = x.double().cpu().numpy(), np.zeros((2, V), bool), np.array([1, 2]), 1e6
    stats, H = _oracle_stats(x64, scale, closed, t)
    g = np.array([1e33, -1e33], dtype=np.float32)
    dx = B.vl_token_logprobs_backward(x, torch.from_numpy(t).cuda(), stats, torch.from_numpy(g).cuda(), scale=scale).double().cpu().numpy()
    assert np.all(dx[:, ::4] == 0) and not np.any(np.isnan(dx))
    want = ref.grad_row(x64[0], scale, closed[0], 1, float(g[0]), 0.0)
    ok = (np.abs(want) < 1e38) & (want != 0)
    # p = exp(-80): (12 + 4 (80 + 1)) u and a few roundings
    assert np.count_nonzero(ok) and np.all(np.abs(dx[0][ok] - want[ok]) <= 500 * U * np.abs(want[ok]))


def test_masks_on_a_side_stream_belong_to_it(B):
    """Masks that stay on the device: memory that the current stream frees, or takes while a side stream still works with them, is another's."""
    import torch
    prog = synth.build_program(synth.shape_tiny(), 0)
    rows, _ = synth.candidate_rows(prog, 2, 0.4, 3)
    gp = B.Program(prog)
    gp.vl_liveness()
    row = torch.from_numpy(rows.view(np.int16)).cuda().view(torch.uint16)[0]
    want = gp.vl_occupied_masks(row, prog.P, words=True)
    x = torch.randn(want.shape[0], prog.P, device="cuda")
    scores = B.vl_token_logprobs(x, occupied=want, top=4)
    nbytes = want.numel() * 4
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for number in (False, True):
        st = side.cuda_stream if number else side
        for cycles in (0, 400_000_000, 400_000_000):      # first without a delay: memory and kernels are there from then on
            masks = gp.vl_occupied_masks(row, prog.P, stream=st, words=True)
            if cycles:
                with torch.cuda.stream(side):
                    torch.cuda._sleep(cycles)
            got = B.vl_token_logprobs(x, occupied=masks, top=4, stream=st)
            del masks
            others = [torch.full((nbytes // 4,), -1, dtype=torch.int32, device="cuda") for _ in range(3000)]
            assert not cycles or not side.query()          # they were written before the side stream began
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, scores) if a is not None)
            del others, got
    gp.close()


def test_rows_of_logits_and_gradient_in_turn(B):
    """Both are columns of one matrix; what is neither's is left as it was, and columns in common are refused."""
    import torch
    rng = np.random.default_rng(3)
    for dtype in ("f32", "bf16"):
        for R, V in [(5, 24), (70, 37), (1, 50), (4, 1001), (3, 9003)]:
            big = torch.full((R, 2 * V + 3), float("nan"), dtype=_type(dtype), device="cuda")
            for a, b in ((0, V), (V + 3, 0), (1, V + 2)):
                x, out = big[:, a:a + V], big[:, b:b + V]
                big.fill_(float("nan"))
                x.copy_(torch.from_numpy(_make(rng, R, V)))
                keep = x.clone()
                t = torch.from_numpy(rng.integers(0, V, R)).cuda()
                f = B.vl_token_logprobs(keep, t)
                g = torch.ones(R, device="cuda")
                want = B.vl_token_logprobs_backward(keep, t, f.row_stats, g)
                got = B.vl_token_logprobs_backward(x, t, f.row_stats, g, out=out)
                rest = torch.ones(2 * V + 3, dtype=torch.bool, device="cuda")
                rest[a:a + V] = rest[b:b + V] = False
                assert torch.equal(got, want) and torch.equal(x, keep) and bool(torch.isnan(big[:, rest]).all())
            for a, b in ((0, V - 1), (3, 0)):
                with pytest.raises(B.VlError):
                    B.vl_token_logprobs_backward(big[:, a:a + V], t, f.row_stats, g, out=big[:, b:b + V])


@pytest.mark.parametrize("side", [False, True])
def test_results_that_are_kept_keep_nothing_else(B, side):
    """A log of losses or log probabilities holds what it shows, not the calls' other results and working memory."""
    import torch
    stream = torch.cuda.Stream() if side else None
    x, t = torch.randn(5000, 64, device="cuda"), torch.zeros(5000, dtype=torch.int64, device="cuda")
    v, off = torch.zeros(1000, 4, dtype=torch.int32, device="cuda"), torch.arange(0, 5001, 5, device="cuda")
    torch.cuda.synchronize()
    o = B.vl_token_logprobs(x, t, top=16, stream=stream)
    torch.cuda.synchronize()
    for r in list(o) + list(B.vl_policy_loss([v], off, o.logprob, stream=stream)):
        assert r.untyped_storage().nbytes() == r.numel() * r.element_size()
    torch.cuda.synchronize()


@pytest.mark.parametrize("V", [5, 16, 31, 64, 200, 250, 256, 300, 512, 1000, 1024, 2500, 4100, 9001, 40013])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_masks_and_widths_without_alternatives(B, dtype, V):
    """Several rows a warp, each under a mask and a width of its own, and many long rows: closed logits hold infinities and no numbers, some rows
    have nothing left, some are under no mask, some are left out."""
    import torch
    rng = np.random.default_rng(V)
    R, n = (70, 9) if V <= 4100 else (5, 5)
    for share, widths, pad in [(0.5, None, 0), (0.15, [0, 1, 2, 4, 5, 31], 0), (0.004, [32, 33, 64, 65, 200, 255], 8), (None, [1, 3, 40], 5), (0.3, [1, 2], 3)]:
        m = None if share is None else _masks(rng, n, V, share)
        if m is not None:
            m[3], m[4] = 0xFFFFFFFF, 0
        which = rng.integers(-1, n + 1, R).astype(np.int32)
        which[:3] = [3, 4, -2 ** 31]
        w = None if widths is None else rng.choice(widths, R).astype(np.uint8)
        closed = np.array([ref.closed_entries(V, m[which[r]] if m is not None and 0 <= which[r] < n else None, 1 if w is None else w[r])
                           for r in range(R)])
        fill = rng.choice([np.nan, np.inf, -np.inf, {"f32": 3.4e38, "f16": 65504.0, "bf16": 3.3e38}[dtype]], (R, V))
        x = _rows(np.where(closed, fill, _make(rng, R, V)), dtype, pad=pad, shift=pad % 4)
        t = rng.integers(0, V, R)
        t[1] = 65535
        got = B.vl_token_logprobs(x, torch.from_numpy(t.astype(np.uint16)).cuda(),
                                  occupied=None if m is None else torch.from_numpy(m.view(np.int32)).cuda(),
                                  mask_rows=None if m is None else torch.from_numpy(which).cuda(),
                                  widths=None if w is None else torch.from_numpy(w).cuda())
        _check_scores(got, x.double().cpu().numpy(), 1.0, closed, t, 0)


def test_more_masked_long_rows_than_places(B):
    """Blocks go from row to row under masks: against the same rows with the closed entries set to minus infinity, bit for bit."""
    import torch
    rng = np.random.default_rng(7)
    for R, V, dtype in [(3000, 9000, "bf16"), (2500, 4500, "f32"), (5000, 5003, "f16"), (90, 70000, "bf16")]:
        n = 61
        m = _masks(rng, n, V, 0.4)
        closed = torch.from_numpy(np.array([ref.closed_entries(V, m[j]) for j in range(n)])).cuda()
        which = torch.randint(0, n, (R,), device="cuda")
        x = torch.randn(R, V, device="cuda").to(_type(dtype))
        t = torch.randint(-1, V, (R,), device="cuda")
        occ = torch.from_numpy(m.view(np.int32)).cuda()
        want = B.vl_token_logprobs(x.masked_fill(closed[which], float("-inf")), t)
        got = B.vl_token_logprobs(x, t, occupied=occ, mask_rows=which.to(torch.int32))
        assert torch.equal(got.logprob, want.logprob) and torch.equal(got.entropy, want.entropy) and torch.equal(got.row_stats, want.row_stats)
        lp = torch.log_softmax(x[:50].double().masked_fill(closed[which[:50]], float("-inf")), dim=1)
        real = t[:50] >= 0
        exact = lp.gather(1, t[:50].clamp(min=0)[:, None])[:, 0][real]
        # S of the module's tolerance, and 3 u (|ln p| + 2 L) with L < ln V + 6
        S = (V / 32 + 40 + 2 * (20 + np.log(V))) * U
        near = (got.logprob[:50][real].double() - exact).abs() <= S + 3 * U * (exact.abs() + 2 * (np.log(V) + 6))
        assert bool((near | (got.logprob[:50][real].double() == exact)).all())


@pytest.mark.parametrize("R,V", [(3, 12), (3, 700), (2, 9001), (1, 131072)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_differences_beyond_the_range_of_numbers(B, dtype, R, V):
    """Logits at both ends of the type: their difference is no 32-bit number, its product with a small scale is."""
    import torch
    rng = np.random.default_rng(V)
    vals = rng.choice([3.2e38, -3.2e38, 2e38, -1e30], (R, V))
    vals[:, 0], vals[:, 1] = 3.2e38, -3.2e38
    x = _rows(vals, dtype)
    x64, closed = x.double().cpu().numpy(), np.zeros((R, V), bool)
    for scale in (1e-6, 1e-3, 0.25):
        scale = float(np.float32(scale))
        for t in (np.full(R, 1), rng.integers(0, V, R)):
            for top in (0, 12):
                _check_scores(B.vl_token_logprobs(x, torch.from_numpy(t).cuda(), scale=scale, top=top), x64, scale, closed, t, top)
