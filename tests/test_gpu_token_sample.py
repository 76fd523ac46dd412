"""Drawing a token of every row: CUDA path against a plain 64-bit form.

Tolerances.  Which token, and how many entries are kept: equal (both sides decide in 64 bits; sums of up to 2^17 terms in another order differ
by some 2^-46 of their size, and what they are compared with is drawn at random or an exact number).  Log probabilities: u = 2^-24 is half a step
of a 32-bit number.  A sum of 32-bit terms is within S = (V / 32 + 40 + 2 D) u of its value relatively as derived in
tests/test_gpu_token_scores.py, so ln p within S + 3 u (|ln p| + 2 |L|); the one of what was kept likewise.
"""
import numpy as np
import pytest

from tests import sample_oracle as ref
from tests import score_oracle
from tests.test_gpu_token_scores import DTYPES, U, B, _make, _masks, _rows, _sum_error  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu

RULES = [dict(), dict(top_k=1), dict(top_k=7), dict(top_p=0.9), dict(min_p=0.05), dict(top_k=40, top_p=0.8), dict(top_p=0.97, min_p=0.01),
         dict(top_k=300, top_p=0.99, min_p=0.001)]


def _uniform(rng, R):
    u = rng.random(R).astype(np.float32)
    u[u >= 1.0] = 0.5
    return u


def check(got, x64, scale, closed, u, rules, rows=None):
    """got: TokenSample; x64: [R, V] as the device holds them."""
    R, V = x64.shape
    S = _sum_error(V)
    tok, lp, drawn, kept = (t.cpu().numpy() for t in got)
    scale = float(np.float32(scale))
    for r in range(R) if rows is None else rows:
        want = ref.sample_row(x64[r], scale, closed[r], float(u[r]), **rules)
        assert (int(tok[r]), int(kept[r])) == (want[0], want[3]), (r, int(tok[r]), int(kept[r]), want, rules)
        for a, b in ((lp[r], want[1]), (drawn[r], want[2])):
            if np.isfinite(b):
                assert abs(a - b) <= S + 3 * U * (abs(b) + 2 * abs(want[1])) and a <= 0, (r, a, b)
            else:
                assert a == b or (np.isnan(a) and np.isnan(b)), (r, a, b)


SIZES = [(3, 1), (5, 2), (7, 7), (33, 16), (9, 31), (6, 32), (7, 33), (5, 64), (4, 100), (9, 128), (17, 255), (40, 256), (5, 257), (8, 512),
         (6, 1000), (3, 1024), (3, 1025), (4, 2047), (3, 2048), (3, 4097), (3, 8191), (2, 20011), (3, 50021), (2, 131072), (1, 131075)]


@pytest.mark.parametrize("R,V", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_many_sizes_and_rules(B, dtype, R, V):
    import torch
    rng = np.random.default_rng(V * 5 + R)
    for j, rules in enumerate(RULES):
        scale, pad, shift = [(1.0, 0, 0), (0.7, 3, 1), (1.4, 8, 8)][j % 3]
        x = _rows(_make(rng, R, V), dtype, pad, shift)
        u = _uniform(rng, R)
        got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), scale=scale, **rules)
        check(got, x.double().cpu().numpy(), scale, np.zeros((R, V), bool), u, rules)


@pytest.mark.parametrize("kind", ["levels", "flat", "holes", "rising"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_equal_impossible_and_sorted_entries(B, dtype, kind):
    import torch
    rng = np.random.default_rng(6)
    for R, V in [(3, 9), (4, 200), (5, 256), (3, 777), (2, 3000), (2, 40013)]:
        x = _rows(_make(rng, R, V, kind), dtype)
        for rules in RULES + [dict(top_p=0.5), dict(min_p=1.0), dict(top_k=V), dict(top_k=V + 5), dict(top_p=1e-9)]:
            u = _uniform(rng, R)
            got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), **rules)
            check(got, x.double().cpu().numpy(), 1.0, np.zeros((R, V), bool), u, rules)


@pytest.mark.parametrize("V", [1, 3, 16, 40, 64, 250, 256, 264, 512, 1000, 1024, 2056, 9000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_masks_and_widths(B, dtype, V):
    """Closed entries hold no numbers; one mask leaves nothing, one everything; some rows are under no mask."""
    import torch
    rng = np.random.default_rng(V)
    R, n = 23, 6
    m = _masks(rng, n, V, 0.5)
    m[0], m[1] = 0xFFFFFFFF, 0
    which = rng.integers(-1, n + 1, R).astype(np.int32)
    which[:3] = [0, 1, -1]
    w = rng.choice([0, 1, 2, 4, 33], R).astype(np.uint8)
    for widths in (None, w):
        closed = np.array([score_oracle.closed_entries(V, m[which[r]] if 0 <= which[r] < n else None, 1 if widths is None else w[r])
                           for r in range(R)])
        x = _rows(np.where(closed, rng.choice([np.nan, np.inf, -np.inf, 3e4], (R, V)), _make(rng, R, V)), dtype, pad=V % 5)
        for rules in RULES[:7]:
            u = _uniform(rng, R)
            got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), occupied=torch.from_numpy(m.view(np.int32)).cuda(),
                                    mask_rows=torch.from_numpy(which).cuda(),
                                    widths=None if widths is None else torch.from_numpy(w).cuda(), scale=0.8, **rules)
            check(got, x.double().cpu().numpy(), 0.8, closed, u, rules)


@pytest.mark.parametrize("V", [5, 200, 1500, 30000])
def test_numbers_at_the_ends_and_rows_left_out(B, V):
    import torch
    rng = np.random.default_rng(V)
    u = np.array([0.0, np.float32(1 - 2.0 ** -24), 2.0 ** -149, 1.0, -1e-9, np.nan, np.inf, -0.0, 0.5], dtype=np.float32)
    R = len(u)
    x = _rows(_make(rng, R, V), "f32")
    for rules in RULES:
        got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), **rules)
        check(got, x.double().cpu().numpy(), 1.0, np.zeros((R, V), bool), u, rules)


def test_exact_borders_of_equal_entries(B):
    """Weights of 1: every sum is exact, and a number on a border belongs to the entry behind it."""
    import torch
    for V in (8, 64, 1024, 4096):
        x = torch.full((V, V), -2.5, device="cuda")
        u = torch.arange(V, device="cuda") / V
        got = B.vl_token_sample(x, u)
        assert torch.equal(got.tokens, torch.arange(V, device="cuda")) and bool((got.kept == V).all())
        got = B.vl_token_sample(x, u, top_p=0.25)
        assert torch.equal(got.tokens, torch.arange(V, device="cuda") // 4) and bool((got.kept == V // 4).all())


@pytest.mark.parametrize("V", [40, 700, 5000, 70001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_without_results(B, dtype, V):
    import torch
    rng = np.random.default_rng(V)
    x64 = _make(rng, 6, V)
    x64[0, V // 2] = np.nan
    x64[1, V - 1] = np.inf
    x64[2] = -np.inf
    x64[3] = -np.inf
    x64[3, V // 3] = -5.0
    x64[4, ::2] = -np.inf
    x = _rows(x64, dtype)
    for rules in RULES:
        u = _uniform(rng, 6)
        got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), **rules)
        check(got, x.double().cpu().numpy(), 1.0, np.zeros((6, V), bool), u, rules)


@pytest.mark.parametrize("dtype,middle,step,scale", [("f32", -1e10, 1024.0, 1e-3), ("f32", 1e20, 2.0 ** 43, 1e-6), ("f32", 5000.0, 2.0 ** -11, 1e6),
                                                     ("f32", -3e38, 2.0 ** 104, 1.0), ("f16", 65504.0, 32.0, 0.01), ("f16", -65504.0, 32.0, 1e6),
                                                     ("bf16", 1e10, 2.0 ** 26, 1e-6), ("bf16", -3e38, 2.0 ** 121, 1e-6)])
def test_large_logits_and_scales(B, dtype, middle, step, scale):
    import torch
    rng = np.random.default_rng(11)
    most = {"f32": 3.4e38, "f16": 65504.0, "bf16": 3.3e38}[dtype]
    for R, V in [(5, 50), (5, 1000), (3, 9001), (2, 60000)]:
        x = _rows(np.clip(middle + step * rng.integers(-24, 25, (R, V)), -most, most), dtype)
        for rules in RULES[::2]:
            u = _uniform(rng, R)
            got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), scale=scale, **rules)
            tok, kept = got.tokens.cpu().numpy(), got.kept.cpu().numpy()
            x64 = x.double().cpu().numpy()
            for r in range(R):
                want = ref.sample_row(x64[r], float(np.float32(scale)), np.zeros(V, bool), float(u[r]), **rules)
                assert (tok[r], kept[r]) == (want[0], want[3]), (r, V, rules)


@pytest.mark.parametrize("R,V,dtype", [(4000, 96, "bf16"), (2500, 512, "f32"), (1300, 1100, "f16"), (700, 5000, "bf16"), (300, 20000, "f32")])
def test_many_rows_against_sorting(B, R, V, dtype):
    """Every row's token and count, with sums on the device in 64 bits."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = (torch.randn(R, V, generator=gen, device="cuda") * 2.5).to(B._Torch.load() and {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype])
    x[::3, V // 2] += 9
    u = torch.rand(R, generator=gen, device="cuda")
    for rules in RULES:
        got = B.vl_token_sample(x, u, scale=0.9, **rules)
        xd = x.double()
        w = torch.exp((xd - xd.amax(1, keepdim=True)) * float(np.float32(0.9)))
        order = torch.sort(x.float(), dim=1, descending=True, stable=True).indices
        ws = w.gather(1, order)
        keep = torch.arange(V, device="cuda")[None] < (rules.get("top_k") or V)
        sums = torch.cumsum(ws * keep, 1)
        if rules.get("top_p", 1.0) < 1.0:
            keep = keep & ((sums - ws) < rules["top_p"] * sums[:, -1:])
        keep = keep & (ws >= rules.get("min_p", 0.0))
        here = torch.zeros_like(keep).scatter(1, order, keep)
        sums = torch.cumsum(w * here, 1)
        tok = torch.searchsorted(sums, u[:, None].double() * sums[:, -1:], right=True)[:, 0]
        assert torch.equal(got.kept.long(), keep.sum(1)), rules
        assert torch.equal(got.tokens, tok), rules


def test_token_types_strides_streams_and_graphs(B):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    for R, V in [(50, 300), (9, 7000)]:
        x = torch.randn(R, V, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)
        u = torch.rand(R, generator=gen, device="cuda")
        want = B.vl_token_sample(x, u, top_p=0.9)
        for kind in (torch.int32, torch.uint16, torch.int16):
            got = B.vl_token_sample(x, u, top_p=0.9, token_dtype=kind)
            assert got.tokens.dtype == kind and torch.equal(got.tokens.to(torch.int32).long(), want.tokens)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = B.vl_token_sample(x, u, top_p=0.9, stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        xs, us = x.clone(), u.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = B.vl_token_sample(xs, us, top_p=0.9)
        for k in range(3):
            xs.copy_(x.roll(k, 1))
            us.copy_(u.roll(k))
            graph.replay()
            again = B.vl_token_sample(xs, us, top_p=0.9)
            assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_outputs_are_written_and_nothing_else(B):
    import ctypes as C
    import torch
    gen = torch.Generator(device="cuda").manual_seed(4)
    for R, V in [(37, 40), (5, 3000)]:
        x = torch.randn(R, V, generator=gen, device="cuda")
        u = torch.rand(R, generator=gen, device="cuda")
        want = B.vl_token_sample(x, u, top_k=5, token_dtype=torch.int32)
        d = B.vl_logits(logits=x.data_ptr(), dtype=B.VL_F32, n_rows=R, n_vocab=V, row_stride=V, scale=1.0)
        rules = B.vl_sampling(5, 1.0, 0.0)
        outs = [torch.full((R + 8,), 77, device="cuda", dtype=t) for t in (torch.int32, torch.float32, torch.float32, torch.int32)]
        p = [o[4:].data_ptr() for o in outs]
        work, size = torch.empty(64, device="cuda", dtype=torch.uint8), 64
        assert B._lib.vl_token_sample(0, C.byref(d), C.byref(rules), u.data_ptr(), p[0], 4, p[1], p[2], p[3], work.data_ptr(), size, None) == B.VL_OK
        torch.cuda.synchronize()
        for o, wanted in zip(outs, want):
            assert torch.equal(o[4:-4], wanted.to(o.dtype)) and bool((o[:4] == 77).all()) and bool((o[-4:] == 77).all())
        again = torch.empty(R, device="cuda", dtype=torch.int32)
        assert B._lib.vl_token_sample(0, C.byref(d), C.byref(rules), u.data_ptr(), again.data_ptr(), 4, None, None, None, work.data_ptr(), size, None) == B.VL_OK
        torch.cuda.synchronize()
        assert torch.equal(again, want.tokens)


def _peaked(gen, R, V, dtype):
    """Rows of a model: few favourites, some possible entries, the rest far below; flat ones, one with a single possible favourite, some
    whose first entries, or all but a few, are shut by large negative logits."""
    import torch
    x = torch.randn(R, V, generator=gen, device="cuda") * 2
    at = torch.randint(0, V, (R, 40), generator=gen, device="cuda")
    x.scatter_(1, at, torch.rand(R, 40, generator=gen, device="cuda") * 8 + 8)
    x[::7] = torch.randn(V, generator=gen, device="cuda")
    x[1::7, V // 2] = 60.0
    x[2::7, : V - V // 3] = torch.finfo(dtype).min
    x[3::7, 50:] = -1e4
    x[4::7, ::2] = -float("inf")
    return x.to(dtype)


@pytest.mark.parametrize("R,V,dtype", [(1, 131072, "bf16"), (3, 100003, "f16"), (20, 65536, "f32"), (150, 32768, "f16"), (600, 16000, "bf16"),
                                       (1300, 8200, "f32"), (2000, 2100, "bf16")])
def test_rows_of_a_model(B, R, V, dtype):
    """Against sorting on the device in 64 bits, and the same again when called again."""
    import torch
    kind = B._Torch.load() and {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(R + V)
    x = _peaked(gen, R, V, kind)
    u = torch.rand(R, generator=gen, device="cuda")
    xd = x.double()
    w = torch.exp((xd - xd.amax(1, keepdim=True)) * float(np.float32(1.1)))
    order = torch.sort(x.float(), dim=1, descending=True, stable=True).indices
    ws = w.gather(1, order)
    possible = (xd > -np.inf).gather(1, order)
    for rules in RULES + [dict(top_k=50), dict(top_k=1500, top_p=0.9), dict(top_p=0.5), dict(min_p=0.3, top_p=0.95), dict(min_p=1e-9)]:
        got = B.vl_token_sample(x, u, scale=1.1, **rules)
        keep = possible & (torch.arange(V, device="cuda")[None] < (rules.get("top_k") or V))
        sums = torch.cumsum(ws * keep, 1)
        if rules.get("top_p", 1.0) < 1.0:
            keep = keep & torch.cat([torch.ones_like(keep[:, :1]), (sums < rules["top_p"] * sums[:, -1:])[:, :-1]], 1)
        keep = keep & (ws >= rules.get("min_p", 0.0))
        here = torch.zeros_like(keep).scatter(1, order, keep)
        sums = torch.cumsum(w * here, 1)
        T = sums[:, -1:]
        tok = torch.searchsorted(sums, u[:, None].double() * T, right=True)
        assert torch.equal(got.kept.long(), keep.sum(1)), rules
        assert torch.equal(got.tokens, tok[:, 0]), rules
        z = torch.log(w.gather(1, tok)[:, 0])
        for a, b in ((got.logprob, z - torch.log(w.sum(1))), (got.drawn_logprob, z - torch.log(T[:, 0]))):
            assert bool(((a.double() - b).abs() <= _sum_error(V) + 3 * U * 3 * (z.abs() + 20)).all()), rules
        again = B.vl_token_sample(x, u, scale=1.1, **rules)
        assert all(torch.equal(a, b) for a, b in zip(got, again)), rules


@pytest.mark.parametrize("R,V,dtype", [(2, 600000, "bf16"), (9, 300000, "f32"), (40, 9000, "f16"), (3, 140000, "f16")])
def test_broad_rows_that_no_list_holds(B, R, V, dtype):
    """Tens of thousands of entries are kept, ties among them, of rows up to ones that no shared memory holds; the same in a graph."""
    import torch
    kind = B._Torch.load() and {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    gen = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(R, V, generator=gen, device="cuda").mul_(1.5).to(kind)
    x[0] = (x[0].float() * 2).round().to(kind)          # some dozen values
    x[-1, V // 3:] = x[-1, V // 2]                      # most entries alike
    u = torch.rand(R, generator=gen, device="cuda")
    zeros = np.zeros((R, V), bool)
    for rules in [dict(), dict(top_p=0.95), dict(top_p=0.4), dict(top_k=5000), dict(top_k=3000, top_p=0.7), dict(min_p=0.02, top_p=0.9), dict(min_p=0.001)]:
        got = B.vl_token_sample(x, u, scale=0.9, **rules)
        check(got, x.double().cpu().numpy(), 0.9, zeros, u.cpu().numpy(), rules, rows=range(min(R, 6)))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            again = B.vl_token_sample(x, u, scale=0.9, **rules)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, again)), rules
