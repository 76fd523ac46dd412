"""The global gradient norm and clipping: CUDA path against a plain 64-bit form.

Tolerances.  u = 2^-24.  A thread's sum of at most 64 squares in 32 bits: each square and each of the at most 8 + 3 additions it goes through is
rounded once, so it is within 12 u of its value; everything behind it is in 64 bits.  The norm, its root: 6 u, and 1 u for its own rounding.  A result is
scale * factor * x, where the factor has the norm's error (max_norm / norm: 7 u) unless the norm is below max_norm, with one rounding (1 u; in
16 bits by way of 32: half a step of the type more).
"""
import numpy as np
import pytest

from tests import sample_oracle as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}      # a step of the smallest numbers


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


def _name(t):
    import torch
    return {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[t.dtype]


def _tensor(rng, n, dtype, size=1.0, shift=0):
    """A CUDA vector of n elements that starts `shift` elements into its memory."""
    import torch
    store = torch.full((n + shift + 9,), float("nan"), dtype=_type(dtype), device="cuda")
    t = store[shift:shift + n]
    t.copy_(torch.from_numpy(rng.normal(0, size, n)))
    return t


def _check(B, grads, scale, max_norm, in_place=False, outs=None):
    import torch
    arrays = [g.double().cpu().numpy() for g in grads]
    norm = ref.norm(arrays, scale)
    got = B.vl_grad_norm(grads, scale=scale)
    if norm >= 2.0 ** 128:          # above the largest number of 32 bits: it reads as infinity there, and is one everywhere else
        assert float(got.norm) == np.inf
    else:
        assert abs(float(got.norm) - norm) <= 7 * U * norm, (float(got.norm), norm)
    if np.isinf(norm):              # (an element that its type holds as infinity)
        assert float(got.sum_squares) == np.inf
    else:
        assert abs(float(got.sum_squares) - norm ** 2) <= 12 * U * norm ** 2
    if not in_place and outs is None:
        outs = [torch.empty_like(g) for g in grads]
    c = B.vl_clip_grads(grads, max_norm, scale=scale, outs=outs)
    f = ref.factor(norm, max_norm)
    assert float(c.norm) == float(got.norm)
    assert abs(float(c.factor) - f) <= 8 * U * f
    for a, o in zip(arrays, c.outs):
        t = _name(o)
        want = a * (scale * f) if f else np.zeros_like(a)
        err = np.abs(o.double().cpu().numpy() - want)
        rel = (7 * U if norm > max_norm * (1 - 8 * U) else 0.0) + U + (HALF[t] if t != "f32" else 0.0)
        assert np.all(err <= rel * 1.0001 * np.abs(want) + LEAST[t]), (t, float(err.max()))
    return c


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 255, 1000, 4096, 16384, 16385, 131071, 1000003])
def test_one_tensor(B, dtype, n):
    rng = np.random.default_rng(n)
    for shift, scale, max_norm in [(0, 1.0, 0.5), (1, 0.25, 1e9), (3, 1.0 / 1024, 1.0), (8, 1.0, 0.0)]:
        _check(B, [_tensor(rng, n, dtype, 1.0, shift)], scale, max_norm)


@pytest.mark.parametrize("count", [0, 2, 63, 64, 65, 960, 961, 2500])
def test_many_tensors_of_all_types(B, count):
    rng = np.random.default_rng(count)
    grads = [_tensor(rng, int(rng.choice([0, 1, 5, 300, 5000])), ["f32", "f16", "bf16"][j % 3], 0.1 * (1 + j % 5), j % 4) for j in range(count)]
    if count == 0:
        got = B.vl_clip_grads([], 1.0)
        assert float(got.norm) == 0.0 and float(got.factor) == 1.0 and float(B.vl_grad_norm([]).sum_squares) == 0.0
        return
    _check(B, grads, 0.5, 1.0)
    _check(B, grads, 0.5, 1.0, in_place=True)


def test_results_elsewhere_in_their_vectors(B):
    """Results that start elsewhere in their 16 bytes than the tensors do; nothing around them is written."""
    import torch
    rng = np.random.default_rng(2)
    for dtype in ("f32", "f16", "bf16"):
        for n in (5, 100, 40001):
            for shift, to in [(0, 1), (3, 0), (1, 2), (2, 2)]:
                store = torch.full((n + 16,), 77.0, dtype=_type(dtype), device="cuda")
                _check(B, [_tensor(rng, n, dtype, 1.0, shift)], 1.0, 0.7, outs=[store[to:to + n]])
                assert bool((store[:to] == 77).all()) and bool((store[to + n:] == 77).all())


@pytest.mark.parametrize("dtype,size", [("f32", 1e-30), ("f32", 3e-42), ("f32", 1e25), ("f32", 1e37), ("bf16", 1e-30), ("bf16", 1e30), ("f16", 3e-7), ("f16", 2e4), ("f16", 1e4)])
def test_sizes_beyond_what_squares_of_32_bits_hold(B, dtype, size):
    rng = np.random.default_rng(9)
    grads = [_tensor(rng, n, dtype, size, n % 3) for n in (7, 3000, 70001)]
    norm = ref.norm([g.double().cpu().numpy() for g in grads], 1.0)
    _check(B, grads, 1.0, norm / 3)
    _check(B, grads, 1.0, norm * 3)


def test_zeros_and_a_few_large_ones(B):
    import torch
    g = torch.zeros(100000, device="cuda")
    got = B.vl_clip_grads([g], 1.0)
    assert float(got.norm) == 0.0 and float(got.factor) == 1.0 and not bool(g.any())
    g[77777] = 1e-38
    g[5] = -2e30
    _check(B, [g], 1.0, 1.0)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_no_number_makes_every_result_0(B, dtype, bad):
    import torch
    rng = np.random.default_rng(4)
    grads = [_tensor(rng, n, dtype, 1.0, n % 2) for n in (33, 20000, 3)]
    grads[1][19999] = bad
    for max_norm in (1.0, float("inf")):
        outs = [torch.full_like(g, 5.0) for g in grads]
        got = B.vl_clip_grads(grads, max_norm, outs=outs)
        assert float(got.factor) == 0.0 and not np.isfinite(float(got.norm))
        assert not any(bool(o.any()) for o in outs)
    assert not np.isfinite(float(B.vl_grad_norm(grads).norm))
    B.vl_clip_grads(grads, 1.0)
    assert not any(bool(g.any()) for g in grads)


def test_parts_of_ranks_together(B):
    """A norm whose squares were added up over ranks; infinite elements of a tensor that the given sum knows nothing of stay infinite."""
    import torch
    rng = np.random.default_rng(8)
    ranks = [[_tensor(rng, n, "f32", 2.0) for n in (10, 5000)], [_tensor(rng, n, "bf16", 2.0) for n in (333, 9)]]
    total = sum(B.vl_grad_norm(r, scale=0.5).sum_squares for r in ranks)
    norm = ref.norm([g.double().cpu().numpy() for r in ranks for g in r], 0.5)
    for r in ranks:
        arrays = [g.double().cpu().numpy() for g in r]
        got = B.vl_clip_grads(r, 1.0, scale=0.5, sum_squares=total)
        assert abs(float(got.norm) - norm) <= 7 * U * norm
        for a, g in zip(arrays, r):
            want = a * 0.5 / norm
            assert np.all(np.abs(g.double().cpu().numpy() - want) <= (8 * U + HALF[_name(g)]) * 1.0001 * np.abs(want))
    g = torch.tensor([1.0, float("inf"), -float("inf")], device="cuda")
    B.vl_clip_grads([g], 1.0, sum_squares=torch.tensor(9.0, device="cuda", dtype=torch.float64))
    assert g.tolist()[1:] == [float("inf"), -float("inf")] and abs(g.tolist()[0] - 1 / 3) <= 2 * U


def test_matrices_streams_and_graphs(B):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    a = torch.randn(70, 90, generator=gen, device="cuda")
    grads = [a.t(), torch.randn(4, 5, 6, generator=gen, device="cuda").permute(2, 0, 1), torch.randn((), generator=gen, device="cuda")]
    _check(B, grads, 1.0, 2.0, outs=[torch.empty_like(g) for g in grads])
    with pytest.raises(B.VlError):
        B.vl_grad_norm([a[:, ::2]])
    want = [torch.empty_like(g) for g in grads]
    first = B.vl_clip_grads(grads, 2.0, outs=want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(g) for g in grads]
    torch.cuda.synchronize()
    got = B.vl_clip_grads(grads, 2.0, outs=outs, stream=side)
    side.synchronize()
    assert torch.equal(got.norm, first.norm) and all(torch.equal(x, y) for x, y in zip(outs, want))
    big = torch.randn(3000000, generator=gen, device="cuda")
    held, graph = big.clone(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.vl_clip_grads([held, grads[0]], 1.0, outs=[held, outs[0]])
    for k in (1.0, 3.0, 1e-6):
        held.copy_(big * k)
        graph.replay()
        fresh = (big * k).clone()
        again = B.vl_clip_grads([fresh, grads[0]], 1.0, outs=[fresh, torch.empty_like(grads[0])])
        assert torch.equal(got.norm, again.norm) and torch.equal(got.factor, again.factor) and torch.equal(held, fresh)


def test_equal_inputs_give_equal_results(B):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    grads = [torch.randn(n, generator=gen, device="cuda").to(torch.bfloat16) for n in (10, 400000, 7000001)]
    first = B.vl_grad_norm(grads)
    for _ in range(5):
        got = B.vl_grad_norm(grads)
        assert torch.equal(got.norm, first.norm) and torch.equal(got.sum_squares, first.sum_squares)
