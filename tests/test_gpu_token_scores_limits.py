"""Scores of tokens and their gradient where sizes, values and streams reach their limits; tolerances as in tests/test_gpu_token_scores.py."""
import numpy as np
import pytest

from tests import score_oracle as ref
from tests.test_gpu_token_scores import B, _check_scores, _make, _masks, _rows  # noqa: F401 (B is a fixture)

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
