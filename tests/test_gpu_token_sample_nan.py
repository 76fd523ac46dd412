"""Rows with an open entry that is no number, where nothing in its neighbourhood is possible: no token, ln p no number, whatever their length."""
import numpy as np
import pytest

from tests import score_oracle
from tests.test_gpu_token_sample import RULES, check
from tests.test_gpu_token_scores import DTYPES, B, _make, _rows  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


def _values(rng, V):
    """Row by row: nothing but NaN; NaN alone among impossible entries (first, last, in the middle); a quarter or an eighth impossible but for
    a NaN, the rest ordinary; the same with the NaN behind the ordinary ones; NaN from the middle on; and ordinary rows between them."""
    x = _make(rng, 10, V)
    x[0] = np.nan
    for r, i in ((1, 0), (2, V - 1), (3, V // 2)):
        x[r] = -np.inf
        x[r, i] = np.nan
    x[4, : V // 4] = -np.inf
    x[4, V // 8] = np.nan
    x[5, V // 2: V // 2 + V // 8] = -np.inf
    x[5, V // 2 + V // 16] = np.nan
    x[6, V - V // 4:] = -np.inf
    x[6, V - 1] = np.nan
    x[7, V // 2:] = np.nan
    return x


@pytest.mark.parametrize("V", [40, 700, 1025, 5000, 33000, 70001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_no_number_among_impossible_entries(B, dtype, V):
    import torch
    rng = np.random.default_rng(V)
    x = _rows(_values(rng, V), dtype, pad=V % 3)
    R = x.shape[0]
    for rules in RULES:
        u = rng.random(R).astype(np.float32)
        got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), **rules)
        check(got, x.double().cpu().numpy(), 1.0, np.zeros((R, V), bool), u, rules)


@pytest.mark.parametrize("V", [40, 700, 1025, 5000, 70001])
@pytest.mark.parametrize("dtype", DTYPES)
def test_no_number_among_closed_entries(B, dtype, V):
    """The same where a mask closes what lies around it; a NaN that is closed itself does not count."""
    import torch
    rng = np.random.default_rng(V + 1)
    R = 4
    x64 = _make(rng, R, V)
    taken = np.zeros((R, (V + 31) // 32 * 32), dtype=bool)
    taken[:2, : V // 2] = True
    taken[2:, V - V // 3: V] = True
    x64[0, V // 4] = np.nan                 # open
    taken[0, V // 4] = False
    x64[1, V // 4] = np.nan                 # closed
    x64[2, V - 1] = np.nan                  # open
    taken[2, V - 1] = False
    m = np.packbits(taken, axis=1, bitorder="little").view(np.uint32)
    closed = np.array([score_oracle.closed_entries(V, m[r], 1) for r in range(R)])
    x = _rows(x64, dtype)
    for rules in RULES:
        u = rng.random(R).astype(np.float32)
        got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), occupied=torch.from_numpy(m.view(np.int32)).cuda(), **rules)
        check(got, x.double().cpu().numpy(), 1.0, closed, u, rules)


@pytest.mark.parametrize("R,V", [(700, 2100), (600, 9000)])
def test_no_number_in_many_rows(B, R, V):
    """As many rows as a warp each takes."""
    import torch
    x = torch.randn(R, V, device="cuda", dtype=torch.float32, generator=torch.Generator(device="cuda").manual_seed(V)).to(torch.bfloat16)
    x[::3] = float("nan")
    x[1::3, V // 8: V // 4] = -float("inf")
    x[1::3, V // 6] = float("nan")
    u = torch.rand(R, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V))
    for rules in RULES:
        got = B.vl_token_sample(x, u, **rules)
        none = got.tokens == -1
        assert bool(none[::3].all()) and bool(none[1::3].all()) and not bool(none[2::3].any()), rules
        assert torch.equal(got.logprob.isnan(), none) and torch.equal(got.drawn_logprob.isnan(), none) and torch.equal(got.kept == 0, none), rules
