"""Drawing where min_p's border is a logit of 0: rows whose largest entry is 0, of either sign, against the plain 64-bit form (tokens and counts
equal, log probabilities within the bounds of tests/test_gpu_token_sample.py)."""
import numpy as np
import pytest

from tests.test_gpu_token_sample import check
from tests.test_gpu_token_scores import DTYPES, B, _rows  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu

RULES = [dict(min_p=1.0), dict(min_p=1.0, top_p=0.75), dict(min_p=1.0, top_k=5), dict(min_p=1.0, top_k=600), dict(min_p=1.0, top_k=600, top_p=0.5),
         dict(min_p=0.5), dict(min_p=0.5, top_p=0.75)]
NUMBERS = np.array([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 2.0 ** -149, 0.3], dtype=np.float32)   # borders of equal entries among them


def _zeros(kind, R, V):
    rng = np.random.default_rng(V + 1)
    if kind == "zero":
        x = np.zeros((R, V))
    elif kind == "signs":                       # both zeros
        x = rng.choice([0.0, -0.0], (R, V))
    else:                                       # some entries at 0, the rest below: a lowest number's distance, half a unit, three, impossible
        x = rng.choice([0.0, -0.0, -2.0 ** -24, -0.5, -3.0, -np.inf], (R, V))
        x[:, V // 2] = 0.0
    return x


@pytest.mark.parametrize("V", [1, 16, 250, 700, 1000, 1500, 5000, 40003])
@pytest.mark.parametrize("kind", ["zero", "signs", "below"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_largest_logit_of_zero(B, dtype, kind, V):
    import torch
    R = len(NUMBERS)
    x = _rows(_zeros(kind, R, V), dtype)
    for j, rules in enumerate(RULES):
        scale = (1.0, 0.7)[j % 2]
        got = B.vl_token_sample(x, torch.from_numpy(NUMBERS).cuda(), scale=scale, **rules)
        check(got, x.double().cpu().numpy(), scale, np.zeros((R, V), bool), NUMBERS, rules)


@pytest.mark.parametrize("V", [64, 2000])
def test_many_rows_of_zeros(B, V):
    """As many rows as there are entries, a number on each border: row r draws entry r."""
    import torch
    x = torch.zeros((V, V), device="cuda")
    u = torch.arange(V, device="cuda") / V
    at = torch.floor(u.double() * V).long()     # (a rounded quotient may lie just below its border)
    got = B.vl_token_sample(x, u, min_p=1.0)
    assert torch.equal(got.tokens, at) and bool((got.kept == V).all())
    assert torch.allclose(got.drawn_logprob.double(), torch.full((V,), -float(np.log(V)), device="cuda", dtype=torch.float64), rtol=1e-6)


@pytest.mark.parametrize("V", [16, 700, 5000])
def test_one_possible_entry_under_a_mask(B, V):
    """Log probabilities of a row with one possible register: 0 there, the rest closed."""
    import torch
    R = len(NUMBERS)
    x = torch.zeros((R, V), device="cuda")
    words = torch.full((R, (V + 31) // 32), -1, dtype=torch.int32, device="cuda")
    open_at = [(7 * r + 3) % V for r in range(R)]
    for r, i in enumerate(open_at):
        words[r, i // 32] = int(np.uint32(0xFFFFFFFF ^ (1 << i % 32)).view(np.int32))
    got = B.vl_token_sample(x, torch.from_numpy(NUMBERS).cuda(), occupied=words, min_p=1.0)
    assert got.tokens.tolist() == open_at and got.kept.tolist() == [1] * R
    assert got.logprob.tolist() == [0.0] * R and got.drawn_logprob.tolist() == [0.0] * R
