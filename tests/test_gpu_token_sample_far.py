"""Rows whose logits lie around the largest magnitude at which a product with the scale is rounded to less than an eighth of a power of two, on both
sides of it: 2^22 ln 2 / scale.  Against the plain 64-bit form, with the tolerances of tests/test_gpu_token_sample.py."""
import numpy as np
import pytest

from tests.test_gpu_token_sample import RULES, check
from tests.test_gpu_token_scores import B, _rows  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.0, 1e-3, 30.0])
@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("R,V", [(6, 300), (6, 5000), (6, 70001), (600, 1500)])
def test_logits_on_both_sides(B, R, V, sign, scale):
    """Parts of a row beyond it (a quarter, an eighth, all but a few entries), the rest a little short of it, one or two powers apart."""
    import torch
    rng = np.random.default_rng(V)
    limit = sign * 2.0 ** 22 * np.log(2.0) / scale
    step = float(np.spacing(np.float32(abs(limit))))
    near = limit + step * rng.integers(1, 9, (R, V))       # steps of a quarter or so, in units of 1 / scale
    far = limit - step * rng.integers(0, 9, (R, V))
    x64 = near.copy()
    for r in range(R):
        a, b = [(0, V // 4), (V // 2, V // 2 + V // 8), (0, V - V // 16), (V - V // 3, V), (0, 0), (0, V)][r % 6]
        x64[r, a:b] = far[r, a:b]
    x = _rows(x64, "f32")
    u = rng.random(R).astype(np.float32)
    for rules in RULES:
        got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), scale=scale, **rules)
        check(got, x.double().cpu().numpy(), scale, np.zeros((R, V), bool), u, rules, rows=range(min(R, 12)))


@pytest.mark.parametrize("V", [5000, 70001])
def test_logits_that_rise_across(B, V):
    """A warp's own entries cross the limit on the way."""
    import torch
    limit = -2.0 ** 22 * np.log(2.0)
    x64 = np.stack([limit + 0.25 * np.linspace(-40, 12, V).round(), limit + 0.25 * np.linspace(12, -40, V).round(),
                    limit + 0.25 * (np.arange(V) % 53 - 40)])
    x = _rows(x64, "f32")
    u = np.array([0.1, 0.6, 0.9], dtype=np.float32)
    for rules in RULES:
        got = B.vl_token_sample(x, torch.from_numpy(u).cuda(), **rules)
        check(got, x.double().cpu().numpy(), 1.0, np.zeros((3, V), bool), u, rules)
