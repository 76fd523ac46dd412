"""Equal rows get equal results, bit for bit, where sums of 64 bits in another order would round to the other side of a border."""
import numpy as np
import pytest

from tests.test_gpu_token_scores import B  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,V", [(200, 9000), (200, 20000), (40, 60000)])
def test_borders_within_a_rounding(B, R, V):
    """The cut falls among 400 logits next to each other, all over the row; top_p is varied by half units of the last place around a border."""
    import torch
    rng = np.random.default_rng(V)
    row = rng.normal(0, 0.5, V).astype(np.float32)
    at = rng.permutation(V)[:400]
    row[at] = 0.5 + (1 + np.arange(400)) * np.float32(2.0 ** -23)
    w = np.exp(row.astype(np.float64) - float(row.max()))
    order = np.argsort(-row, kind="stable")
    sums = np.cumsum(w[order])
    middle = int(np.flatnonzero(row[order] <= 0.5 + 200 * 2.0 ** -23)[0])
    x = torch.from_numpy(row).cuda().repeat(R, 1)
    u = torch.full((R,), 0.37, device="cuda")
    share = sums[middle] / w.sum()
    for k in range(-60, 61):
        got = B.vl_token_sample(x, u, top_p=float(share * (1.0 + k * 2.0 ** -53)))
        for name, v in zip(got._fields, got):
            assert bool((v == v[0]).all()), (k, name, torch.unique(v).tolist())
