"""Further refusals of the operators over logits and verdicts, before they touch a device."""
import ctypes as C

import pytest

from tests.test_token_score_refusals import B, _good  # noqa: F401 (B is a fixture)


@pytest.mark.parametrize("rows,stride,out_stride,by", [(2, 40, 40, 4), (2, 40, 40, 156), (2, 40, 40, 160), (3, 40, 40, 160), (2, 100, 100, 156), (2, 100, 100, -156),
                                                       (2, 100, 100, 244), (2, 100, 120, 160), (2, 120, 100, 160), (1, 40, 40, 156), (1, 40, 40, -156),
                                                       (3, 100, 100, 400), (3, 100, 100, -400), (3, 100, 100, 396), (2, 100, 100, 400)])
def test_gradients_that_overlap_the_logits(B, rows, stride, out_stride, by):
    """Matrices of 40 entries a row at the given strides, `by` bytes apart, that share entries."""
    at = 1 << 20
    taken = {at + 4 * (r * stride + i) for r in range(rows) for i in range(40)}
    shared = any(at + by + 4 * (r * out_stride + i) in taken for r in range(rows) for i in range(40))
    d = B.vl_logits(**{**_good(B), "logits": at, "n_rows": rows, "row_stride": stride, "n_masks": rows})
    assert shared or stride != out_stride
    assert B._lib.vl_token_logprobs_backward(0, C.byref(d), 4096, None, 4096, None, at + by, out_stride, None) == B.VL_ERR_INVALID_ARG


@pytest.mark.parametrize("rules", [dict(eps=1e-320), dict(eps=9e-101), dict(pair_cost=1.1e20), dict(pair_cost=-1e300), dict(bank_cost=1e308),
                                   dict(kl=1.1e30), dict(kl=-1e300)], ids=str)
def test_rules_out_of_range(B, rules):
    """Sizes whose squares, inverses or products leave the range of numbers: advantages of equal rewards would be none."""
    outs, K, size = (C.c_void_p * 1)(4096), (C.c_uint64 * 1)(3), B._lib.vl_policy_work(3, 10)
    r = B.vl_policy_rules(**{**dict(eps=1e-6, clip_lo=0.2, clip_hi=0.2, normalise=1), **rules})
    assert B._lib.vl_policy_loss(0, 1, outs, K, 4096, 10, 4096, None, 4096, C.byref(r), 4096, None, None, 4096, size, None) == B.VL_ERR_INVALID_ARG
