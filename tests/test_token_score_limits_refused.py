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
