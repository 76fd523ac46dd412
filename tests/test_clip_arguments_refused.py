"""Lists of gradients, of results and sums that hold something else than tensors are refused like other bad arguments."""
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2506_17506_b200 import build
    build.build()
    from paper_2506_17506_b200 import binding
    return binding


@pytest.mark.parametrize("where", [0, 1])
@pytest.mark.parametrize("other", [None, 1.0, "x"])
def test_no_tensor_among_the_gradients(B, where, other):
    import torch
    grads = [torch.zeros(3), torch.zeros(5)]
    grads[where] = other                    # [p.grad for p in ...] of a parameter that was not used
    for call in (lambda g: B.vl_grad_norm(g), lambda g: B.vl_clip_grads(g, 1.0), lambda g: B.vl_clip_grads(iter(g), 1.0)):
        with pytest.raises(B.VlError, match="grads"):
            call(grads)


@pytest.mark.gpu
def test_on_the_device(B):
    import torch
    a, b = torch.ones(3, device="cuda"), torch.ones(5, device="cuda")
    for grads in ([None, a], [a, None], [a, 2.0]):
        with pytest.raises(B.VlError, match="grads"):
            B.vl_clip_grads(grads, 1.0)
    for outs in ([None, b], [a, None], [a], 7, [a.tolist(), b]):
        with pytest.raises(B.VlError, match="outs"):
            B.vl_clip_grads([a, b], 1.0, outs=outs)
    for total in (4.0, "x", torch.ones(1), torch.ones(2, dtype=torch.float64, device="cuda")):
        with pytest.raises(B.VlError, match="sum_squares"):
            B.vl_clip_grads([a, b], 1.0, sum_squares=total)
    assert bool((a == 1).all()) and bool((b == 1).all())
    got = B.vl_clip_grads([a, b], 2.0, outs=iter([torch.empty_like(a), torch.empty_like(b)]))
    assert len(got.outs) == 2 and float((got.outs[0] - 2.0 / 8 ** 0.5).abs().max()) <= 8 * 2.0 ** -24    # the norm's error, and a rounding
