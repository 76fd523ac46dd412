"""What drawing tokens and clipping gradients refuse, before they touch a device."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2506_17506_b200 import build
    build.build()
    from paper_2506_17506_b200 import binding
    return binding


def _logits(B, **change):
    return B.vl_logits(**{**dict(logits=4096, dtype=B.VL_F32, n_rows=2, n_vocab=40, row_stride=40, scale=1.0), **change})


def test_bad_draws(B):
    nan, inf = float("nan"), float("inf")

    def call(rules=(0, 1.0, 0.0), uniform=4096, tokens=4096, size=8, lp=4096, drawn=None, kept=None, work=4096, bytes_=64, **change):
        d = _logits(B, **change)
        r = None if rules is None else C.byref(B.vl_sampling(*rules))
        return B._lib.vl_token_sample(0, C.byref(d), r, uniform, tokens, size, lp, drawn, kept, work, bytes_, None)

    bad = B.VL_ERR_INVALID_ARG
    for rules in (None, (0, 0.0, 0.0), (0, -0.5, 0.0), (0, 1.0001, 0.0), (0, nan, 0.0), (0, 1.0, -0.1), (0, 1.0, 1.5), (0, 1.0, nan), (0, inf, 0.0)):
        assert call(rules) == bad, rules
    for change in (dict(uniform=None), dict(uniform=4097), dict(tokens=None), dict(tokens=4100), dict(size=1), dict(size=0), dict(size=16),
                   dict(size=2, tokens=4097), dict(lp=4097), dict(work=None, n_vocab=1021, row_stride=2000), dict(bytes_=7, n_vocab=1021, row_stride=2000), dict(work=4098, n_vocab=1021, row_stride=2000), dict(drawn=4098), dict(kept=4097), dict(scale=0.0), dict(scale=nan), dict(logits=None),
                   dict(row_stride=39), dict(dtype=7), dict(n_vocab=0), dict(size=2, n_vocab=65536, row_stride=65536)):
        assert call(**change) == bad, change
    d = _logits(B, tokens=4096, token_bytes=8)
    assert B._lib.vl_token_sample(0, C.byref(d), C.byref(B.vl_sampling(0, 1.0, 0.0)), 4096, 4096, 8, None, None, None, 4096, 64, None) == bad
    assert B._lib.vl_token_sample(0, None, C.byref(B.vl_sampling(0, 1.0, 0.0)), 4096, 4096, 8, None, None, None, 4096, 64, None) == bad
    assert call(n_rows=0, logits=None, uniform=None, tokens=None, lp=None, work=None) == B.VL_OK


def _tensors(B, *items):
    return (B.vl_gradient * max(len(items), 1))(*[B.vl_gradient(*i) for i in items])


def test_bad_gradients(B):
    nan, inf = float("nan"), float("inf")
    bad = B.VL_ERR_INVALID_ARG
    size = B._lib.vl_grad_work(2)
    good = [(4096, 8192, 16, 0), (16384, 16384, 100, 2)]

    def norm(items=good, n=None, scale=1.0, out=4096, squares=4096, work=65536, bytes_=size):
        return B._lib.vl_grad_norm(0, len(items) if n is None else n, _tensors(B, *items), scale, out, squares, work, bytes_, None)

    def clip(items=good, n=None, scale=1.0, most=1.0, given=None, out=4096, factor=4096, work=65536, bytes_=size):
        return B._lib.vl_clip_grads(0, len(items) if n is None else n, _tensors(B, *items), scale, most, given, out, factor, work, bytes_, None)

    for call in (norm, clip):
        for change in (dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf), dict(scale=1e-19), dict(scale=1e19), dict(work=None),
                       dict(work=65544), dict(bytes_=size - 1), dict(out=4097), dict(items=[(None, 4096, 3, 0)]), dict(items=[(4098, 4096, 3, 0)]),
                       dict(items=[(4097, 4096, 3, 1)]), dict(items=[(4096, 4096, 3, 3)]), dict(items=[(4096, 4096, 3, -1)]),
                       dict(items=[(4096, 4096, (1 << 40) + 1, 0)])):
            assert call(**change) == bad, change
    assert norm(squares=4100) == bad
    assert B._lib.vl_grad_norm(0, 1, None, 1.0, 4096, 4096, 65536, size, None) == bad
    for change in (dict(most=-1.0), dict(most=nan), dict(given=4100), dict(factor=4098), dict(items=[(4096, None, 3, 0)]), dict(items=[(4096, 8194, 3, 0)])):
        assert clip(**change) == bad, change
    # results that share bytes: with each other, with their own tensor at another place, with another tensor, one tensor twice
    for items in ([(4096, 8192, 16, 0), (16384, 8192 + 60, 16, 0)], [(4096, 4100, 16, 0)], [(4096, 4096, 16, 0), (16384, 4096 + 60, 1, 0)],
                  [(4096, 4096, 16, 0), (4096, 4096, 16, 0)], [(4096, 8192, 16, 0), (8192 + 32, 16384, 16, 1)],
                  [(4096 * k, 4096 * k, 16, 0) for k in range(1, 70)] + [(4096 * 33 + 32, 4096 * 80, 16, 0)]):
        assert clip(items, bytes_=1 << 20) == bad, items
    assert B._lib.vl_grad_work(0) > 0 and B._lib.vl_grad_work(10000) > B._lib.vl_grad_work(10)


def test_the_binding_refuses(B):
    import torch
    with pytest.raises(B.VlError):
        B.vl_token_sample(torch.zeros(2, 4), torch.zeros(2))
    with pytest.raises(B.VlError):
        B.vl_grad_norm([torch.zeros(2)])
    with pytest.raises(B.VlError):
        B.vl_clip_grads([torch.zeros(2)], 1.0)
    with pytest.raises(B.VlError):
        B.vl_clip_grads([torch.zeros(2, dtype=torch.int32)], 1.0)
