"""What the operators over logits and verdicts refuse, before they touch a device."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2506_17506_b200 import build
    build.build()
    from paper_2506_17506_b200 import binding
    return binding


def _good(B):
    return dict(logits=4096, dtype=B.VL_F32, n_rows=2, n_vocab=40, row_stride=40, tokens=4096, token_bytes=8, occupied=4096, n_masks=2,
                mask_rows=None, widths=4097, scale=1.0)


BAD = [dict(logits=None), dict(logits=4098), dict(dtype=3), dict(dtype=-1), dict(n_vocab=0), dict(n_vocab=(1 << 30) + 1, row_stride=1 << 31),
       dict(row_stride=39), dict(n_rows=(1 << 40) + 1), dict(n_rows=1 << 30, n_masks=1 << 30, row_stride=1 << 30), dict(token_bytes=1), dict(tokens=4100), dict(occupied=4097), dict(mask_rows=4098),
       dict(occupied=None, mask_rows=4096), dict(n_masks=1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
       dict(scale=float("inf"))]


@pytest.mark.parametrize("change", BAD, ids=lambda c: ",".join(c))
def test_bad_descriptors(B, change):
    d = B.vl_logits(**{**_good(B), **change})
    assert B._lib.vl_token_logprobs(0, C.byref(d), 4096, 4096, 4096, 0, None, None, None) == B.VL_ERR_INVALID_ARG
    assert B._lib.vl_token_logprobs_backward(0, C.byref(d), 4096, None, 4096, None, 8192, 40, None) == B.VL_ERR_INVALID_ARG


def test_bad_outputs(B):
    f, h = B._lib.vl_token_logprobs, B._lib.vl_token_logprobs_backward
    bad = B.VL_ERR_INVALID_ARG
    d = B.vl_logits(**_good(B))
    r = C.byref(d)
    assert f(0, None, 4096, 4096, 4096, 0, None, None, None) == bad
    assert f(0, r, 4097, 4096, 4096, 0, None, None, None) == bad
    assert f(0, r, 4096, 4098, 4096, 0, None, None, None) == bad
    assert f(0, r, 4096, 4096, 4100, 0, None, None, None) == bad            # statistics: pairs
    assert f(0, r, 4096, 4096, 4096, 33, 4096, 4096, None) == bad
    assert f(0, r, 4096, 4096, 4096, 2, None, 4096, None) == bad
    assert f(0, r, 4096, 4096, 4096, 2, 4096, None, None) == bad
    assert h(0, r, None, None, 4096, None, 8192, 40, None) == bad
    assert h(0, r, 4096, None, 4096, None, None, 40, None) == bad
    assert h(0, r, 4096, None, 4096, None, 8194, 40, None) == bad
    assert h(0, r, 4096, None, 4096, None, 8192, 39, None) == bad
    assert h(0, r, 4096, None, 4096, 4096, 8192, 40, None) == bad           # a gradient of the entropy without the entropy
    assert h(0, r, 4096, None, 4096, None, 4096, 48, None) == bad           # in place with another stride
    d = B.vl_logits(**{**_good(B), "tokens": None})
    assert f(0, C.byref(d), 4096, 4096, 4096, 0, None, None, None) == bad   # ln p of which tokens?
    assert h(0, C.byref(d), 4096, None, 4096, None, 8192, 40, None) == bad
    d = B.vl_logits(**{**_good(B), "n_rows": 0, "n_masks": 0, "logits": None})
    assert f(0, C.byref(d), None, None, None, 0, None, None, None) == B.VL_OK
    assert h(0, C.byref(d), None, None, None, None, None, 40, None) == B.VL_OK


def test_bad_policy_calls(B):
    f = B._lib.vl_policy_loss
    bad = B.VL_ERR_INVALID_ARG
    outs, K = (C.c_void_p * 2)(4096, 8192), (C.c_uint64 * 2)(3, 2)
    size = B._lib.vl_policy_work(5, 100)
    good = dict(n=2, out=outs, K=K, off=4096, T=100, lp=4096, old=None, ref=None, loss=4096, adv=None, g=None, work=4096, size=size)

    def call(rules=None, **change):
        a = {**good, **change}
        r = B.vl_policy_rules(**{**dict(eps=1e-6, clip_lo=0.2, clip_hi=0.2, normalise=1), **(rules or {})})
        return f(0, a["n"], a["out"], a["K"], a["off"], a["T"], a["lp"], a["old"], a["ref"], None if rules is False else C.byref(r),
                 a["loss"], a["adv"], a["g"], a["work"], a["size"], None)

    for change in (dict(out=None), dict(K=None), dict(off=None), dict(off=4100), dict(T=(1 << 40) + 1), dict(lp=None), dict(lp=4097),
                   dict(old=4098), dict(ref=4097), dict(loss=None), dict(loss=4097), dict(adv=4098), dict(g=4097), dict(work=None),
                   dict(work=4100), dict(size=size - 1), dict(out=(C.c_void_p * 2)(4096, None)), dict(out=(C.c_void_p * 2)(4096, 4104)),
                   dict(K=(C.c_uint64 * 2)(3, 1 << 40))):
        assert call(**change) == bad, change
    nan, inf = float("nan"), float("inf")
    for rules in (dict(eps=0.0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(clip_lo=-0.1), dict(clip_hi=-0.1), dict(clip_lo=nan),
                  dict(clip_hi=nan), dict(kl=0.1), dict(kl=nan), dict(kl=inf), dict(pair_cost=nan), dict(bank_cost=inf)):
        assert call(rules) == bad, rules
    assert f(0, 2, outs, K, 4096, 100, 4096, None, None, None, 4096, None, None, 4096, size, None) == bad
    assert B._lib.vl_policy_work(0, 0) > 0


def test_the_binding_refuses_host_tensors(B):
    import torch
    with pytest.raises(B.VlError):
        B.vl_token_logprobs(torch.zeros(2, 4))
    with pytest.raises(B.VlError):
        B.vl_token_logprobs_backward(torch.zeros(2, 4), None, torch.zeros(2, 2))
    with pytest.raises(B.VlError):
        B.vl_policy_loss([], torch.zeros(1, dtype=torch.int64), torch.zeros(3))
