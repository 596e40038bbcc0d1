"""8-bit operators: what they refuse, and that a call without tokens does nothing.  No GPU: every check comes before the first
CUDA call, pointers are made up and never read."""
import ctypes

import pytest
import torch

from paper_2507_17301_b200 import build

build.build()
from paper_2507_17301_b200 import nm  # noqa: E402

X, R, S, W, Q, SC = (0x10000000 * i for i in range(1, 7))   # made-up addresses, far apart
F32, BF16, F16 = 0, 1, 2


def rmsnorm(x=X, x_ld=64, r=R, r_ld=64, s=S, s_ld=64, w=W, t=BF16, wt=BF16, tokens=4, h=64, eps=1e-6, q=Q, q_ld=64, sc=SC):
    return nm._lib.nm_q8_rmsnorm(x, x_ld, r, r_ld, s, s_ld, w, t, wt, tokens, h, eps, q, q_ld, sc, None)


@pytest.mark.parametrize("change", [
    {"x": None}, {"w": None}, {"q": None}, {"sc": None}, {"r": None}, {"s": None}, {"t": 3}, {"wt": -1}, {"wt": F16}, {"tokens": -1}, {"h": 0},
    {"eps": 0.0}, {"eps": float("nan")}, {"eps": 2.0}, {"eps": -1e-6}, {"x_ld": 63}, {"r_ld": 0}, {"s_ld": 63}, {"q_ld": 48}, {"q_ld": 72},
    {"q": Q + 8}, {"x": X + 1}, {"w": W + 1}, {"sc": SC + 2}, {"s": X + 16}, {"s": R + 64, "s_ld": 65}, {"q": X}, {"q": S}, {"sc": Q + 64}, {"sc": X + 64},
    {"s": W}, {"q": W}, {"s": SC}, {"r_ld": 128, "s": R, "s_ld": 64},
])
def test_rmsnorm_refuses(change):
    assert rmsnorm(**change) == nm.NM_ERR_INVALID_ARG, change


def test_too_long_rows_are_refused():
    assert rmsnorm(h=65536, x_ld=65536, r_ld=65536, s_ld=65536, q_ld=65536) == nm.NM_ERR_UNSUPPORTED


def test_no_tokens_is_a_call_that_does_nothing():
    assert rmsnorm(tokens=0) == nm.NM_OK
    assert rmsnorm(tokens=0, x=None, r=None, s=None, w=None, q=None, sc=None) == nm.NM_OK
    assert nm._lib.nm_q8_rows(None, 0, F32, 0, 5, None, 0, None, None) == nm.NM_OK
    assert nm._lib.nm_q8_silu_mul(None, 0, None, 0, F32, 0, 5, None, 0, None, None) == nm.NM_OK


def test_silu_mul_and_rows_refuse():
    rows, silu = nm._lib.nm_q8_rows, nm._lib.nm_q8_silu_mul
    assert rows(X, 63, BF16, 2, 64, Q, 64, SC, None) == nm.NM_ERR_INVALID_ARG
    assert rows(X, 64, 7, 2, 64, Q, 64, SC, None) == nm.NM_ERR_INVALID_ARG
    assert rows(X, 64, F32, 2, 64, Q, 60, SC, None) == nm.NM_ERR_INVALID_ARG
    assert rows(X, 64, F32, 2, 64, X + 16, 64, SC, None) == nm.NM_ERR_INVALID_ARG
    assert silu(X, 64, None, 64, BF16, 2, 64, Q, 64, SC, None) == nm.NM_ERR_INVALID_ARG
    assert silu(X, 64, R, 32, BF16, 2, 64, Q, 64, SC, None) == nm.NM_ERR_INVALID_ARG
    assert silu(X, 64, R, 64, BF16, 2, 64, Q, 64, Q, None) == nm.NM_ERR_INVALID_ARG
    assert "overlaps" in nm.nm_last_error()


def test_weights_refuse():
    out = ctypes.c_void_p()
    prune = lambda *a: nm._lib.nm_q8_prune(*a, None, ctypes.byref(out))                      # noqa: E731
    load = lambda *a: nm._lib.nm_q8_weights_import(*a, None, ctypes.byref(out))              # noqa: E731
    assert prune(None, 8, 8, 2, 4, 8) == nm.NM_ERR_INVALID_ARG
    assert prune(X + 2, 8, 8, 2, 4, 8) == nm.NM_ERR_INVALID_ARG
    for bad in ((0, 8, 2, 4, 8), (8, 0, 2, 4, 8), (8, 8, 0, 4, 8), (8, 8, 5, 4, 8), (8, 8, 2, 4, 0)):
        assert prune(X, *bad) == nm.NM_ERR_INVALID_ARG
        assert load(X, R, S, *bad) == nm.NM_ERR_INVALID_ARG
    for big in ((8, 65536, 2, 4, 8), (8, 8, 2, 4, 257), (65536, 8, 2, 4, 1)):
        assert prune(X, *big) == nm.NM_ERR_UNSUPPORTED
        assert load(X, R, S, *big) == nm.NM_ERR_UNSUPPORTED
    for nulls in ((None, R, S), (X, None, S), (X, R, None), (X, R + 1, S), (X, R, S + 1)):
        assert load(*nulls, 8, 8, 2, 4, 8) == nm.NM_ERR_INVALID_ARG
    assert nm._lib.nm_q8_prune(X, 8, 8, 2, 4, 8, None, None) == nm.NM_ERR_INVALID_ARG
    assert nm._lib.nm_q8_weights_dims(None, None, None, None, None, None) == nm.NM_ERR_INVALID_ARG
    assert nm._lib.nm_q8_weights_export(None, None, None, None, None) == nm.NM_ERR_INVALID_ARG
    assert nm._lib.nm_q8_weights_check(None, None) == nm.NM_ERR_INVALID_ARG
    assert nm._lib.nm_q8_weights_free(None) == nm.NM_OK
    assert nm._lib.nm_q8_linear(None, X, 64, SC, 1, None, S, 64, F32, None) == nm.NM_ERR_INVALID_ARG


def test_a_handle_of_the_other_kind_is_refused():
    """The first word tells the kinds apart: a convolution's handle is no linear layer's."""
    other = (ctypes.c_uint32 * 256)(0x4E4D5754)
    assert nm._lib.nm_q8_linear(ctypes.addressof(other), X, 64, SC, 1, None, S, 64, F32, None) == nm.NM_ERR_INVALID_ARG
    assert "handle" in nm.nm_last_error()


class _Fake:
    """What nm_q8_linear looks at in a handle: magic, device, ..., c_out, k (see nm_q8.h)."""

    def __init__(self, c_out=128, k=96):
        self.mem = (ctypes.c_uint32 * 64)()
        self.mem[0], self.mem[1] = 0x4E4D5138, 0
        self.mem[6], self.mem[7] = c_out, k
        self.addr = ctypes.addressof(self.mem)


def test_linear_refuses():
    w = _Fake()
    out = [ctypes.c_int() for _ in range(5)]
    assert nm._lib.nm_q8_weights_dims(w.addr, *[ctypes.byref(d) for d in out]) == nm.NM_OK and [d.value for d in out[:2]] == [128, 96]
    call = lambda x=X, x_ld=96, xs=SC, tokens=3, bias=None, y=S, y_ld=128, t=F32: nm._lib.nm_q8_linear(w.addr, x, x_ld, xs, tokens, bias, y, y_ld, t, None)  # noqa: E731
    for bad in ({"x": None}, {"xs": None}, {"y": None}, {"t": 5}, {"tokens": -2}, {"x_ld": 80}, {"x_ld": 100}, {"x": X + 8}, {"y_ld": 127}, {"y": S + 2},
                {"xs": SC + 1}, {"bias": W + 2}, {"y": X + 64}, {"xs": S + 4}, {"bias": S + 512}, {"y": SC}):
        assert call(**bad) == nm.NM_ERR_INVALID_ARG, bad
    assert call(tokens=0) == nm.NM_OK and call(tokens=0, x=None, y=None, xs=None) == nm.NM_OK


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros(4, 64)
    for bad in (x, x.double(), None, 3, x[0]):
        with pytest.raises(TypeError, match="two-dimensional"):
            nm.nm_q8_rows(bad)
        with pytest.raises(TypeError, match="two-dimensional"):
            nm.nm_q8_silu_mul(bad, bad)
        with pytest.raises(TypeError, match="two-dimensional"):
            nm.nm_q8_rmsnorm(bad, x[0])
    w = nm.Q8Weights.__new__(nm.Q8Weights)
    w._h, w._addr, w.c_out, w.k = None, 0, 8, 64
    with pytest.raises(TypeError, match="xq must be"):
        nm.nm_q8_linear(w, x.to(torch.int8), x[:, 0])
    with pytest.raises(TypeError, match="w_dense"):
        nm.nm_q8_prune(x, 2, 4, 8)
    with pytest.raises(TypeError, match="values"):
        nm.nm_q8_weights_import(x.to(torch.int8), x[:, 0].contiguous(), x.to(torch.uint16), 64, 2, 4, 4)


def test_the_self_test_refuses_what_the_product_refuses():
    w = _Fake()
    call = lambda h=w.addr, x=X, x_ld=96, xs=SC, tokens=3, y=S, y_ld=128, block=0: nm._lib.nm_selftest_q8_wait_expiry(h, x, x_ld, xs, tokens, y, y_ld, block, None)  # noqa: E731
    for bad in ({"h": None}, {"block": -1}, {"x": None}, {"xs": None}, {"y": None}, {"tokens": -2}, {"x_ld": 80}, {"x": X + 8}, {"y_ld": 127}, {"y": X + 64}):
        assert call(**bad) == nm.NM_ERR_INVALID_ARG, bad
    assert call(tokens=0) == nm.NM_OK
