"""What the calls on a bounded cache refuse at their edges, seen without a GPU."""
import ctypes as C

import pytest

from paper_2604_12056_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    from paper_2604_12056_b200 import build
    build.build()
    return B._typed_lib()


class Host:
    """A context that has met no device (a handle is the shape and zeros behind it), a cache and queries of addresses that nobody reads: for refusals."""

    def __init__(self, dtype=B.LOSA_BF16, kv_format=B.LOSA_KV_NATIVE):
        self.memory = (C.c_char * 65536)()
        self.handle = (C.addressof(self.memory) + 63) // 64 * 64
        shape = B.ShapeT(2, 8, 2, 128, 8, 32, 16, dtype, 0.1)
        C.memmove(self.handle, C.addressof(shape), C.sizeof(shape))
        at = [4096 * (i + 1) for i in range(12)]
        self.kv = B.KvT(at[0], at[1], 2 * 32 * 128, 32 * 128, 128, None, None, at[2], at[3], 40, kv_format, at[4], at[5])
        self.queries = B.QueriesT(None, 0, at[6], at[7], 0, 0, 0, 0, 1)
        self.q, self.out, self.lse, self.weights = at[8:]


@pytest.mark.parametrize("dtype,kv_format", [(B.LOSA_F32, B.LOSA_KV_NATIVE), (B.LOSA_BF16, B.LOSA_KV_NATIVE), (B.LOSA_BF16, B.LOSA_KV_FP8_E4M3), (B.LOSA_BF16, B.LOSA_KV_INT4)])
@pytest.mark.parametrize("most", [-1, -2 ** 31])
def test_fewer_than_no_tokens_are_refused_also_where_there_are_none(lib, dtype, kv_format, most):
    """max_tokens below zero: a call without tokens would take it for a count."""
    h = Host(dtype, kv_format)
    assert lib.losa_window_attn(h.handle, C.byref(h.queries), C.byref(h.kv), None, None, None) == B.LOSA_OK          # (no tokens, none at most)
    h.queries.max_tokens = most
    assert lib.losa_window_attn(h.handle, C.byref(h.queries), C.byref(h.kv), None, None, None) == B.LOSA_ERR_INVALID_ARG
    assert lib.losa_kv_weights(h.handle, C.byref(h.queries), C.byref(h.kv), None, 1.0, h.weights, None) == B.LOSA_ERR_INVALID_ARG
    h.queries.n_tokens, h.queries.q = 1, h.q
    assert lib.losa_window_attn(h.handle, C.byref(h.queries), C.byref(h.kv), h.out, None, None) == B.LOSA_ERR_INVALID_ARG
    assert lib.losa_kv_weights(h.handle, C.byref(h.queries), C.byref(h.kv), h.lse, 1.0, h.weights, None) == B.LOSA_ERR_INVALID_ARG


def test_a_layer_without_weights_is_refused(lib, monkeypatch):
    """LosaLayer.evict before any add_weights: the library's refusal, not a missing attribute."""
    from paper_2604_12056_b200.layer import LosaLayer
    h = Host()

    class Ctx:
        _h, shape, _check = C.c_void_p(h.handle), B.ShapeT.from_address(h.handle), B.Context._check

    layer = LosaLayer.__new__(LosaLayer)
    layer.ctx, layer.kv = Ctx(), h.kv
    monkeypatch.setattr(B, "_stream", lambda: None)
    with pytest.raises(B.LosaError) as e:
        layer.evict(B.EvictionT(h.q, h.out, h.lse, 5, 0, 0))
    assert e.value.code == B.LOSA_ERR_INVALID_ARG
