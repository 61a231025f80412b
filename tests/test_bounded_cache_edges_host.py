"""What the calls on a bounded cache refuse at their edges, seen without a GPU."""
import ctypes as C

import pytest
import torch

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

    def ctx(self):
        class Ctx:
            _h, shape, _check = C.c_void_p(self.handle), B.ShapeT.from_address(self.handle), B.Context._check
            _queries, _kv_heads = (8, 128, torch.bfloat16, 2), (2, 2)
        return Ctx()


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

    layer = LosaLayer.__new__(LosaLayer)
    layer.ctx, layer.kv = h.ctx(), h.kv
    monkeypatch.setattr(B, "_stream", lambda: None)
    eviction = B.EvictionT(h.q, h.out, h.lse, 5, 0, 0)
    eviction._of = (2, 2)
    with pytest.raises(B.LosaError) as e:
        layer.evict(eviction)
    assert e.value.code == B.LOSA_ERR_INVALID_ARG


def test_tensors_of_another_shape_than_the_contexts_are_refused(lib, monkeypatch):
    """Heads, their size, type or number of sequences that are not the context's would be read and written past their ends."""
    h = Host()
    monkeypatch.setattr(B, "_stream", lambda: None)
    monkeypatch.setattr(B, "_ptr", lambda t: None if t is None else 4096)
    weights, bf16 = torch.empty(40, 2, 32), torch.bfloat16

    def calls(shape=(3, 8, 128), dtype=bf16, sequences=2, kept=(2, 2, 5)):
        """Whether each of the three calls comes as far as the library, which refuses its null pointers."""
        q = torch.empty(shape, dtype=dtype)
        queries, eviction = B.QueriesT(None, 0, None, None, 3, 3, 0, 0, 1), B.EvictionT(None, None, None, 5, 0, 0)
        queries._keep, queries._of = (q, None, None), (*shape[1:], dtype, sequences)
        eviction._of = kept[:2]
        lse = torch.empty(shape[:2])
        for call in (lambda: B.losa_window_attn(h.ctx(), queries, h.kv, q, lse), lambda: B.losa_kv_weights(h.ctx(), queries, h.kv, lse, weights),
                     lambda: B.losa_kv_evict(h.ctx(), h.kv, weights, eviction)):
            try:
                call()
            except B.LosaError as e:
                assert e.code == B.LOSA_ERR_INVALID_ARG
                yield True
            except AssertionError:
                yield False

    assert [*calls()] == [True, True, True]
    for wrong in (dict(shape=(3, 4, 128)), dict(shape=(3, 8, 64)), dict(dtype=torch.float32), dict(sequences=1), dict(sequences=3)):
        assert [*calls(**wrong)] == [False, False, True], wrong
    for kept in ((2, 1, 5), (1, 2, 5)):
        assert [*calls(kept=kept)] == [True, True, False]
