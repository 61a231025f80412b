"""What of windowed attention, the keys' weights and eviction needs no GPU: refusals before a device is touched, and the plain forms."""
import ctypes as C

import torch

import bounded_cache_ref as ref
from paper_2604_12056_b200 import binding as B


def test_calls_without_a_context_are_refused():
    from paper_2604_12056_b200 import build
    build.build()
    lib = B._typed_lib()
    q, kv, ev = C.byref(B.QueriesT()), C.byref(B.KvT()), C.byref(B.EvictionT())
    assert lib.losa_window_attn(None, q, kv, None, None, None) == B.LOSA_ERR_INVALID_ARG
    assert lib.losa_kv_weights(None, q, kv, None, 1.0, None, None) == B.LOSA_ERR_INVALID_ARG
    assert lib.losa_kv_evict(None, kv, None, ev, None) == B.LOSA_ERR_INVALID_ARG


def test_which_keys_a_token_sees():
    ok = ref.visible(3, 4, 9, 0, 0, 1)
    assert [int(r.sum()) for r in ok] == [4, 5, 6, 7]
    assert [j for j in range(9) if ref.visible(6, 1, 9, 3, 2, 1)[0, j]] == [0, 1, 4, 5, 6]
    assert [j for j in range(9) if ref.visible(4, 1, 9, 2, 0, 4)[0, j]] == [3, 4, 5, 6, 7]
    assert not ref.visible(50, 2, 9, 10, 0, 1).any() and ref.visible(50, 2, 9, 10, 3, 1).sum() == 6


def test_which_tokens_stay():
    assert ref.stays([5, 1, 1, 1, 9, 0], 4, 1, 1) == [0, 1, 4, 5]
    assert ref.stays([1.0, float("nan"), 7.0], 1, 0, 0) == [1]
    assert ref.stays([0.0, -0.0, 0.0], 2, 0, 0) == [0, 1]
    assert ref.stays([1, 2, 3, 4], 2, 5, 5) == [0, 1] and ref.stays([9, 9, 9, 9], 2, 0, 5) == [2, 3]


def test_the_plain_forms_agree_with_a_softmax():
    gen = torch.Generator().manual_seed(1)
    q, k, v = torch.randn(5, 2, 64, generator=gen).double(), torch.randn(9, 64, generator=gen).double(), torch.randn(9, 64, generator=gen).double()
    ok = ref.visible(4, 5, 9, 4, 1, 1)
    o, lse, *_ = ref.attention(q, k, v, ok, 0.125, True)
    s = (q @ k.T * 0.125).masked_fill(~ok[:, None], -float("inf"))
    assert torch.allclose(o, torch.softmax(s, -1) @ v)
    w, _ = ref.weights(q, k, ok, lse, 0.125, True)
    assert torch.allclose(w, torch.softmax(s, -1).sum((0, 1))) and torch.allclose(w.sum(), torch.tensor(10.0).double())
