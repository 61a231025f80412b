"""Windowed attention, weights and eviction together, and what the calls refuse (needs a B200)."""
import os
import sys

import pytest
import torch

import bounded_cache_ref as ref
from bounded_cache_ref import Cache

pytestmark = pytest.mark.gpu


def test_the_example_runs():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import bounded_cache
    out, merged, decoded, left = bounded_cache.run()
    assert all(x.isfinite().all() for x in (out, merged, decoded))
    # cut to 600 before every token but one behind, the short sequence grows
    assert left == [601, 37 + 32 + 4, 601]


@pytest.mark.parametrize("fmt", ["f32", "bf16", "fp8", "int4"])
def test_attend_weigh_evict_attend_again(fmt):
    """A run of the three: what is attended to after an eviction is what stayed, head by head."""
    lens, budgets = [500, 77, 300], [128, 77, 40]
    c = Cache(lens, fmt=fmt)
    c.tokens([20, 1, 300], [480, 76, 0])
    w = torch.zeros(c.kp.shape[0], c.hkv, c.g, device="cuda")
    assert c.attend(200, 4, 1) == 0
    c.check()
    c.B.losa_kv_weights(c.ctx, c.queries(200, 4, 1), c.kv, c.lse, w)
    length, budget = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, budgets))
    kept = torch.full((3, c.hkv, 128), -1, dtype=torch.int32, device="cuda")
    before = {n: c.rows(n) for n in "kv"}
    table = c.table.cpu().long()
    stay = [[ref.stays(w.cpu()[table[s, torch.arange(L) // c.g], h, torch.arange(L) % c.g].tolist(), b, 4, 16) if b < L else list(range(L)) for h in range(c.hkv)]
            for s, (L, b) in enumerate(zip(lens, budgets))]
    c.B.losa_kv_evict(c.ctx, c.kv, w, c.B.make_eviction(length, budget, kept, 4, 16))
    assert c.ctx.poll_status() == 0
    assert kept[0].tolist() == stay[0]
    c.lens = [min(a, b) for a, b in zip(lens, budgets)]
    for n in "kv":
        for s, x in enumerate(c.rows(n)):
            for h in range(c.hkv):
                want = before[n][s][stay[s][h], h]
                step = 2.0 ** -4 * want.abs() + 2.0 ** -10 * 2.0 ** 7 if fmt == "fp8" else 0.0       # (FP8 pages are quantised again: half a step, or half of the smallest at the largest scale)
                assert ((x[:, h] - want).abs() <= step).all()
    c.tokens([1, 1, 1], c.lens)
    assert c.attend(0, 0, 1) == 0
    c.check()


def test_refusals():
    c = Cache([100, 40], fmt="bf16")
    c.tokens([3, 2], [97, 38])
    B = c.B
    w, kept = torch.zeros(c.kp.shape[0], c.hkv, c.g, device="cuda"), torch.zeros(2, c.hkv, 50, dtype=torch.int32, device="cuda")
    length, budget = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([100, 40], [50, 40]))

    def code(f, *a):
        with pytest.raises(B.LosaError) as e:
            f(*a)
        return e.value.code

    for change in (dict(window=-1), dict(sinks=-1), dict(span=0), dict(span=65537), dict(max_tokens=0), dict(n_tokens=-1), dict(q=None), dict(cu=None), dict(start=None), dict(q_stride=8)):
        q = c.queries()
        for name, value in change.items():
            setattr(q, name, value)
        assert code(B.losa_window_attn, c.ctx, q, c.kv, c.out, c.lse) == B.LOSA_ERR_INVALID_ARG, change
        assert code(B.losa_kv_weights, c.ctx, q, c.kv, c.lse, w) == B.LOSA_ERR_INVALID_ARG, change
    q = c.queries()
    q.q += 8                                          # rows that are not aligned
    assert code(B.losa_window_attn, c.ctx, q, c.kv, c.out, c.lse) == B.LOSA_ERR_UNSUPPORTED
    q = c.queries()
    q.n_tokens = 2 * (c.pmax * c.g + 1) + 1           # more tokens than the context has room for
    assert code(B.losa_window_attn, c.ctx, q, c.kv, c.out, c.lse) == B.LOSA_ERR_UNSUPPORTED
    assert code(B.losa_window_attn, c.ctx, c.queries(), c.kv, c.q.contiguous(), c.lse) == B.LOSA_ERR_INVALID_ARG if c.q.is_contiguous() else True
    for keep in (-1.0, float("nan"), float("inf")):
        assert code(B.losa_kv_weights, c.ctx, c.queries(), c.kv, c.lse, w, keep) == B.LOSA_ERR_INVALID_ARG
    for change in (dict(length=None), dict(budget=None), dict(kept=None), dict(kept_stride=0), dict(sinks=-1), dict(recent=-1), dict(length=c.kv_len.data_ptr())):
        e = B.make_eviction(length, budget, kept)
        for name, value in change.items():
            setattr(e, name, value)
        assert code(B.losa_kv_evict, c.ctx, c.kv, w, e) == B.LOSA_ERR_INVALID_ARG, change
    kmin = torch.zeros(c.kp.shape[0], c.hkv, c.d, dtype=torch.bfloat16, device="cuda")
    assert code(B.losa_kv_evict, c.ctx, B.make_kv(c.kp, c.vp, kmin, None, c.table, c.kv_len), w, B.make_eviction(length, budget, kept)) == B.LOSA_ERR_INVALID_ARG
    launches = c.ctx.launch_count()
    assert code(B.losa_window_attn, c.ctx, q, c.kv, c.out, c.lse) == B.LOSA_ERR_UNSUPPORTED and c.ctx.launch_count() == launches
    assert c.attend() == 0
    c.check()


def test_no_tokens_at_all():
    c = Cache([100], fmt="bf16")
    c.tokens([0], [100])
    launches = c.ctx.launch_count()
    c.B.losa_window_attn(c.ctx, c.queries(), c.kv, c.out, c.lse)
    assert c.ctx.launch_count() == launches and c.ctx.poll_status() == 0


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "f32"])
def test_a_wait_that_runs_out_ends_the_calls(fmt):
    """A bound shorter than a look at a barrier: the tensor-core kernels give up, report it, and the context stays usable (fp32 has no such waits)."""
    c = Cache([700, 300], fmt=fmt)
    c.tokens([100, 1], [600, 299])
    w = torch.zeros(c.kp.shape[0], c.hkv, c.g, device="cuda")
    c.ctx.set_wait_limit(1)
    want = 0 if fmt == "f32" else c.B.LOSA_ERR_TIMEOUT
    assert c.attend(0, 0, 1) == want
    c.B.losa_kv_weights(c.ctx, c.queries(), c.kv, c.lse, w)
    assert c.ctx.poll_status() == want
    c.ctx.set_wait_limit(0)
    assert c.attend(0, 0, 1) == 0
    c.check()


def test_another_stream_and_outputs_aligned_to_16_bytes():
    c = Cache([400, 33], fmt="bf16")
    c.tokens([150, 1], [250, 32])
    buf = torch.empty(c.out.numel() + 8, dtype=torch.bfloat16, device="cuda")
    c.out = buf[8:].view(c.out.shape)                 # 16 bytes behind an aligned start
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert c.attend(100, 4, 1) == 0
    torch.cuda.current_stream().wait_stream(side)
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int4", "f32"])
def test_many_pieces_of_one_group_and_tokens_that_see_nothing(fmt):
    """Tiles of one group, of two, and without any, in all orders: the warps of a block run ahead of one another across them."""
    n = 250                                           # (a context has at most 1,024 sequences times KV heads)
    lens = [(0, 5, 130, 260, 0, 0, 0, 64)[i % 8] for i in range(n)]
    new = [(3, 1, 2, 40, 1, 1, 1, 64)[i % 8] for i in range(n)]
    c = Cache(lens, fmt=fmt, hkv=4, G=4, g=16, d=64)
    c.tokens(new, [0 if L == 0 else max(0, L - k) for L, k in zip(lens, new)])
    assert c.attend(0, 0, 1) == 0
    c.check()
