"""losa_rope_append and what goes with it where contexts, pointers or numbers are out of the ordinary (needs a B200)."""
import pytest
import torch

import cache_ops_ref as ref
from test_gpu_rope_append import KINDS, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_contexts_of_different_batches_in_turn(kv, dtype, d):
    """Contexts of 64, 2, 1000 and 1 sequences append, twice in turn: what one of them sets up must not refuse another's call."""
    cases = [Case([1 + i % 2 for i in range(n)], [i % 40 for i in range(n)], kv=kv, dtype=dtype, d=d, hq=1, hkv=1, seed=n) for n in (64, 2, 1000, 1)]
    for _ in range(2):
        for c in cases:
            assert c.run() == 0
    for c in cases[:2]:
        for t, old in zip((c.kp, c.vp, c.ks, c.vs, c.kmin, c.kmax), c.before):
            if t is not None:
                t.copy_(old)
        assert c.run() == 0
        c.check()


def held(codes, scales):
    """What 4-bit rows stand for, float64; scale byte 255: NaN."""
    x = ref.int4_value(ref.int4_unpack(codes.cpu()), scales.cpu().long().clamp(max=247))
    return torch.where((scales.cpu() == 255).repeat_interleave(32, -1), torch.nan, x)


@pytest.mark.parametrize("g,d,rot", [(16, 64, 0), (32, 128, 0), (32, 128, 64), (64, 128, 128)])
def test_nan_in_4_bit_pages_stays_visible(g, d, rot):
    """A run with a NaN is NaN in the cache and in k_out / v_out; every other run is as ever; the summaries pass over it."""
    kw = dict(kv="int4", g=g, d=d, rot=rot, hq=4, hkv=2)
    a, b = Case([g + 3], [5], **kw), Case([g + 3], [5], **kw)
    a.k[2, 1, 5] = torch.nan                          # (rotated, it takes its partner along, half the rotated part further on)
    a.v[g, 0, d - 1] = torch.nan
    a.v[3, 1, 33] = -torch.nan
    assert a.run() == 0 and b.run() == 0
    k_runs = {0} | ({(5 + rot // 2) // 32} if rot else set())
    bad_k, bad_v = (torch.zeros(g + 3, 2, d // 32, dtype=torch.bool) for _ in range(2))
    bad_k[2, 1, list(k_runs)] = True
    bad_v[g, 0, (d - 1) // 32] = bad_v[3, 1, 1] = True
    at = 5 + torch.arange(g + 3)
    phys, slot = a.table.cpu()[0].long()[at // g], at % g
    for bad, pool, scale, other, other_scale, out in ((bad_k, a.kp, a.ks, b.kp, b.ks, a.k_out), (bad_v, a.vp, a.vs, b.vp, b.vs, a.v_out)):
        codes, bytes_ = pool.cpu()[phys, :, slot], scale.cpu()[phys, :, slot]
        assert ((bytes_ == 255) == bad).all()
        same = ~bad
        assert (codes.unflatten(-1, (-1, 16))[same] == other.cpu()[phys, :, slot].unflatten(-1, (-1, 16))[same]).all()
        assert (bytes_[same] == other_scale.cpu()[phys, :, slot][same]).all()
        assert torch.equal(held(codes, bytes_).nan_to_num(nan=1e9), out.cpu().double().nan_to_num(nan=1e9))
    for page in sorted(set(phys.tolist())):
        n = g if page == int(a.table[0, 0]) else 8 if g + 8 < 2 * g else g
        x = held(a.kp[page], a.ks[page])[:, :n]
        assert (a.kmin[page].cpu().double() == x.nan_to_num(nan=torch.inf).amin(1)).all() and (a.kmax[page].cpu().double() == x.nan_to_num(nan=-torch.inf).amax(1)).all()


def test_nan_in_a_bf16_cache_turned_into_4_bits_reaches_the_attention():
    from paper_2604_12056_b200 import binding as B
    g, d, hkv, L = 32, 128, 2, 70
    c = Case([1], [L - 1], kv="native", g=g, d=d, hkv=hkv, hq=8, extra_pages=0)
    n_phys = c.kp.shape[0]
    c.kp[c.table[0, 1].long(), 0, 7, 40] = torch.nan   # KV head 0: a key; KV head 1: a value
    c.vp[c.table[0, 2].long(), 1, 5, 100] = torch.nan
    c.kp[c.table[0, 2].long(), 1, 6] = torch.nan       # past the end: nothing to see
    codes = [torch.zeros((n_phys, hkv, g, d // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((n_phys, hkv, g, d // 32), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    kv_len = torch.tensor([L], dtype=torch.int32, device="cuda")
    dst = B.make_kv(*codes, c.kmin, c.kmax, c.table, kv_len, *scales)
    B.losa_quantize_kv_pages(c.ctx, B.make_kv(c.kp, c.vp, c.kmin, c.kmax, c.table, kv_len), dst)
    assert c.ctx.poll_status() == 0
    assert int((scales[0][c.table[0, 1].long()] == 255).sum()) == 1 and int((scales[1][c.table[0, 2].long(), :, :6] == 255).sum()) == 1
    for block in (1, 3, 32):
        ctx = B.Context(1, 8, hkv, d, block, g, c.table.shape[1], B.LOSA_BF16, d ** -0.5)
        q = torch.randn(1, block, 8, d, device="cuda").bfloat16()
        out, lse = torch.zeros_like(q), torch.zeros(1, block, 8, device="cuda")
        B.losa_int4_attn(ctx, q, dst, out, lse)
        assert ctx.poll_status() == 0
        assert out[:, :, :4].isnan().all() and lse[:, :, :4].isnan().all()
        bad = torch.zeros(d, dtype=torch.bool, device="cuda")
        bad[96:] = True
        assert (out[:, :, 4:].isnan() == bad).all() and lse[:, :, 4:].isfinite().all()


@pytest.mark.parametrize("kv,dtype", KINDS)
@pytest.mark.parametrize("g,d", [(16, 64), (32, 128), (64, 128)])
def test_summaries_beside_nan_are_those_of_the_cache(kv, dtype, g, d):
    """NaN in single columns of single tokens, one column with NaN alone: an append leaves the summaries that
    losa_build_page_summaries makes of the same pages."""
    c = Case([3, 2 * g, 1], [0, g - 5, g], kv=kv, dtype=dtype, g=g, d=d, rot=0)
    c.k[1, 0, 0] = c.k[2, 1, 9] = c.k[5, 0, 16] = torch.nan
    c.k[:3, 0, 8] = torch.nan                         # all tokens of the first page
    assert c.run() == 0
    got = c.kmin.clone(), c.kmax.clone()
    # (rows before the appended ones are part of the cache; pages that no token touched stay as they were)
    c.B.losa_build_page_summaries(c.ctx, c.kv)
    assert c.ctx.poll_status() == 0
    for s, (a, n) in enumerate(zip(c.start, c.new)):
        for p in range(a // g, (a + n - 1) // g + 1):
            phys = int(c.table[s, p])
            assert torch.equal(got[0][phys], c.kmin[phys]) and torch.equal(got[1][phys], c.kmax[phys])


@pytest.mark.parametrize("which", [0, 1])
def test_a_block_at_an_odd_address_is_refused_by_4_bit_finalisation(which):
    c = Case([8, 8], [5, 0], kv="int4", rot=0, packed=False)
    B = c.B
    ctx = B.Context(2, c.hq, c.hkv, c.d, 8, c.g, c.table.shape[1], B.LOSA_BF16, 0.1)
    one = torch.ones(2, dtype=torch.int32, device="cuda")
    state = B.make_state(c.q_out, c.q_out.float(), one.float(), one)
    c.kv_len.copy_(c.st)
    rows = [c.k.data_ptr(), c.v.data_ptr()]
    rows[which] += 2                                  # (still inside the tensor's first rows; refused before anything is read)
    launched = ctx.launch_count()
    with pytest.raises(B.LosaError) as e:
        B.losa_update_prefix_cache(ctx, c.kv, state, None, *rows, True)
    assert e.value.code == B.LOSA_ERR_UNSUPPORTED and ctx.launch_count() == launched
    assert (c.kv_len == c.st).all() and (one == 1).all()
    B.losa_update_prefix_cache(ctx, c.kv, state, None, c.k, c.v, True)
    assert ctx.poll_status() == 0
    c.q_out = c.k_out = None
    c.check()


@pytest.mark.parametrize("kv,dtype", KINDS)
def test_outputs_over_their_inputs(kv, dtype):
    """Contiguous rows may be replaced by what the cache holds of them; rows that lie apart would be overwritten before they are read."""
    from paper_2604_12056_b200 import binding as B
    new, start = [70, 1, 200], [3, 64, 31]
    a, b = (Case(new, start, kv=kv, dtype=dtype, g=64, packed=False) for _ in range(2))
    assert b.run() == 0
    B.losa_rope_append(a.ctx, a.kv, a.rope, B.make_new_tokens(a.q, a.k, a.v, a.cu, a.st, None, a.q, a.k, a.v))
    assert a.ctx.poll_status() == 0
    for x, y in ((a.q, b.q_out), (a.k, b.k_out), (a.v, b.v_out), (a.kp, b.kp), (a.vp, b.vp)):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
    c = Case(new, start, kv=kv, dtype=dtype)           # rows side by side with the others'
    launched = c.ctx.launch_count()
    for name in "qkv":
        t = B.make_new_tokens(c.q, c.k, c.v, c.cu, c.st, None, c.q_out, c.k_out, c.v_out)
        setattr(t, name + "_out", getattr(t, name))
        with pytest.raises(B.LosaError) as e:
            B.losa_rope_append(c.ctx, c.kv, c.rope, t)
        assert e.value.code == B.LOSA_ERR_INVALID_ARG
    assert c.ctx.launch_count() == launched


@pytest.mark.parametrize("kv,dtype,g,T", [("native", "bf16", 32, 8200), ("native", "f32", 32, 4100), ("int4", "bf16", 16, 8200), ("fp8", "bf16", 64, 2100), ("fp8", "bf16", 32, 2100)])
@pytest.mark.parametrize("pairs", [False, True])
def test_prompts_whose_pages_and_queries_are_two_launches(kv, dtype, g, T, pairs):
    """Just beyond 64 MB of queries (FP8: 16 MB), a ragged batch with starts inside pages, an empty sequence and one of a single token."""
    new = [T // 2 - 3, 0, 1, T // 4 + 5, 9]
    new.append(T - sum(new))
    start = [7, 3, g - 1, 2 * g + 5, 5, 0]
    c = Case(new, start, kv=kv, dtype=dtype, g=g, hq=32, hkv=2, rot=96, interleaved=pairs, seed=T)
    launched = c.ctx.launch_count()
    assert c.run() == 0 and c.ctx.launch_count() == launched + 2
    c.check()


def test_the_larger_launch_below_the_limits_is_one():
    for kv, T in (("int4", 8190), ("fp8", 2040)):
        c = Case([T - 50, 50], [9, 40], kv=kv, hq=32, hkv=2, rot=64, g=32, outs=True)
        launched = c.ctx.launch_count()
        assert c.run() == 0 and c.ctx.launch_count() == launched + 1
        c.check()


@pytest.mark.parametrize("kv,T", [("native", 8200), ("fp8", 2100)])
def test_two_launches_leave_alone_what_does_not_fit(kv, T):
    from paper_2604_12056_b200 import binding as B
    new, start = [T - 40, 30, 10], [5, 90, 0]
    c = Case(new, start, kv=kv, hq=32, hkv=2, g=32, n_pos=T - 35)
    c.st[1] = T                                        # past the rotation table and the row of pages
    c.start[1] = T
    assert c.run() == B.LOSA_ERR_BOUNDS
    c.check(skipped=(1,))
