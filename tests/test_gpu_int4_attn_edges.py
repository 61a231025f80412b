"""Attention over a 4-bit cache where rows or numbers are out of the ordinary, against the plain 64-bit form (needs a B200)."""
import pytest
import torch

import cache_ops_ref as ref
from test_gpu_int4_attn import Cache

pytestmark = pytest.mark.gpu

# few and many query rows per KV head, by eight, by sixteen, by 128 and with a row group that is not full
ROWS = [(1, 4), (3, 5), (5, 5), (32, 4), (33, 4)]


def dev(*a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("g,d", [(32, 64), (32, 128), (16, 128)])
@pytest.mark.parametrize("block,G", [(5, 5), (9, 5), (31, 3), (33, 4)])
def test_partly_filled_warps_with_tokens_that_do_not_exist(block, G, g, d):
    """The lanes of one warp find rows, no rows and rows of tokens outside the block: reported, and the others' results are right,
    in segments of one CTA and of several."""
    lens = [40, 9011]
    c = Cache(lens, block=block, G=G, g=g, d=d, hkv=2, seed=block)
    B, N, pmax = c.B, 2, c.table.shape[1]
    act = torch.arange(block, dtype=torch.int32, device="cuda").repeat(N, 1)
    act[:, 1::4] = block + 7                          # every fourth entry: no such token
    act[:, 3::8] = -5
    good = [t for t in range(block) if int(act[0, t]) == t]
    pages = torch.arange(pmax, dtype=torch.int32, device="cuda").repeat(N, c.hkv, 1).contiguous()
    count = torch.tensor([[-(-L // g)] * c.hkv for L in lens], dtype=torch.int32, device="cuda")
    o_p, lse = torch.full(c.q.shape, 55.0, device="cuda"), torch.full_like(c.lse, 55)
    state = B.make_state(c.q, o_p, lse, c.kv_len)
    for _ in range(2):
        B.losa_sparse_prefix_attn(c.ctx, c.q, c.kv, act, dev(block, block), pages, count, state)
        assert c.ctx.poll_status() == B.LOSA_ERR_BOUNDS
    off = [t for t in range(block) if t not in good]
    assert (o_p[:, off] == 55).all() and (lse[:, off] == 55).all()
    for s in range(N):
        for h in range(c.hkv):
            c.check(o_p, lse, s, h, good)


def check_rows(c, sm_scale):
    """All of the cache's rows under another softmax scale."""
    for s in range(len(c.lens)):
        for h in range(c.hkv):
            k, v = c.rows(s, h)
            heads = slice(h * c.G, (h + 1) * c.G)
            o, l, do, dl = ref.attention(c.q.cpu()[s, :, heads].double().reshape(-1, c.d), k, v, sm_scale)
            got, gl = c.out.cpu()[s, :, heads].double().reshape(-1, c.d), c.lse.cpu()[s, :, heads].double().reshape(-1)
            assert ((got - o).abs() <= do + 2.0 ** -8 * (o.abs() + do)).all()
            assert ((gl - l).abs() <= dl).all() if k.shape[0] else (gl == -float("inf")).all()


@pytest.mark.parametrize("sm_scale", [1e-3, 1e-5, 1e-12, 1e-38, 3.0])
@pytest.mark.parametrize("block,G", ROWS)
def test_rows_of_zeros_under_any_softmax_scale(block, G, sm_scale):
    """Rows of zeros, rows of the smallest bf16 numbers and ordinary ones: the mean of the values and log L, not an empty sum."""
    c = Cache([130, 1, 0, 9011], block=block, G=G, seed=block)
    c.q[0] = 0
    c.q[1::2, :, 0] = 0
    c.q[3, :, -1] = 2.0 ** -120
    c.ctx = c.B.Context(4, c.hkv * G, c.hkv, c.d, block, c.g, c.table.shape[1], c.B.LOSA_BF16, sm_scale)
    assert c.attn() == 0
    check_rows(c, sm_scale)


@pytest.mark.parametrize("block,G", ROWS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_query_that_is_no_number_stays_visible(block, G, bad):
    """One bad element: its row is NaN whether one CTA has the segment or several, the others are as ever."""
    c = Cache([40, 20011], block=block, G=G, hkv=1, seed=block)
    c.q[:, 0, 0, 3] = bad
    c.ks[c.table[:, 0].long(), :, 0] = 100            # (infinity: the first token's key is finite, and not zero there)
    c.kp[c.table[:, 0].long(), :, 0, 1] = 0x31
    assert c.attn() == 0
    assert c.out[:, 0, 0].isnan().all() and c.lse[:, 0, 0].isnan().all()
    c.q[:, 0, 0, 3] = 0
    want = c.out.clone(), c.lse.clone()
    assert c.attn() == 0
    keep = torch.ones(c.lse.shape, dtype=torch.bool, device="cuda")
    keep[:, 0, 0] = False
    assert (c.out[keep] == want[0][keep]).all() and (c.lse[keep] == want[1][keep]).all()
    c.check_all()


def test_the_time_of_stage_4_is_that_of_the_kernel_that_works():
    """Eight rows in a context of 128 take what they take in a context of eight (a kernel without work: some 5 us)."""
    ms = {}
    for block in (2, 32):
        c = Cache([32768] * 4, block=block, G=4, hkv=8)
        B, N, pmax = c.B, 4, c.table.shape[1]
        act = torch.zeros(N, block, dtype=torch.int32, device="cuda")
        act[:, 1] = 1
        pages = torch.arange(pmax, dtype=torch.int32, device="cuda").repeat(N, 8, 1).contiguous()
        count = torch.full((N, 8), 1024, dtype=torch.int32, device="cuda")
        state = B.make_state(c.q, torch.zeros(c.q.shape, device="cuda"), torch.zeros_like(c.lse), c.kv_len)
        c.ctx.profile_stage4(True)
        ms[block] = []
        for _ in range(6):
            B.losa_sparse_prefix_attn(c.ctx, c.q, c.kv, act, dev(*[2] * N), pages, count, state)
            ms[block].append(c.ctx.stage4_last_ms())
        assert c.ctx.poll_status() == 0
        c.attn()                                      # not stage 4: the last one's time stays
        assert c.ctx.stage4_last_ms() == ms[block][-1]
    few, many = min(ms[2]), min(ms[32])
    assert few > 0.02 and 0.8 * few < many < 2 * few + 0.05, ms


@pytest.mark.parametrize("block,G", ROWS)
@pytest.mark.parametrize("down", [16.0, 20.5, 23.0, 26.0])
def test_small_weights_count(block, G, down):
    """Every 32nd token takes nearly all weight and has values of zero; what comes out is made of weights 2^-down of its weight.
    They keep 11 bits down to 2^-21 of the largest and are within 2^-32 of it below."""
    L, d, hkv = 3001, 128, 2
    c = Cache([L], block=block, G=G, hkv=hkv, d=d)
    c.kp[:], c.vp[:] = 0x88, 0xff                     # keys 0, values 7 * scale
    c.ks[:], c.vs[:] = 120, 100                       # 1 and 2^(12 - 15) * 1.5
    tall = torch.arange(5, L, 32, device="cuda")
    page, slot = c.table[0].long()[tall // c.g], tall % c.g
    for h in range(hkv):
        c.kp[page, h, slot, 0] = 0x8f                 # element 0: 7
        c.vp[page, h, slot] = 0x88
    c.q[:] = 0
    c.q[..., 0] = down * 0.6931472 * d ** 0.5 / 7     # (rounded to bf16: the reference takes it as it is)
    assert c.attn() == 0
    for h in range(hkv):
        k, v = c.rows(0, h)
        heads = slice(h * G, (h + 1) * G)
        q = c.q.cpu()[0, :, heads].double().reshape(-1, d)
        s = q @ k.T * d ** -0.5
        p = torch.softmax(s, -1)
        o, l, _, dl = ref.attention(q, k, v, d ** -0.5)
        # scores: one product, exact in the accumulator; the factor, the reference, the exponent and the exponential are within 2^-22 of exponents
        # up to 2^5: 2^-17 of each weight; fp32 sums of 3,001 terms 2^-12 at most
        do = o.abs() * (2.0 ** -11 + 2.0 ** -16 + 2.0 ** -12) + L * 2.0 ** -32 * p.amax(-1, keepdim=True) * v.abs().amax() + 2.0 ** -8 * o.abs()
        got = c.out.cpu()[0, :, heads].double().reshape(-1, d)
        assert ((got - o).abs() <= do).all(), float(((got - o).abs() / do).max())
        assert ((c.lse.cpu()[0, :, heads].double().reshape(-1) - l).abs() <= dl).all()
