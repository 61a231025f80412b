"""Attention over the paged cache with a sliding window and first tokens that stay visible (losa_window_attn) against the plain 64-bit
form (needs a B200)."""
import pytest
import torch

from bounded_cache_ref import Cache

pytestmark = pytest.mark.gpu

FORMATS = ["f32", "bf16", "fp8", "int4"]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("g,d", [(16, 64), (32, 64), (64, 64), (16, 128), (32, 128), (64, 128)])
@pytest.mark.parametrize("mask", [(0, 0, 1), (70, 5, 1), (1, 0, 1), (130, 200, 32)])
def test_formats_pages_and_masks(fmt, g, d, mask):
    """Single tokens, none, prompts from nothing and behind earlier turns, lengths around pages and groups."""
    lens = [1, g - 1, g, g + 1, 127, 128, 129, 9 * g + 5, 700, 0, 333]
    new = [1, 1, 3, g + 1, 127, 1, 2, 33, 300, 0, 70]
    c = Cache(lens, fmt=fmt, g=g, d=d, seed=g + d)
    c.tokens(new, [L - n for L, n in zip(lens, new)])
    assert c.attend(*mask) == 0
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,G", [(1, 1), (1, 16), (3, 5), (2, 3), (4, 8), (8, 4)])
def test_heads(fmt, hkv, G):
    c = Cache([400, 65, 13], fmt=fmt, hkv=hkv, G=G, seed=G, d=64)
    c.tokens([200, 17, 1], [200, 48, 12])
    assert c.attend(100, 7, 1) == 0
    c.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("mask", [(0, 0, 1), (300, 4, 1), (64, 16, 16)])
def test_tokens_behind_the_cache(fmt, mask):
    """A block that is not stored sees the window before it; one far behind sees the sinks alone, or nothing."""
    lens = [0, 1, 500, 1000, 130]
    c = Cache(lens, fmt=fmt)
    c.tokens([8, 8, 8, 8, 3], [0, 1, 500, 1000, 5000])
    assert c.attend(*mask) == 0
    c.check()


def test_rows_without_any_key():
    c = Cache([300, 0, 40], fmt="bf16")
    c.tokens([5, 70, 300], [900, 0, 30])
    assert c.attend(100, 0, 1) == 0
    c.check()
    assert (c.out[:75] == 0).all() and (c.lse[:75] == -float("inf")).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [1, 4, 37, 150])
def test_one_long_sequence_shared_by_all_ctas(fmt, n):
    c = Cache([20011], fmt=fmt, hkv=1, G=4)
    c.tokens([n], [20011 - n])
    first = None
    for mask in ((0, 0, 1), (7001, 500, 1), (0, 0, 1)):
        assert c.attend(*mask) == 0
        c.check()
        first = c.out.clone() if first is None else first
    assert torch.equal(first, c.out)                  # a call repeats itself bit by bit


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "f32"])
def test_many_short_sequences(fmt):
    lens = [(i * 53) % 200 + 1 for i in range(300)]
    new = [1 + (i % 7 == 0) * (i % 13) for i in range(300)]
    new = [min(a, b) for a, b in zip(new, lens)]
    c = Cache(lens, fmt=fmt, hkv=2, G=4, g=16, d=64)
    c.tokens(new, [L - n for L, n in zip(lens, new)])
    assert c.attend(64, 4, 1) == 0
    c.check()


def test_strides_token_major_pools_and_no_lse():
    c = Cache([300, 77], fmt="bf16", token_major=True)
    c.tokens([90, 77], [210, 0], strided=True)
    assert c.attend(120, 3, 1, lse=False) == 0
    assert (c.lse == 55).all()
    assert c.attend(120, 3, 1) == 0
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
def test_rows_behind_the_last_sequence_stay(fmt):
    c = Cache([100, 50], fmt=fmt)
    c.tokens([10, 20], [90, 30], extra=7)
    assert c.attend(0, 0, 1) == 0
    c.check()
    assert (c.out[30:] == 55).all() and (c.lse[30:] == 55).all()


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("amp", [1e-30, 1e-3, 30.0])
def test_queries_of_all_sizes(fmt, amp):
    c = Cache([300, 77], fmt=fmt)
    c.tokens([40, 1], [260, 76], amp=amp)
    assert c.attend(200, 4, 1) == 0
    c.check()


@pytest.mark.parametrize("fmt", FORMATS)
def test_scores_so_large_that_one_key_takes_all(fmt):
    c = Cache([300, 77], fmt=fmt, hkv=1, G=1)
    c.tokens([40, 1], [260, 76])
    c.q.mul_(1e26 if fmt == "f32" else 1e30)
    assert c.attend(200, 4, 1) == 0
    k, v = c.rows("k"), c.rows("v")
    for s, tokens, ok in c.each():
        sc = c.q[tokens, 0].cpu().double() @ k[s][:, 0].T
        sc[~ok] = -float("inf")
        two = sc.topk(2).values
        clear = two[:, 0] - two[:, 1] > 1e-5 * two[:, 0].abs()           # (far above what fp32 sums may be off by)
        want = v[s][:, 0][sc.argmax(-1)]
        got = c.out[tokens, 0].cpu().double()
        assert clear.any() and got.isfinite().all()
        assert ((got - want).abs() <= 2.0 ** -8 * want.abs())[clear].all()


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_is_no_number_stays_where_it_is_seen(fmt, value):
    """Keys and values that are no finite numbers: rows that do not see them are as without them, rows that see a NaN are NaN."""
    c = Cache([400], fmt=fmt, hkv=1, G=4)
    c.tokens([300], [100])
    bad = 250
    page, slot = int(c.table[0, bad // c.g]), bad % c.g
    c.vp[page, 0, slot, 3:9] = value
    assert c.attend(60, 4, 1) == 0
    sees = torch.arange(100, 400)
    sees = (sees >= bad) & (sees < bad + 60)
    got = c.out.clone()
    assert not got[sees][..., 3:9].isfinite().any()
    assert got[sees][..., 9:].isfinite().all() and got[sees][..., :3].isfinite().all()
    c.vp[page, 0, slot, 3:9] = 0.0
    assert c.attend(60, 4, 1) == 0
    c.check()
    assert torch.equal(got[~sees], c.out[~sees])
    if value != value:
        c.kp[page, 0, slot, 5] = value
        assert c.attend(60, 4, 1) == 0
        assert c.out[sees].isnan().all() and torch.equal(got[~sees], c.out[~sees]) and c.lse[sees].isnan().all()


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "f32"])
def test_what_is_wrong_with_a_sequence_is_reported_and_the_others_are_right(fmt):
    """More tokens than max_tokens, a length above the page-table row, tokens outside 0 .. T - 1, a negative start."""
    c = Cache([300, 77, 200, 64], fmt=fmt)
    c.tokens([40, 3, 2, 10], [260, 74, 198, 54])
    assert c.attend(0, 0, 1, max_tokens=10) == c.B.LOSA_ERR_BOUNDS
    out = c.out.clone()
    assert (out[10:40] == 55).all()
    assert c.attend(0, 0, 1) == 0
    c.check()
    assert torch.equal(out[40:], c.out[40:])
    c.out.fill_(55)
    c.start_t[1] = -5
    assert c.attend(0, 0, 1) == c.B.LOSA_ERR_BOUNDS
    assert (c.out[40:43] == 55).all() and torch.equal(c.out[43:], out[43:])
    c.start_t[1] = 74
    c.out.fill_(55)
    c.cu[-1] = 56                                     # one more than there are
    assert c.attend(0, 0, 1) == c.B.LOSA_ERR_BOUNDS
    assert (c.out[45:] == 55).all() and torch.equal(c.out[40:45], out[40:45])
    c.cu[-1] = 55
    table = c.table.clone()
    c.table[0, 3] = c.kp.shape[0]                     # outside the pool
    assert c.attend(0, 0, 1) == c.B.LOSA_ERR_BOUNDS
    assert torch.equal(c.out[40:], out[40:])
    c.table.copy_(table)
    assert c.attend(0, 0, 1) == 0
    c.check()


def test_captured_and_replayed_beside_the_other_calls_of_a_context():
    """A graph of attention and weights, replayed with other lengths; the context's other calls in between."""
    c = Cache([500, 60, 1000], fmt="bf16")
    c.tokens([1, 1, 1], [499, 59, 999])
    queries = c.queries(256, 4, 1)
    w = torch.zeros(c.kp.shape[0], c.hkv, c.g, device="cuda")
    assert c.attend(256, 4, 1) == 0
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            c.B.losa_window_attn(c.ctx, queries, c.kv, c.out, c.lse)
            c.B.losa_kv_weights(c.ctx, queries, c.kv, c.lse, w, 0.0)
    for lens in ([500, 60, 1000], [1, 33, 700]):
        c.lens, c.start = lens, [L - 1 for L in lens]
        c.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        c.start_t.copy_(torch.tensor(c.start, dtype=torch.int32))
        c.out.fill_(55)
        graph.replay()
        torch.cuda.synchronize()
        assert c.ctx.poll_status() == 0
        c.check()
        total = torch.stack([w[c.table[s].long()].transpose(0, 1).flatten(1)[:, :L].sum() for s, L in enumerate(lens)])
        assert torch.allclose(total, torch.full_like(total, float(c.hq)), rtol=1e-4)


def test_windowed_prefix_merged_with_a_block():
    """A block that is being denoised: the prefix part from here, the block part and the merge from stage 5."""
    block, lens = 16, [500, 40, 0]
    c = Cache(lens, fmt="bf16", block=block)
    c.tokens([block] * 3, lens)
    assert c.attend(128, 4, 1) == 0
    c.check()
    kb, vb = (torch.randn(3, block, c.hkv, c.d, device="cuda").bfloat16() for _ in range(2))
    out, lse = torch.zeros(3, block, c.hq, c.d, device="cuda", dtype=torch.bfloat16), torch.zeros(3, block, c.hq, device="cuda")
    unused = torch.zeros(1, device="cuda")
    state = c.B.make_state(unused, c.out.view(3, block, c.hq, c.d), c.lse.view(3, block, c.hq), unused)
    c.B.losa_block_attn_merge(c.ctx, c.q.contiguous(), kb, vb, state, out, lse)
    assert c.ctx.poll_status() == 0
    k, v = c.rows("k"), c.rows("v")
    for s, tokens, ok in c.each():
        for h in range(c.hkv):
            heads = slice(h * c.G, (h + 1) * c.G)
            q = c.q[tokens, heads].cpu().double()
            kk, vv = torch.cat([k[s][:, h], kb[s, :, h].cpu().double()]), torch.cat([v[s][:, h], vb[s, :, h].cpu().double()])
            sc = torch.einsum("ngd,td->ngt", q, kk) * c.d ** -0.5
            sc[:, :, :lens[s]].masked_fill_(~ok[:, None], -float("inf"))
            want = torch.einsum("ngt,td->ngd", torch.softmax(sc, -1), vv)
            got = out[s, :, heads].cpu().double()
            assert ((got - want).abs() <= 2e-2 + 1e-2 * want.abs()).all()
            assert ((lse[s, :, heads].cpu().double() - torch.logsumexp(sc, -1)).abs() <= 1e-3).all()
