"""What a bounded cache's calls do at their edges: waits that run out with work begun, padding tokens, sequences that are left out, what is
no number on quantised pages (needs a B200)."""
import pytest
import torch

import bounded_cache_ref as ref
from bounded_cache_ref import Cache

pytestmark = pytest.mark.gpu

FORMATS = ["f32", "bf16", "fp8", "int4"]
QUICK = [*range(1, 32), 40, 100, 300, 1000, 3000, 10000, 25000]         # cycles: below 32 the group of keys before which copies end, then bounds that some waits may not keep


def weights_of(c, w, mask=(0, 0, 1), keep=1.0):
    """The weights after a call on a copy of w, and the status."""
    w = w.clone()
    c.B.losa_kv_weights(c.ctx, c.queries(*mask), c.kv, c.lse, w, keep)
    return w, c.ctx.poll_status()


# prompts, blocks, single tokens: pieces that one set of warps or both work on, many short ones and few long ones
BATCHES = [([700, 300, 64], [100, 1, 64]), ([4000] * 3, [1, 1, 1]), ([90] * 40, [1] * 40), ([600] * 20, [32] * 20), ([2500], [2500])]


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int4"])
@pytest.mark.parametrize("lens,new", BATCHES)
def test_weights_whose_waits_run_out_with_work_begun(fmt, lens, new):
    """Bounds at which some warps may give up while others have copies and products in flight: the call ends, right or reported, and the next one is right."""
    c = Cache(lens, fmt=fmt)
    c.tokens(new, [L - n for L, n in zip(lens, new)])
    assert c.attend(0, 0, 1) == 0
    zero = torch.zeros(c.kp.shape[0], c.hkv, c.g, device="cuda")
    right, status = weights_of(c, zero)
    assert status == 0
    for limit in QUICK:
        c.ctx.set_wait_limit(limit)
        got, status = weights_of(c, zero)
        assert status == c.B.LOSA_ERR_TIMEOUT or (status == 0 and torch.equal(got, right)), limit
        c.ctx.set_wait_limit(0)
        got, status = weights_of(c, zero)
        assert status == 0 and torch.equal(got, right), limit


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int4"])
@pytest.mark.parametrize("lens,new", BATCHES)
def test_attention_whose_waits_run_out_with_work_begun(fmt, lens, new):
    """Likewise for the attention, whose two sets of warps meet at the end of a piece."""
    c = Cache(lens, fmt=fmt)
    c.tokens(new, [L - n for L, n in zip(lens, new)])
    for limit in QUICK:
        c.ctx.set_wait_limit(limit)
        status = c.attend(0, 0, 1)
        assert status in (0, c.B.LOSA_ERR_TIMEOUT), limit
        if status == 0:
            c.check()
        c.ctx.set_wait_limit(0)
        c.out.fill_(55)
        assert c.attend(0, 0, 1) == 0
        right = c.out.clone() if limit == QUICK[0] else right
        assert torch.equal(c.out, right), limit
    c.check()


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int4"])
@pytest.mark.parametrize("n", [1, 2, 3, 5, 8])
def test_copies_end_before_the_nth_group(fmt, n):
    """Long sequences, so that blocks have more groups and tiles than that: always reported."""
    c = Cache([30000, 30000], fmt=fmt, hkv=4, G=1)
    c.tokens([700, 700], [29300, 29300])
    assert c.attend(0, 0, 1) == 0
    out = c.out.clone()
    c.ctx.set_wait_limit(n)
    assert weights_of(c, torch.zeros(c.kp.shape[0], c.hkv, c.g, device="cuda"))[1] == c.B.LOSA_ERR_TIMEOUT
    assert c.attend(0, 0, 1) == c.B.LOSA_ERR_TIMEOUT
    c.ctx.set_wait_limit(0)
    assert c.attend(0, 0, 1) == 0 and torch.equal(c.out, out)


@pytest.mark.parametrize("limit", [1, 31])
def test_eviction_under_a_bound_below_a_look_moves_first_pages_alone(limit):
    """Pages with others before them give up: always reported, whatever stood ready, and rows behind the first page are as before; a head of one page waits for nothing."""
    for lens, moved in (([2011, 700], 32), ([60, 33], 30)):
        c = Cache(lens, fmt="bf16", d=64)
        w = torch.rand(c.kp.shape[0], c.hkv, c.g, generator=c.gen, device="cuda")
        length, budget = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, [L // 2 for L in lens]))
        kept = torch.zeros(len(lens), c.hkv, max(lens) // 2, dtype=torch.int32, device="cuda")
        before = c.rows("k")
        c.ctx.set_wait_limit(limit)
        c.B.losa_kv_evict(c.ctx, c.kv, w, c.B.make_eviction(length, budget, kept))
        assert c.ctx.poll_status() == (c.B.LOSA_ERR_TIMEOUT if moved == 32 else 0)
        for s, rows in enumerate(c.rows("k")):
            for h in range(c.hkv):
                n = min(moved, lens[s] // 2)
                assert torch.equal(rows[:n, h], before[s][kept[s, h, :n].cpu().long(), h]) and torch.equal(rows[32:, h], before[s][32:, h])
        c.ctx.set_wait_limit(0)
        assert c.ctx.poll_status() == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_padding_tokens_give_nothing_whatever_they_hold(fmt, value):
    """Tokens whose log-normaliser is -inf, in whole jobs, in parts of them and alone: the same bits as with ordinary queries in their rows."""
    new = [70, 1, 33, 4]
    c = Cache([500, 40, 33, 200], fmt=fmt)
    c.tokens(new, [430, 39, 0, 196])
    assert c.attend(200, 4, 1) == 0
    dead = torch.tensor([*range(3, 60), 70, 75, 90, 104])               # (one of several in a job, a sequence's only one)
    c.lse[dead] = -float("inf")
    c.lse[104:, 1] = -float("inf")                                       # one head of the last sequence's tokens
    w = torch.rand(c.kp.shape[0], c.hkv, c.g, generator=c.gen, device="cuda")
    want, status = weights_of(c, w, (200, 4, 1))
    assert status == 0
    c.q[dead, :, 5:9] = value
    c.q[104:, 1, 60] = value
    got, status = weights_of(c, w, (200, 4, 1))
    assert status == 0 and got.isfinite().all() and torch.equal(got, want)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("keep", [1.0, 0.5, 0.0])
@pytest.mark.parametrize("wrong", ["start", "far", "tokens", "order"])
def test_weights_of_a_sequence_that_is_left_out_stay(fmt, keep, wrong):
    """A negative start, one above 2^30, tokens behind the last, tokens in descending order: reported, and the sequence's weights are as before."""
    lens = [300, 77, 260]
    c = Cache(lens, fmt=fmt)
    c.tokens([5, 2, 3], [295, 75, 257])
    assert c.attend(0, 0, 1) == 0
    w = torch.rand(c.kp.shape[0], c.hkv, c.g, generator=c.gen, device="cuda")
    right, status = weights_of(c, w, keep=keep)
    assert status == 0
    out = {"start": [1], "far": [1], "tokens": [2], "order": [1]}[wrong]
    if wrong == "start":
        c.start_t[1] = -5
    elif wrong == "far":
        c.start_t[1] = (1 << 30) + 1
    elif wrong == "tokens":
        c.cu[3] = 11                                  # one more than there are
    else:
        c.cu[1], c.cu[2] = 5, 4                       # the second has -1; the third's tokens begin one early
        c.start_t[2] = 256
        out = [1, 2]                                  # (the third is computed with other tokens: not looked at)
    got, status = weights_of(c, w, keep=keep)
    assert status == c.B.LOSA_ERR_BOUNDS
    skip = 2 if wrong == "order" else None
    for s in range(3):
        if s != skip:
            pages = c.table[s].long()
            assert torch.equal(got[pages], (w if s in out else right)[pages]), s


@pytest.mark.parametrize("fmt", FORMATS)
def test_sequences_that_share_pages_are_weighed_one_after_the_other(fmt):
    """A common prefix: a call for each sequence, the others without tokens at their ends, gives the sum of both."""
    c = Cache([200, 170], fmt=fmt)
    c.tokens([3, 2], [197, 168])
    shared = 160 // c.g
    c.table[1, :shared] = c.table[0, :shared]
    mask = (0, 0, 1)
    assert c.attend(*mask) == 0
    c.check()
    w = torch.rand(c.kp.shape[0], c.hkv, c.g, generator=c.gen, device="cuda")
    got, cu, start = w.clone(), c.cu.clone(), c.start_t.clone()
    for s in (0, 1):
        c.cu.copy_(cu)
        c.cu[1 + s:] = c.cu[1 + s].clone()            # (the sequences before have none as well)
        c.cu[:1 + s] = c.cu[s].clone()
        c.start_t.copy_(torch.tensor([a if i == s else L for i, (a, L) in enumerate(zip(c.start, c.lens))], dtype=torch.int32))
        before = got.clone()
        got, status = weights_of(c, before, mask)
        assert status == 0
        other = c.table[1 - s, shared:].long()
        assert torch.equal(got[other], before[other])
    c.cu.copy_(cu)
    k, q, lse, old = c.rows("k"), c.q.cpu().double(), c.lse.cpu().double(), w.cpu().double()
    table = c.table.cpu().long()
    want, tol = old.clone(), torch.zeros_like(old)
    for s, tokens, ok in c.each():
        place = torch.arange(c.lens[s])
        page, slot = table[s, place // c.g], place % c.g
        for h in range(c.hkv):
            heads = slice(h * c.G, (h + 1) * c.G)
            add, off = ref.weights(q[tokens, heads], k[s][:, h], ok, lse[tokens, heads], c.d ** -0.5, c.fmt != "f32")
            want[page, h, slot] = torch.where(place < c.start[s], want[page, h, slot], 0.0) + add
            tol[page, h, slot] += off + 2.0 ** -23 * want[page, h, slot]
    assert ((got.cpu().double() - want).abs() <= tol).all()


def test_kept_rows_may_lie_far_apart():
    """kept_stride is only a distance: the largest there is, with one row."""
    c = Cache([300], fmt="bf16", hkv=1, G=4)
    w = torch.rand(c.kp.shape[0], 1, c.g, generator=c.gen, device="cuda")
    want = ref.stays([float(w[c.table[0, j // c.g].long(), 0, j % c.g]) for j in range(300)], 100, 4, 16)
    length, budget = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (300, 100))
    kept = torch.full((1, 1, 100), -1, dtype=torch.int32, device="cuda")
    before = c.rows("k")[0]
    ev = c.B.make_eviction(length, budget, kept, 4, 16)
    ev.kept_stride = 2 ** 31 - 1
    c.B.losa_kv_evict(c.ctx, c.kv, w, ev)
    assert c.ctx.poll_status() == 0 and kept.flatten().tolist() == want
    c.lens = [100]
    assert torch.equal(c.rows("k")[0], before[want])


@pytest.mark.parametrize("hkv,G,n", [(1, 4, 8192), (2, 1, 30000), (1, 8, 3000)])
def test_weights_of_a_prompt_keep_the_bits_of_fp32(hkv, G, n):
    """Thousands of terms per key: the 2-norm of the error over that of the weights is within four steps of fp32's half unit, 2^-24.
    A chain of k additions of like terms walks at random: a step is off by at most 2^-24 of its partial sum, 2^-24 / sqrt(3) in the mean square, and the partial sums grow
    evenly, so 2^-24 sqrt(k) / 3.  A job's columns are added up in four chains of 32, 2^-24 * 1.9 / sqrt(4); jobs, of which either set has at most 128 here, in a chain each,
    2^-24 * 3.8 / sqrt(2): 2.9 of these steps together.  (One chain of all the terms a set has, 3,750 in four: 2^-24 * 20 / sqrt(8), 7.2 steps.)  Terms are
    off each for itself by a few steps, of which the mean of hundreds leaves less than one."""
    c = Cache([n], fmt="bf16", hkv=hkv, G=G, g=32)
    c.tokens([n], [0])
    assert c.attend(0, 0, 1) == 0
    got, status = weights_of(c, torch.zeros(c.kp.shape[0], hkv, c.g, device="cuda"))
    assert status == 0
    place = torch.arange(n, device="cuda")
    pages = c.table[0].long()[place // c.g]
    for h in range(hkv):
        k = c.kp[pages, h, place % c.g].double()
        want = torch.zeros(n, dtype=torch.float64, device="cuda")
        for a in range(0, n, 1024):
            q, l = c.q[a:a + 1024, h * G:(h + 1) * G].double(), c.lse[a:a + 1024, h * G:(h + 1) * G].double()
            s = torch.einsum("tgd,kd->tgk", q, k[:a + 1024]) * c.d ** -0.5 - l[..., None]
            s.masked_fill_((place[:a + 1024] > place[a:a + 1024, None])[:, None], -float("inf"))
            want[:a + 1024] += s.exp_().sum((0, 1))
        far = float((got[pages, h, place % c.g].double() - want).norm() / want.norm())
        assert far <= 2.0 ** -22, far


@pytest.mark.parametrize("fmt", ["fp8", "int4"])
@pytest.mark.parametrize("new,start", [(300, 100), (1, 270), (7, 260)])
def test_nan_on_quantised_pages_stays_where_it_is_seen(fmt, new, start):
    """A value, or a run of them, that is NaN: rows that do not see it are as without it, rows that do are NaN there; then a key."""
    c = Cache([400], fmt=fmt, hkv=1, G=4)
    c.tokens([new], [start])
    bad, cols = 250, slice(32, 64) if fmt == "int4" else slice(3, 9)
    page, slot = int(c.table[0, bad // c.g]), bad % c.g

    def spoil(pool, scale):
        at = scale[page, 0, slot, 1:2] if fmt == "int4" else pool[page, 0, slot, cols]
        old = at.clone()
        at.fill_(255 if fmt == "int4" else 0x7f)
        return lambda: at.copy_(old)

    p = torch.arange(start, start + new)
    for window, sinks in ((60, 4), (0, 0), (25, 0)):
        sees = (p >= bad) & ((p < bad + window) | (window == 0))
        assert c.attend(window, sinks, 1) == 0
        c.check()
        clean, lse = c.out.clone(), c.lse.clone()
        restore = spoil(c.vp, c.vs)
        assert c.attend(window, sinks, 1) == 0
        restore()
        got = c.out.clone()
        assert got[sees][..., cols].isnan().all() and torch.equal(got[~sees], clean[~sees]) and torch.equal(c.lse, lse)
        left = torch.ones(c.d, dtype=torch.bool)
        left[cols] = False
        assert torch.equal(got[sees][..., left], clean[sees][..., left])
        restore = spoil(c.kp, c.ks)
        assert c.attend(window, sinks, 1) == 0
        restore()
        assert c.out[sees].isnan().all() and torch.equal(c.out[~sees], clean[~sees]) and c.lse[sees].isnan().all() and torch.equal(c.lse[~sees], lse[~sees])


@pytest.mark.parametrize("a,b", [("bf16", "fp8"), ("int4", "bf16"), ("f32", "bf16")])
def test_two_contexts_on_two_streams_at_once(a, b):
    """Prompts and single tokens, attention, weights and eviction of two caches side by side: the same bits as one after the other."""
    caches = []
    for fmt, lens, new in ((a, [3000, 700], [3000, 64]), (b, [5000] * 4, [1] * 4)):
        c = Cache(lens, fmt=fmt)
        c.tokens(new, [L - n for L, n in zip(lens, new)])
        c.w = torch.zeros(c.kp.shape[0], c.hkv, c.g, device="cuda")
        c.length, c.budget = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, [L // 3 for L in lens]))
        c.kept = torch.zeros(len(lens), c.hkv, max(lens) // 3, dtype=torch.int32, device="cuda")
        c.held = [x.clone() for x in (c.kp, c.vp, c.w, c.kv_len, *([] if c.ks is None else [c.ks, c.vs]))]
        caches.append(c)

    def calls(c):
        for x, old in zip((c.kp, c.vp, c.w, c.kv_len, *([] if c.ks is None else [c.ks, c.vs])), c.held):
            x.copy_(old)
        c.B.losa_window_attn(c.ctx, c.queries(1000, 4, 1), c.kv, c.out, c.lse)
        c.B.losa_kv_weights(c.ctx, c.queries(1000, 4, 1), c.kv, c.lse, c.w)
        c.B.losa_kv_evict(c.ctx, c.kv, c.w, c.B.make_eviction(c.length, c.budget, c.kept, 4, 16))

    def state(c):
        assert c.ctx.poll_status() == 0
        return [x.contiguous().view(torch.uint8).clone() for x in (c.out, c.lse, c.w, c.kp, c.vp, c.kept, c.kv_len)]

    want = []
    for c in caches:
        calls(c)
        want.append(state(c))
    streams = [torch.cuda.Stream() for _ in caches]
    for _ in range(10):
        torch.cuda.synchronize()
        for c, stream in zip(caches, streams):
            with torch.cuda.stream(stream):
                calls(c)
        torch.cuda.synchronize()
        for c, right in zip(caches, want):
            assert all(torch.equal(x, y) for x, y in zip(state(c), right))
