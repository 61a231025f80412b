"""The softmax weight that cached tokens receive (losa_kv_weights) against the plain 64-bit form (needs a B200)."""
import pytest
import torch

import bounded_cache_ref as ref
from bounded_cache_ref import Cache

pytestmark = pytest.mark.gpu

FORMATS = ["f32", "bf16", "fp8", "int4"]


def run(c, mask, keep=1.0, lse=None):
    """Weights before (NaN where they are not to be read) and after, against the definition."""
    w = torch.rand(c.kp.shape[0], c.hkv, c.g, generator=c.gen, device="cuda")
    for s, (L, a) in enumerate(zip(c.lens, c.start)):
        for p in range(c.pmax):
            w[c.table[s, p].long(), :, max(0, min(c.g, (a if keep else 0) - p * c.g)):] = float("nan")
    before = w.clone()
    if lse is None:
        assert c.attend(*mask) == 0
    else:
        c.lse.copy_(lse)
    seen = []
    for _ in range(2):                                # twice from the same weights: the same bits
        w.copy_(before)
        c.B.losa_kv_weights(c.ctx, c.queries(*mask), c.kv, c.lse, w, keep)
        assert c.ctx.poll_status() == 0
        seen.append(w.nan_to_num(-1.0))
    assert torch.equal(*seen)
    k, q, lse = c.rows("k"), c.q.cpu().double(), c.lse.cpu().double()
    after, before = w.cpu().double(), before.cpu().double()
    table = c.table.cpu().long()
    untouched = torch.ones(after.shape, dtype=torch.bool)
    for s, tokens, ok in c.each():
        L, a = c.lens[s], c.start[s]
        place = torch.arange(L)
        page, slot = table[s, place // c.g], place % c.g
        untouched[page, :, slot] = False
        for h in range(c.hkv):
            heads = slice(h * c.G, (h + 1) * c.G)
            want, tol = ref.weights(q[tokens, heads], k[s][:, h], ok, lse[tokens, heads], c.d ** -0.5, c.fmt != "f32")
            old = torch.where(place < a, before[page, h, slot], 0.0) * keep if keep else torch.zeros(L, dtype=torch.float64)
            tol = tol + 2.0 ** -23 * (want + old)
            got = after[page, h, slot]
            far = (got - want - old).abs() / tol.clamp_min(1e-38)
            assert not L or far.max() <= 1, (s, h, float(far.max()))
    assert torch.equal(after[untouched].nan_to_num(-1.0), before[untouched].nan_to_num(-1.0))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("g,d", [(16, 64), (32, 128), (64, 128), (64, 64), (16, 128)])
@pytest.mark.parametrize("mask,keep", [((0, 0, 1), 1.0), ((70, 5, 1), 0.75), ((130, 200, 32), 0.0)])
def test_formats_pages_and_masks(fmt, g, d, mask, keep):
    lens = [1, g - 1, g, g + 1, 127, 128, 129, 9 * g + 5, 700, 0, 333]
    new = [1, 1, 3, g + 1, 127, 1, 2, 33, 300, 0, 70]
    c = Cache(lens, fmt=fmt, g=g, d=d, seed=g + d)
    c.tokens(new, [L - n for L, n in zip(lens, new)])
    run(c, mask, keep)


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
@pytest.mark.parametrize("hkv,G", [(1, 1), (1, 16), (3, 5), (2, 3), (8, 4)])
def test_heads(fmt, hkv, G):
    c = Cache([400, 65, 13], fmt=fmt, hkv=hkv, G=G, seed=G, d=64)
    c.tokens([200, 17, 1], [200, 48, 12], strided=True)
    run(c, (100, 7, 1))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n", [1, 4, 5, 70, 600])
def test_long_sequences(fmt, n):
    c = Cache([9011, 5000], fmt=fmt, hkv=1, G=4)
    c.tokens([n, 1], [9011 - n, 4999])
    run(c, (0, 0, 1))


@pytest.mark.parametrize("fmt", ["bf16", "f32"])
def test_tokens_behind_the_cache_and_lse_of_more_keys(fmt):
    """A block that is not stored: a log-normaliser over its own keys too makes the weights smaller; -inf gives nothing."""
    c = Cache([500, 1, 0, 300], fmt=fmt)
    c.tokens([8, 8, 8, 8], [500, 1, 0, 4000])
    lse = torch.randn(32, c.hq, generator=c.gen, device="cuda") + 9
    lse[3:6] = -float("inf")
    run(c, (200, 4, 1), lse=lse)


def test_no_tokens_only_forget():
    c = Cache([100, 40], fmt="bf16")
    c.tokens([0, 0], [100, 40])
    run(c, (0, 0, 1), 0.5, lse=c.lse)
    c = Cache([100, 40], fmt="f32")
    c.tokens([0, 0], [100, 40])
    run(c, (10, 0, 1), 1.0, lse=c.lse)


def test_a_bad_page_is_reported():
    c = Cache([300, 77], fmt="bf16")
    c.tokens([4, 1], [296, 76])
    assert c.attend(0, 0, 1) == 0
    w = torch.zeros(c.kp.shape[0], c.hkv, c.g, device="cuda")
    c.B.losa_kv_weights(c.ctx, c.queries(), c.kv, c.lse, w)
    right = w.clone()
    c.table[0, 2] = -1
    w.zero_()
    c.B.losa_kv_weights(c.ctx, c.queries(), c.kv, c.lse, w)
    assert c.ctx.poll_status() == c.B.LOSA_ERR_BOUNDS
    pages = c.table[1, :3].long()
    assert torch.equal(w[pages], right[pages])
