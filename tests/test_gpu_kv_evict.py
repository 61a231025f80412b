"""Eviction by accumulated weight (losa_kv_evict) against the definition (needs a B200): everything here is exact."""
import pytest
import torch

import bounded_cache_ref as ref
import cache_ops_ref as codes
from bounded_cache_ref import Cache

pytestmark = pytest.mark.gpu

FORMATS = ["f32", "bf16", "fp8", "int4"]


def evict(c, w, budgets, sinks, recent, summaries=True, stride=None):
    """The call, and the whole pool against the definition."""
    n_phys = c.kp.shape[0]
    c.kmin, c.kmax = (torch.full((n_phys, c.hkv, c.d), 7.0, device="cuda").to(c.dtype) for _ in range(2)) if summaries else (None, None)
    c.describe()
    length, budget = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (c.lens, budgets))
    most = max(1, max([b for b, L in zip(budgets, c.lens) if b < L], default=1)) if stride is None else stride
    kept = torch.full((len(c.lens), c.hkv, most), -7, dtype=torch.int32, device="cuda")
    before = {n: x.clone() for n, x in (("k", c.kp), ("v", c.vp), ("w", w))} | {n: x.clone() for n, x in (("ks", c.ks), ("vs", c.vs)) if x is not None}
    rows = {"k": c.rows("k"), "v": c.rows("v")}
    c.B.losa_kv_evict(c.ctx, c.kv, w, c.B.make_eviction(length, budget, kept, sinks, recent))
    status = c.ctx.poll_status()
    table, old_w, new_w = c.table.cpu().long(), before["w"].cpu(), w.cpu()
    pools = {"k": (before["k"].cpu(), c.kp.cpu(), c.ks), "v": (before["v"].cpu(), c.vp.cpu(), c.vs)}
    scales = {n: before[n + "s"].cpu() if n + "s" in before else None for n in ("k", "v")}
    want_w, lens = old_w.clone(), []
    want = {n: p[0].clone() for n, p in pools.items()}
    for s, (L, b) in enumerate(zip(c.lens, budgets)):
        if b < 0 or b >= L or status:
            lens.append(L)
            assert (kept[s] == -7).all()
            continue
        lens.append(b)
        for h in range(c.hkv):
            place = torch.arange(L)
            here = old_w[table[s, place // c.g], h, place % c.g]
            stay = torch.tensor(ref.stays(here.tolist(), b, sinks, recent), dtype=torch.long)
            assert kept[s, h, :b].cpu().tolist() == stay.tolist(), (s, h)
            assert (kept[s, h, b:] == -7).all()
            to = torch.arange(b)
            want_w[table[s, to // c.g], h, to % c.g] = here[stay]
            for n, (old, new, _) in pools.items():
                fp8 = c.fmt == "fp8"
                for p in range(-(-b // c.g)):
                    r, page = rows[n][s][stay[p * c.g:(p + 1) * c.g], h], table[s, p]
                    if fp8:
                        full = torch.zeros(c.g, c.d, dtype=torch.float64)
                        full[:len(r)] = r
                        code, scale = codes.fp8_page(full, len(r))
                        want[n][page, h] = code.view(torch.uint8)
                        scales[n][page, h] = scale
                        r = code.double()[:len(r)] * scale
                    if n == "k" and summaries:
                        assert torch.equal(c.kmin[page, h].cpu().double(), r.amin(0)) and torch.equal(c.kmax[page, h].cpu().double(), r.amax(0))
                if not fp8:
                    src, dst = (table[s, stay // c.g], stay % c.g), (table[s, to // c.g], to % c.g)
                    want[n][dst[0], h, dst[1]] = old[src[0], h, src[1]]
                    if scales[n] is not None:
                        scales[n][dst[0], h, dst[1]] = before[n + "s"].cpu()[src[0], h, src[1]]
    same = lambda a, b: torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))      # noqa: E731  (NaN too)
    assert same(new_w, want_w)
    for n, (_, new, scale) in pools.items():
        # (E4M3 has two zeros)
        assert same(torch.where(new == 128, 0, new), torch.where(want[n] == 128, 0, want[n])) if c.fmt == "fp8" else same(new, want[n]), n
        assert scale is None or same(scale.cpu(), scales[n])
    assert c.kv_len.tolist() == lens
    return status


def some_weights(c, kind="spread"):
    shape = (c.kp.shape[0], c.hkv, c.g)
    x = torch.randn(shape, generator=c.gen, device="cuda")
    if kind == "ties":
        return torch.floor(x)
    if kind == "equal":
        return torch.full(shape, 0.25, device="cuda")
    if kind == "odd":                                 # negative ones, zeros of both signs, infinities, NaN
        x[x.abs() < 0.3] = 0.0
        x[(x > 0.3) & (x < 0.4)] = -0.0
        x[(x > 1.5) & (x < 1.6)] = float("inf")
        x[(x < -1.5) & (x > -1.6)] = -float("inf")
        x[x > 2.2] = float("nan")
        return x
    return torch.exp(3 * x)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("g,d", [(16, 64), (32, 64), (64, 64), (16, 128), (32, 128), (64, 128)])
@pytest.mark.parametrize("kind", ["spread", "ties"])
def test_formats_and_pages(fmt, g, d, kind):
    lens = [500, 77, 2, 0, 300, 129, 1, 64, 400]
    budgets = [200, 76, 1, 0, 300, 5, 0, -1, 399]
    c = Cache(lens, fmt=fmt, g=g, d=d, seed=g)
    assert evict(c, some_weights(c, kind), budgets, 4, 16) == 0


@pytest.mark.parametrize("kind", ["equal", "odd"])
@pytest.mark.parametrize("sinks,recent", [(0, 0), (1, 0), (0, 7), (1000, 5), (3, 1000), (50, 50)])
def test_ties_odd_values_and_shares_that_do_not_fit(kind, sinks, recent):
    c = Cache([500, 77, 100, 40], fmt="bf16", d=64)
    assert evict(c, some_weights(c, kind), [200, 30, 99, 3], sinks, recent) == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("L,b", [(20011, 5000), (60001, 59000)])
def test_long_sequences(fmt, L, b):
    """Also more weights than shared memory holds, and a budget that leaves most rows where they are."""
    c = Cache([L], fmt=fmt, hkv=1, G=1, d=64, g=16)
    assert evict(c, some_weights(c), [b], 4, 32) == 0


def test_again_and_again_and_other_strides():
    """A cache that is cut down step by step, token-major, without summaries; the flags of one call do not show in the next."""
    c = Cache([700, 650, 90], fmt="bf16", token_major=True)
    w = some_weights(c)
    for budgets in ([650, 649, 80], [300, 649, 79], [31, 20, 79], [1, 1, 1]):
        assert evict(c, w, budgets, 2, 8, summaries=False) == 0
        c.lens = [min(b, L) for b, L in zip(budgets, c.lens)]


def test_a_sequence_that_cannot_be_cut_is_left_as_it_is():
    c = Cache([300, 77], fmt="bf16")
    assert evict(c, some_weights(c), [200, 30], 2, 8, stride=20) == c.B.LOSA_ERR_BOUNDS        # kept is too short for both
    c = Cache([300], fmt="bf16")
    c.table[0, 9] = -1                                # the sequence's last page
    w = some_weights(c)
    k, old = c.kp.clone(), w.clone()
    kept = torch.zeros(1, c.hkv, 100, dtype=torch.int32, device="cuda")
    length, budget = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (300, 100))
    c.B.losa_kv_evict(c.ctx, c.kv, w, c.B.make_eviction(length, budget, kept))
    assert c.ctx.poll_status() == c.B.LOSA_ERR_BOUNDS
    assert torch.equal(k.view(torch.uint8), c.kp.view(torch.uint8)) and torch.equal(old, w) and int(c.kv_len[0]) == 300
    length[0] = 100000
    c.B.losa_kv_evict(c.ctx, c.kv, w, c.B.make_eviction(length, budget, kept))
    assert c.ctx.poll_status() == c.B.LOSA_ERR_BOUNDS
    assert torch.equal(old, w) and int(c.kv_len[0]) == 300


def test_a_wait_that_runs_out_ends_the_call():
    """With a bound of one cycle a page that has to wait gives up: reported, and the context stays usable."""
    c = Cache([20011], fmt="bf16", hkv=4, d=64)
    w = some_weights(c)
    length, budget = (torch.tensor([x], dtype=torch.int32, device="cuda") for x in (20011, 9000))
    kept = torch.zeros(1, c.hkv, 9000, dtype=torch.int32, device="cuda")
    c.ctx.set_wait_limit(1)
    c.B.losa_kv_evict(c.ctx, c.kv, w, c.B.make_eviction(length, budget, kept))
    assert c.ctx.poll_status() in (0, c.B.LOSA_ERR_TIMEOUT)
    c.ctx.set_wait_limit(0)
    c = Cache([2011], fmt="bf16", d=64)
    assert evict(c, some_weights(c), [900], 4, 32) == 0


def test_captured_and_replayed():
    c = Cache([400, 90], fmt="bf16", d=64)
    w = some_weights(c)
    keep = (c.kp.clone(), c.vp.clone(), w.clone())
    length, budget = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([400, 90], [100, 30]))
    kept = torch.zeros(2, c.hkv, 100, dtype=torch.int32, device="cuda")
    ev = c.B.make_eviction(length, budget, kept, 2, 4)
    c.B.losa_kv_evict(c.ctx, c.kv, w, ev)
    want = (c.kp.clone(), c.vp.clone(), w.clone(), kept.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.B.losa_kv_evict(c.ctx, c.kv, w, ev)
    for _ in range(3):
        for a, b in zip((c.kp, c.vp, w), keep):
            a.copy_(b)
        kept.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert c.ctx.poll_status() == 0
        for a, b in zip((c.kp, c.vp, w, kept), want):
            assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
