"""Attention over a 4-bit cache (losa_int4_attn, stage 4, the whole step) against the plain 64-bit form and the oracle on the
values the codes stand for (needs a B200)."""
import numpy as np
import pytest
import torch

import cache_ops_ref as ref
from helpers import OracleLayer
from paper_2604_12056_b200 import workloads as wl
from test_gpu_parity import compare

pytestmark = pytest.mark.gpu


class Cache:
    """A random 4-bit cache; slots past the lengths hold any codes and scale bytes of all kinds (infinities, NaN)."""

    def __init__(self, lens, *, g=32, d=128, hkv=2, G=4, block=1, seed=0, token_major=False, extra=1, scale_bytes=(100, 125), q_amp=1.0):
        from paper_2604_12056_b200 import binding as B
        gen = torch.Generator(device="cuda").manual_seed(seed)
        ri = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=gen, device="cuda", dtype=torch.int32)
        self.B, self.lens, self.g, self.d, self.hkv, self.G, self.block = B, list(lens), g, d, hkv, G, block
        N = len(lens)
        pmax = max(1, max(-(-L // g) for L in lens)) + extra
        n_phys = N * pmax + 2
        self.table = torch.randperm(n_phys, generator=gen, device="cuda")[:N * pmax].view(N, pmax).int()
        shape = (n_phys, g, hkv, d // 2) if token_major else (n_phys, hkv, g, d // 2)
        self.kp, self.vp = (ri(0, 256, *shape).to(torch.uint8) for _ in range(2))
        if token_major:
            self.kp, self.vp = self.kp.transpose(1, 2), self.vp.transpose(1, 2)
        self.ks, self.vs = (ri(*scale_bytes, n_phys, hkv, g, d // 32).to(torch.uint8) for _ in range(2))
        for s, L in enumerate(lens):                  # past the end
            for p in range(L // g, pmax):
                at = L - p * g if L > p * g else 0
                self.ks[self.table[s, p].long(), :, at:] = 255
                self.vs[self.table[s, p].long(), :, at:] = 248
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        hq = hkv * G
        self.q = (torch.randn(N, block, hq, d, generator=gen, device="cuda") * q_amp).bfloat16()
        self.ctx = B.Context(N, hq, hkv, d, block, g, pmax, B.LOSA_BF16, d ** -0.5)
        self.kv = B.make_kv(self.kp, self.vp, None, None, self.table, self.kv_len, self.ks, self.vs)
        self.out = torch.full_like(self.q, 55)
        self.lse = torch.full((N, block, hq), 55.0, device="cuda")

    def attn(self, lse=True):
        self.B.losa_int4_attn(self.ctx, self.q, self.kv, self.out, self.lse if lse else None)
        return self.ctx.poll_status()

    def rows(self, s, h, pages=None):
        """Keys and values of the (listed) pages, float64."""
        L, g = self.lens[s], self.g
        pages = torch.arange(-(-L // g)) if pages is None else torch.as_tensor(pages, dtype=torch.long)
        phys = self.table[s].cpu()[pages].long()
        t = (pages[:, None] * g + torch.arange(g)).reshape(-1)
        return [ref.int4_value(ref.int4_unpack(p.cpu()[phys, h]), b.cpu()[phys, h]).reshape(-1, self.d)[t < L] for p, b in ((self.kp, self.ks), (self.vp, self.vs))]

    def check(self, out, lse, s, h, tokens, pages=None):
        k, v = self.rows(s, h, pages)
        heads = slice(h * self.G, (h + 1) * self.G)
        q = self.q.cpu()[s, tokens, heads].double().reshape(-1, self.d)
        o, l, do, dl = ref.attention(q, k, v, self.d ** -0.5)
        got = out.cpu()[s, tokens, heads].double().reshape(-1, self.d)
        half_unit = 2.0 ** -8 * (o.abs() + do) if out.dtype == torch.bfloat16 else 0.0
        assert ((got - o).abs() <= do + half_unit).all(), float(((got - o).abs() / (do + half_unit)).max())
        gl = lse.cpu()[s, tokens, heads].double().reshape(-1)
        if k.shape[0] == 0:
            assert (gl == -float("inf")).all() and (got == 0).all()
        else:
            assert ((gl - l).abs() <= dl).all(), float(((gl - l).abs() / dl).max())

    def check_all(self):
        for s in range(len(self.lens)):
            for h in range(self.hkv):
                self.check(self.out, self.lse, s, h, list(range(self.block)))


@pytest.mark.parametrize("g,d", [(16, 64), (32, 64), (64, 64), (16, 128), (32, 128), (64, 128)])
@pytest.mark.parametrize("block,G", [(1, 1), (1, 8), (4, 3), (2, 8), (5, 5), (7, 16), (33, 4)])
def test_lengths_pages_and_rows(g, d, block, G):
    c = Cache([0, 1, g - 1, g, g + 1, 15, 16, 17, 9 * g + 5, 700], g=g, d=d, block=block, G=G, seed=block)
    assert c.attn() == 0
    c.check_all()


@pytest.mark.parametrize("block,G", [(1, 4), (3, 5), (16, 8), (64, 4)])
def test_one_long_sequence_shared_by_all_ctas(block, G):
    c = Cache([20011], block=block, G=G, hkv=1)
    for _ in range(3):                                # (the arrival counters reset themselves)
        c.out.fill_(55)
        assert c.attn() == 0
        c.check_all()


@pytest.mark.parametrize("block", [1, 6, 20])
def test_many_short_sequences(block):
    c = Cache([(i * 53) % 200 for i in range(100)], block=block, hkv=4, G=4, g=16)
    assert c.attn() == 0
    c.check_all()


def test_all_empty_and_no_lse():
    c = Cache([0, 0])
    assert c.attn(lse=False) == 0
    assert (c.out == 0).all() and (c.lse == 55).all()
    c = Cache([0], extra=0, block=40)
    assert c.attn() == 0
    c.check_all()


@pytest.mark.parametrize("block", [1, 33])
@pytest.mark.parametrize("q_amp,scale_bytes", [(1e-30, (100, 125)), (1e30, (24, 30)), (30.0, (140, 150)), (1.0, (24, 32)), (0.01, (190, 200)), (1e-3, (24, 200))])
def test_values_at_both_ends(q_amp, scale_bytes, block):
    """Peaked softmaxes, tiny and huge queries, the smallest scales (2^-12) and large ones."""
    c = Cache([300, 77], q_amp=q_amp, scale_bytes=scale_bytes, block=block)
    if q_amp == 1e30:                                 # scores of any size: one token takes all
        c.q.mul_(0).add_(1e30)
        assert c.attn() == 0
        assert c.out.isfinite().all()
        return
    assert c.attn() == 0
    c.check_all()


@pytest.mark.parametrize("block", [1, 33])
def test_zero_rows_and_largest_scales(block):
    c = Cache([130], block=block)
    c.q[0, 0] = 0                                     # equal weights
    c.vs[:] = 199                                     # 960: the largest scale that is written
    c.vs[c.table[0, 4].long(), :, 2:] = 248
    assert c.attn() == 0
    c.check_all()


@pytest.mark.parametrize("block", [1, 40])
def test_strided_pools(block):
    c = Cache([500, 33], token_major=True, block=block)
    assert c.attn() == 0
    c.check_all()


@pytest.mark.parametrize("block,G", [(1, 4), (3, 5), (8, 4), (32, 4)])
@pytest.mark.parametrize("state_bf16", [False, True])
def test_listed_pages_of_active_tokens(block, G, state_bf16):
    """Stage 4: rows of inactive tokens stay, an empty list gives an empty sum, partial last pages, no active token."""
    g, lens = 32, [32 * 40 + 7, 32 * 9, 5, 0, 64 * 32]
    c = Cache(lens, block=block, G=G, g=g)
    B, N, pmax = c.B, len(lens), c.table.shape[1]
    rng = np.random.default_rng(block)
    act, na = np.full((N, block), -1, np.int32), np.zeros(N, np.int32)
    up, uc = np.full((N, c.hkv, pmax), -1, np.int32), np.zeros((N, c.hkv), np.int32)
    for s in range(N):
        na[s] = 0 if s == 1 and block > 1 else rng.integers(1, block + 1)
        act[s, :na[s]] = np.sort(rng.permutation(block)[:na[s]])
        P = -(-lens[s] // g)
        for h in range(c.hkv):
            uc[s, h] = 0 if (s + h) % 4 == 3 else rng.integers(0, P + 1)
            up[s, h, :uc[s, h]] = np.sort(rng.permutation(P)[:uc[s, h]])
    o_p = torch.full(c.q.shape, 55.0, device="cuda", dtype=torch.bfloat16 if state_bf16 else torch.float32)
    lse = torch.full_like(c.lse, 55)
    state = B.make_state(c.q, o_p, lse, c.kv_len)
    dev = lambda a: torch.from_numpy(a).cuda()
    for _ in range(2):
        B.losa_sparse_prefix_attn(c.ctx, c.q, c.kv, dev(act), dev(na), dev(up), dev(uc), state)
        assert c.ctx.poll_status() == 0
    for s in range(N):
        on = act[s, :na[s]].tolist()
        off = [t for t in range(block) if t not in on]
        assert (o_p[s, off] == 55).all() and (lse[s, off] == 55).all()
        for h in range(c.hkv):
            if on:
                c.check(o_p, lse, s, h, on, up[s, h, :uc[s, h]])


def test_bad_lists_tables_and_lengths_are_reported():
    c = Cache([100, 40])
    B = c.B
    c.table[1, 1] = 10 ** 7
    assert c.attn() == B.LOSA_ERR_BOUNDS
    c = Cache([100, 40], extra=0)
    c.kv_len[0] = 10 ** 6                             # longer than its row of pages
    c.table.clamp_(0)
    c.ks.clamp_max_(125)
    c.vs.clamp_max_(125)
    assert c.attn() == B.LOSA_ERR_BOUNDS
    c.lens[0] = c.table.shape[1] * c.g
    c.check_all()
    c = Cache([100])
    dev = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    state = B.make_state(c.q, c.out, c.lse, c.kv_len)
    lists = torch.full((1, c.hkv, c.table.shape[1]), -1, dtype=torch.int32, device="cuda")
    lists[..., 0] = 4                                 # a page past the prefix
    B.losa_sparse_prefix_attn(c.ctx, c.q, c.kv, dev(0), dev(1), lists, dev(1, 1), state)
    assert c.ctx.poll_status() == B.LOSA_ERR_BOUNDS
    lists[..., 0] = 0
    B.losa_sparse_prefix_attn(c.ctx, c.q, c.kv, dev(3), dev(1), lists, dev(1, 1), state)
    assert c.ctx.poll_status() == B.LOSA_ERR_BOUNDS
    c.attn()
    c.check_all()


@pytest.mark.parametrize("block,G", [(32, 4), (33, 4), (64, 16)])
def test_expired_waits_end_with_a_status_and_the_context_stays_usable(block, G):
    c = Cache([5000, 333], block=block, G=G)
    c.ctx.set_wait_limit(1)
    assert c.attn() == c.B.LOSA_ERR_TIMEOUT
    assert c.ctx.poll_status() == 0
    c.ctx.set_wait_limit(0)
    assert c.attn() == 0
    c.check_all()


@pytest.mark.parametrize("block", [1, 4])
def test_few_rows_wait_for_nothing_that_a_bound_could_end(block):
    c = Cache([5000, 333], block=block)
    c.ctx.set_wait_limit(1)
    assert c.attn() == 0
    c.check_all()


def test_results_do_not_depend_on_the_order_of_arrival():
    c = Cache([30000, 10, 999], block=3, hkv=4)
    assert c.attn() == 0
    first = c.out.clone(), c.lse.clone()
    for _ in range(5):
        c.out.fill_(0)
        assert c.attn() == 0
        assert (c.out == first[0]).all() and (c.lse == first[1]).all()


@pytest.mark.parametrize("block", [1, 32])
def test_the_callers_stream_and_a_graph(block):
    c = Cache([3000, 100], block=block)
    assert c.attn() == 0
    want = c.out.clone()
    side = torch.cuda.Stream()
    q = c.q.clone()
    c.q.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        c.q.copy_(q)
        c.B.losa_int4_attn(c.ctx, c.q, c.kv, c.out, c.lse)
    torch.cuda.synchronize()
    assert (c.out == want).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.B.losa_int4_attn(c.ctx, c.q, c.kv, c.out, c.lse)
    c.out.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert (c.out == want).all()


@pytest.mark.parametrize("block", [1, 33])
def test_pages_beyond_32_bits(block):
    """Codes beyond 2^32 bytes, scales beyond 2^31."""
    from paper_2604_12056_b200 import binding as B
    g, d, hkv = 32, 128, 8
    n_phys = 2 ** 21 // 8 + 70000                       # 16 KiB of codes and 1 KiB of scales per page
    c = Cache([g * 3 + 1], g=g, d=d, hkv=hkv, block=block)
    kp, vp = (torch.empty(n_phys, hkv, g, d // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty(n_phys, hkv, g, d // 32, dtype=torch.uint8, device="cuda") for _ in range(2))
    far = torch.tensor([n_phys - 1, 262144 + 5, n_phys - 9, 7, 9], dtype=torch.int32, device="cuda")[:c.table.shape[1]]
    for new, old in ((kp, c.kp), (vp, c.vp), (ks, c.ks), (vs, c.vs)):
        new[far.long()] = old[c.table[0].long()]
    assert kp.numel() > 2 ** 32
    table = far[None].contiguous()
    B.losa_int4_attn(c.ctx, c.q, B.make_kv(kp, vp, None, None, table, c.kv_len, ks, vs), c.out, c.lse)
    assert c.ctx.poll_status() == 0
    c.check_all()


def test_refusals():
    c = Cache([40])
    B = c.B

    def refused(code, f):
        with pytest.raises(B.LosaError) as e:
            f()
        assert e.value.code == code
    native = torch.zeros(3, c.hkv, c.g, c.d, dtype=torch.bfloat16, device="cuda")
    refused(B.LOSA_ERR_UNSUPPORTED, lambda: B.losa_int4_attn(c.ctx, c.q, B.make_kv(native, native, None, None, c.table, c.kv_len), c.out))
    odd = B.make_kv(c.kp, c.vp, None, None, c.table, c.kv_len, c.ks, c.vs)
    odd.stride_tok = 72
    refused(B.LOSA_ERR_UNSUPPORTED, lambda: B.losa_int4_attn(c.ctx, c.q, odd, c.out))
    odd.stride_tok = 48
    refused(B.LOSA_ERR_INVALID_ARG, lambda: B.losa_int4_attn(c.ctx, c.q, odd, c.out))
    refused(B.LOSA_ERR_INVALID_ARG, lambda: B.losa_int4_attn(c.ctx, None, c.kv, c.out))
    refused(B.LOSA_ERR_INVALID_ARG, lambda: B.losa_int4_attn(c.ctx, c.q, c.kv, None))
    refused(B.LOSA_ERR_UNSUPPORTED, lambda: B.losa_int4_attn(c.ctx, c.q.data_ptr() + 8, c.kv, c.out))
    f32 = B.Context(1, c.hkv * c.G, c.hkv, c.d, 1, c.g, c.table.shape[1], B.LOSA_F32, 0.1)
    refused(B.LOSA_ERR_UNSUPPORTED, lambda: B.losa_int4_attn(f32, c.q, c.kv, c.out))
    # a bf16 cache is made into codes, not the other way
    refused(B.LOSA_ERR_INVALID_ARG, lambda: B.losa_quantize_kv_pages(c.ctx, c.kv, c.kv))


# ---------------------------------------------------------------- the method on a 4-bit cache
class OracleInt4Layer(OracleLayer):
    """The layer over a 4-bit cache: every stage runs, unchanged, on the values the codes stand for."""

    def __init__(self, w, **kw):
        import types
        deq = types.SimpleNamespace(cfg=w.cfg, k_pages=w.k_pages.copy(), v_pages=w.v_pages.copy(), page_table=w.page_table,
                                    kv_len=w.kv_len.copy(), n_phys=w.n_phys)
        g = w.cfg.page_size
        for s, L in enumerate(w.kv_len):
            for p in range(-(-int(L) // g)):
                phys, n = w.page_table[s, p], min(g, int(L) - p * g)
                for pool in (deq.k_pages, deq.v_pages):
                    pool[phys, :, :n] = self.held(pool[phys, :, :n])
        super().__init__(deq, **kw)

    @staticmethod
    def held(bits):
        x = torch.from_numpy(wl.bf16_bits_to_f32(bits)).double()
        return wl.f32_to_bf16_bits(ref.int4_value(*ref.int4_encode(x)).float().numpy())

    def run_step(self, inp, x_sel=None, finalize=False):
        import types
        if finalize:                                  # what is appended is what the codes hold; the in-block part sees the block itself
            res = super().run_step(inp, x_sel, False)
            from oracle import oracle as orc
            held = types.SimpleNamespace(k=self.held(inp.k_blk), v=self.held(inp.v_blk))
            orc.update_prefix_cache(self.sh, self.kv, self.q_prev, self.step, inp.q, held.k, held.v, True)
            return res
        return super().run_step(inp, x_sel, False)


def run_blocks(cfg, n_blocks=1, fused=False, pooled=False, state_bf16=False):
    from paper_2604_12056_b200.layer import LosaLayer, to_device, to_host
    w = wl.Workload(cfg)
    g = LosaLayer(cfg, w.k_pages, w.v_pages, w.page_table, w.kv_len, int4_kv=True, pooled=pooled, state_bf16=state_bf16)
    o = OracleInt4Layer(w, pooled=pooled, state_bf16=state_bf16)

    def same_summaries():
        P = [(int(L) + cfg.page_size - 1) // cfg.page_size for L in o.kv_len]
        used = np.concatenate([w.page_table[s, :P[s]] for s in range(cfg.batch)])
        assert (to_host(g.kmin)[used] == wl.elem_to_f32(o.kmin)[used]).all() and (to_host(g.kmax)[used] == wl.elem_to_f32(o.kmax)[used]).all()
        assert (to_host(g.kv_len) == o.kv_len).all()

    same_summaries()
    for b in range(n_blocks):
        steps = w.block_steps(None)
        for t, inp in enumerate(steps):
            last = t == len(steps) - 1 and n_blocks > 1
            args = (to_device(inp.q), to_device(inp.k_blk), to_device(inp.v_blk), to_device(inp.m_per_seq))
            (g.run_step_fused if fused else g.run_step)(*args)
            snap = g.snapshot()
            assert g.ctx.poll_status() == 0
            want = o.run_step(inp, finalize=last)
            if fused:
                snap["delta"] = want["delta"]
            compare(snap, want, cfg, f"4-bit {cfg.name} block {b} step {t}")
            if last:
                g.finalize_block(args[1], args[2])
                assert g.ctx.poll_status() == 0
                same_summaries()


@pytest.mark.parametrize("fused,pooled,state_bf16", [(False, False, False), (True, False, False), (True, True, False), (True, False, True)])
def test_whole_blocks_of_the_method(fused, pooled, state_bf16):
    run_blocks(wl.config("c2", kv_lens=(2048, 1500), steps=4), fused=fused, pooled=pooled, state_bf16=state_bf16)


@pytest.mark.parametrize("g,d,hq,hkv", [(16, 64, 4, 1), (64, 128, 8, 8), (16, 128, 16, 1), (64, 64, 6, 2)])
def test_ragged_batches_page_sizes_and_appended_blocks(g, d, hq, hkv):
    cfg = wl.config("c2", n_q_heads=hq, n_kv_heads=hkv, head_dim=d, page_size=g, kv_lens=(21 * g + 5, 3, 9 * g, 128 + g),
                    block_size=12, steps=3, topk=5, m_active=3, n_blocks=2)
    run_blocks(cfg, n_blocks=2, fused=True)


def test_host_buffers():
    from paper_2604_12056_b200 import binding as B
    from paper_2604_12056_b200.layer import LosaLayer, to_device
    cfg = wl.config("c2", kv_lens=(700,), steps=2)
    w = wl.Workload(cfg)
    a, b = (LosaLayer(cfg, w.k_pages, w.v_pages, w.page_table, w.kv_len, int4_kv=True) for _ in range(2))
    for inp in w.block_steps(None):
        dev = [to_device(x) for x in (inp.q, inp.k_blk, inp.v_blk, inp.m_per_seq)]
        a.run_step_fused(*dev)
        stage = [torch.empty_like(x) for x in (dev[0], dev[1], dev[2], dev[0])]
        host = [x.cpu().pin_memory() for x in dev[:3]] + [torch.empty(dev[0].shape, dtype=dev[0].dtype).pin_memory()]
        buf = B.StepBuffersT(*[x.data_ptr() for x in stage + [b.active_idx, b.n_active, b.topk_pages, b.union_pages, b.union_count]])
        B.losa_denoise_step_host(b.ctx, *host, b.kv, b.state, buf, dev[3], cfg.topk)
        torch.cuda.synchronize()
        assert (host[3] == a.out.cpu()).all()
