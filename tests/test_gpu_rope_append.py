"""losa_rope_append against the plain 64-bit forms (needs a B200): rotation within fp32's and the type's rounding, and the cache's
contents exactly what the format makes of the rotated keys."""
import pytest
import torch

import cache_ops_ref as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    """A cache with old tokens, and new ones for it."""

    def __init__(self, new, start, *, kv="native", dtype="bf16", d=128, g=32, hq=8, hkv=2, rot=None, interleaved=False, seed=0, packed=True,
                 n_pos=None, summaries=True, token_major=False, extra_pages=1, pos=False, outs=True, amp=1.0):
        from paper_2604_12056_b200 import binding as B
        self.B, self.new, self.start, self.kvf, self.g, self.d, self.hkv, self.hq = B, list(new), list(start), kv, g, d, hkv, hq
        self.rot, self.interleaved, self.dt = d if rot is None else rot, interleaved, DT[dtype]
        gen = torch.Generator(device="cuda").manual_seed(100 + seed)
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        N, T = len(new), sum(new)
        pmax = max(1, max(-(-(a + n) // g) for a, n in zip(start, new))) + extra_pages
        n_phys = N * pmax + 3
        self.table = torch.randperm(n_phys, generator=gen, device="cuda")[:N * pmax].view(N, pmax).int()
        if packed:
            row = (rnd(T, hq + 2 * hkv, d) * amp).to(self.dt)
            self.q, self.k, self.v = row[:, :hq], row[:, hq:hq + hkv], row[:, hq + hkv:]
        else:
            self.q, self.k, self.v = ((rnd(T, h, d) * amp).to(self.dt) for h in (hq, hkv, hkv))
        self.cu = torch.tensor([0] + list(new)).cumsum(0).int().cuda()
        self.st = torch.tensor(start, dtype=torch.int32, device="cuda")
        top = max(a + n for a, n in zip(start, new))
        self.n_pos = n_pos or max(1, top) + 5
        ang = torch.rand(self.n_pos, max(1, self.rot // 2), generator=gen, device="cuda") * 6.28
        self.cos, self.sin = ang.cos(), ang.sin()
        self.pos = torch.randint(0, self.n_pos, (T,), generator=gen, device="cuda").int() if pos else None
        self.kv_len = torch.full((N,), 7777, dtype=torch.int32, device="cuda")
        es = {"native": d, "fp8": d, "int4": d // 2}[kv]
        shape = (n_phys, g, hkv, es) if token_major else (n_phys, hkv, g, es)
        if kv == "native":
            pools = [rnd(*shape).to(self.dt) for _ in range(2)]
            self.ks = self.vs = None
        elif kv == "fp8":
            pools = [(rnd(*shape) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2)]
            self.ks, self.vs = (2.0 ** torch.randint(-6, -2, (n_phys, hkv), generator=gen, device="cuda").float() for _ in range(2))
        else:
            pools = [torch.randint(0, 256, shape, generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8) for _ in range(2)]
            self.ks, self.vs = (torch.randint(90, 130, (n_phys, hkv, g, d // 32), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8) for _ in range(2))
        self.kp, self.vp = (p.transpose(1, 2) if token_major else p for p in pools)
        self.kmin = torch.full((n_phys, hkv, d), 9.0, dtype=self.dt, device="cuda") if summaries else None
        self.kmax = torch.full((n_phys, hkv, d), -9.0, dtype=self.dt, device="cuda") if summaries else None
        self.before = [None if t is None else t.clone() for t in (self.kp, self.vp, self.ks, self.vs, self.kmin, self.kmax)]
        self.q_out = torch.full((T, hq, d), 55.0, dtype=self.dt, device="cuda") if outs else None
        self.k_out, self.v_out = (torch.full((T, hkv, d), 55.0, dtype=self.dt, device="cuda") if outs else None for _ in range(2))
        self.ctx = B.Context(N, hq, hkv, d, 1, g, pmax, B.LOSA_F32 if dtype == "f32" else B.LOSA_BF16, 0.1)
        self.kv = B.make_kv(self.kp, self.vp, self.kmin, self.kmax, self.table, self.kv_len, self.ks, self.vs)
        self.rope = B.make_rope(self.cos, self.sin, interleaved) if self.rot else None
        self.tokens = B.make_new_tokens(self.q, self.k, self.v, self.cu, self.st, self.pos, self.q_out, self.k_out, self.v_out)

    def run(self):
        self.B.losa_rope_append(self.ctx, self.kv, self.rope, self.tokens)
        return self.ctx.poll_status()

    def check(self, skipped=()):
        """Everything the call writes, and that it writes nothing else.  skipped: sequences that must be left alone."""
        new, start, g, d, cpu = self.new, self.start, self.g, self.d, lambda t: t.cpu()
        pos = cpu(self.pos).long() if self.pos is not None else torch.cat([torch.arange(a, a + n) for a, n in zip(start, new)])
        q, k, v = (cpu(t).double() for t in (self.q, self.k, self.v))
        firsts = [sum(new[:s]) for s in range(len(new))]
        live = torch.zeros(sum(new), dtype=torch.bool)
        for s, f in enumerate(firsts):
            live[f:f + new[s]] = s not in skipped
        pos = torch.where(live, pos, 0)
        qr, qs = ref.rotate(q, cpu(self.cos), cpu(self.sin), pos, self.rot, self.interleaved) if self.rot else (q, q * 0)
        kr, ks_ = ref.rotate(k, cpu(self.cos), cpu(self.sin), pos, self.rot, self.interleaved) if self.rot else (k, k * 0)
        if self.q_out is not None:
            assert ref.rounded_close(cpu(self.q_out)[live], qr[live], qs[live], self.dt)
            assert (cpu(self.q_out)[~live] == 55).all()
        # the keys as rotated and rounded by the call that rotates only
        only = torch.zeros_like(self.k).contiguous()
        self.B.losa_rope_append(self.ctx, None, self.rope, self.B.make_new_tokens(None, self.k, None, self.cu, self.st, self.pos, k_out=only))
        self.ctx.poll_status()
        rk = cpu(only)
        assert ref.rounded_close(rk[live], kr[live], ks_[live], self.dt)
        rk = rk.double()
        want_kp, want_vp, want_ks, want_vs, want_min, want_max = (None if t is None else t.cpu().clone() for t in self.before)
        want_k, want_v = rk.clone(), v.clone()
        table, kv_len = cpu(self.table), cpu(self.kv_len)
        for s, (a, n) in enumerate(zip(start, new)):
            if s in skipped or n == 0:
                assert int(kv_len[s]) == 7777
                continue
            assert int(kv_len[s]) == a + n
            f = firsts[s]
            for p in range(a // g, (a + n - 1) // g + 1):
                phys, lo, hi = int(table[s, p]), max(a, p * g), min(a + n, (p + 1) * g)
                dst, src = slice(lo - p * g, hi - p * g), slice(f + lo - a, f + hi - a)
                for h in range(self.hkv):
                    for x, pool, sc, back in ((rk, want_kp, want_ks, want_k), (v, want_vp, want_vs, want_v)):
                        rows = x[src, h]
                        if self.kvf == "native":
                            pool[phys, h, dst] = rows.to(self.dt)
                            page = pool[phys, h].double()
                        elif self.kvf == "int4":
                            code, byte = ref.int4_encode(rows)
                            pool[phys, h, dst] = ref.int4_pack(code)
                            sc[phys, h, dst] = byte.to(torch.uint8)
                            back[src, h] = ref.int4_value(code, byte)
                            page = ref.int4_value(ref.int4_unpack(pool[phys, h]), sc[phys, h])
                        else:
                            page = pool[phys, h].view(torch.float8_e4m3fn).double() * float(sc[phys, h])
                            page[dst] = rows
                            code, scale = ref.fp8_page(page, hi - p * g)
                            pool[phys, h] = code.view(torch.uint8)
                            sc[phys, h] = scale
                            page = code.double() * scale
                            back[src, h] = page[dst]
                        if x is rk and want_min is not None:
                            want_min[phys, h] = page[:hi - p * g].amin(0).to(self.dt)
                            want_max[phys, h] = page[:hi - p * g].amax(0).to(self.dt)
        # (-0 and +0 are the same value, and either may be a page's extreme)
        bits = {"fp8": lambda t: t.view(torch.float8_e4m3fn).float()}.get(self.kvf, lambda t: t)
        for got, want in ((self.kp, want_kp), (self.vp, want_vp)):
            a, b = bits(cpu(got).contiguous()), bits(want.contiguous())
            assert ((a == b) | (a.isnan() & b.isnan()) if a.is_floating_point() else a == b).all()
        for got, want in ((self.ks, want_ks), (self.vs, want_vs), (self.kmin, want_min), (self.kmax, want_max)):
            assert got is None or (cpu(got) == want).all()
        if self.k_out is not None:
            assert (cpu(self.k_out)[live].double() == want_k[live]).all() and (cpu(self.v_out)[live].double() == want_v[live]).all()
            assert (cpu(self.k_out)[~live] == 55).all() and (cpu(self.v_out)[~live] == 55).all()


KINDS = [("native", "bf16"), ("native", "f32"), ("fp8", "bf16"), ("int4", "bf16")]


@pytest.mark.parametrize("kv,dtype", KINDS)
@pytest.mark.parametrize("g,d", [(16, 64), (32, 128), (64, 128), (64, 64)])
def test_ragged_batches_of_any_length(kv, dtype, g, d):
    new = [1, 0, g, 2 * g + 3, 5, g - 1, 0, 1]
    start = [0, 5, g, g - 2, 3 * g - 1, 1, 0, 2 * g]
    c = Case(new, start, kv=kv, dtype=dtype, d=d, g=g, seed=g + d)
    assert c.run() == 0
    c.check()


@pytest.mark.parametrize("kv,dtype", KINDS)
@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (32, True), (48, False), (64, True), (64, False)])
def test_rotated_parts_and_both_kinds_of_pairs(kv, dtype, rot, interleaved):
    c = Case([19, 3], [13, 0], kv=kv, dtype=dtype, d=64, g=16, hq=3, hkv=1, rot=rot, interleaved=interleaved, seed=rot)
    assert c.run() == 0
    c.check()


@pytest.mark.parametrize("kv,dtype", KINDS)
def test_rotation_positions_of_the_callers_own(kv, dtype):
    c = Case([9, 40], [70, 3], kv=kv, dtype=dtype, hq=5, hkv=5, rot=96, pos=True, n_pos=300)
    assert c.run() == 0
    c.check()


@pytest.mark.parametrize("kv,dtype", KINDS)
@pytest.mark.parametrize("kw", [dict(packed=False), dict(token_major=True), dict(summaries=False), dict(outs=False), dict(hq=32, hkv=2), dict(hq=1, hkv=1)])
def test_layouts_and_what_is_left_out(kv, dtype, kw):
    c = Case([33, 1, 64], [31, 64, 0], kv=kv, dtype=dtype, **kw)
    assert c.run() == 0
    c.check()


@pytest.mark.parametrize("n", [40, 130])
def test_many_sequences_of_single_tokens(n):
    c = Case([i % 3 for i in range(n)], [(i * 37) % 100 for i in range(n)], kv="int4", g=16, d=64, hq=2, hkv=1)
    assert c.run() == 0
    c.check()


@pytest.mark.parametrize("amp", [1e-6, 1e-3, 300.0, 3000.0, 1e5])
@pytest.mark.parametrize("kv", ["fp8", "int4"])
def test_scales_at_both_ends(kv, amp):
    c = Case([21, 2], [0, 40], kv=kv, amp=amp)
    c.k[3] = 0                                        # a token of zeros, and one with a single value
    c.v[4] = 0
    c.v[4, :, 7] = amp
    assert c.run() == 0
    c.check()


@pytest.mark.parametrize("kv,dtype", KINDS)
def test_a_sequence_taken_back_and_continued(kv, dtype):
    """Appending again from an earlier length: what lies past the new end counts for nothing."""
    c = Case([40], [20], kv=kv, dtype=dtype)
    assert c.run() == 0
    c.check()
    c.before = [None if t is None else t.clone() for t in (c.kp, c.vp, c.ks, c.vs, c.kmin, c.kmax)]
    c.new, c.start = [3], [35]
    c.q, c.k, c.v = c.q[:3] * 2, c.k[:3] * 2, c.v[:3] * 2
    c.cu, c.st = torch.tensor([0, 3], device="cuda").int(), torch.tensor([35], device="cuda").int()
    c.q_out, c.k_out, c.v_out = c.q_out[:3].contiguous(), c.k_out[:3].contiguous(), c.v_out[:3].contiguous()
    c.tokens = c.B.make_new_tokens(c.q, c.k, c.v, c.cu, c.st, None, c.q_out, c.k_out, c.v_out)
    assert c.run() == 0
    c.check()


@pytest.mark.parametrize("kv,dtype", KINDS)
def test_sequences_that_do_not_fit_are_left_alone_and_reported(kv, dtype):
    from paper_2604_12056_b200 import binding as B
    c = Case([5, 8, 4, 6], [0, 90, 30, 2], kv=kv, dtype=dtype, extra_pages=0, n_pos=96)   # 98 tokens: past the rotation table (96)
    assert c.run() == B.LOSA_ERR_BOUNDS
    c.check(skipped=(1,))
    c = Case([5, 40, 4], [0, 100, 30], kv=kv, dtype=dtype, extra_pages=0, n_pos=1000)     # 140 tokens in a row of pages cut to 128
    short = c.table[:, :4].contiguous()
    c.ctx = B.Context(3, c.hq, c.hkv, c.d, 1, c.g, 4, c.ctx.shape.dtype, 0.1)
    c.kv = B.make_kv(c.kp, c.vp, c.kmin, c.kmax, short, c.kv_len, c.ks, c.vs)
    assert c.run() == B.LOSA_ERR_BOUNDS
    c.check(skipped=(1,))


def test_bad_tables_and_positions_are_reported_and_skipped():
    from paper_2604_12056_b200 import binding as B
    c = Case([5, 5], [0, 0], kv="int4")
    c.table[1, 0] = 10 ** 6
    k0 = c.kp.clone()
    assert c.run() == B.LOSA_ERR_BOUNDS
    keep = torch.ones(c.kp.shape[0], dtype=torch.bool)
    keep[int(c.table[0, 0])] = False
    assert (c.kp.cpu()[keep] == k0.cpu()[keep]).all()
    c = Case([4], [0], pos=True, n_pos=50)
    c.pos.copy_(torch.tensor([3, -1, 50, 49]))
    assert c.run() == B.LOSA_ERR_BOUNDS               # tokens 1 and 2: as they are
    assert (c.q_out[1:3] == c.q[1:3]).all() and (c.k_out[1:3] == c.k[1:3]).all() and not (c.q_out[0] == c.q[0]).all()
    c = Case([4, 4], [-1, 0])
    assert c.run() == B.LOSA_ERR_BOUNDS
    c = Case([4, 4], [0, 0])
    c.cu.copy_(torch.tensor([0, 6, 5]))               # a negative count
    assert c.run() == B.LOSA_ERR_BOUNDS


def test_rotation_in_place_and_without_a_cache():
    c = Case([7, 0, 30], [5, 1, 90], packed=False, outs=False)
    q, k = c.q.clone(), c.k.clone()
    c.B.losa_rope_append(c.ctx, None, c.rope, c.B.make_new_tokens(c.q, c.k, None, c.cu, c.st, q_out=c.q, k_out=c.k))
    assert c.ctx.poll_status() == 0
    pos = torch.cat([torch.arange(a, a + n) for a, n in zip(c.start, c.new)])
    for got, x in ((c.q, q), (c.k, k)):
        y, size = ref.rotate(x.cpu().double(), c.cos.cpu(), c.sin.cpu(), pos, c.rot, False)
        assert ref.rounded_close(got.cpu(), y, size, c.dt)
    # by positions alone: no sequences are needed
    got = torch.zeros_like(q)
    c.B.losa_rope_append(c.ctx, None, c.rope, c.B.make_new_tokens(q, None, None, None, None, pos.int().cuda(), q_out=got))
    assert c.ctx.poll_status() == 0 and (got == c.q).all()
    assert int(c.kv_len[0]) == 7777


def test_the_callers_stream_is_the_one_that_is_used():
    c = Case([200], [3], kv="int4", hq=32, hkv=8)
    want = Case([200], [3], kv="int4", hq=32, hkv=8)
    assert want.run() == 0
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    src = c.k.clone()
    c.k.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                 # the keys arrive late, on the same stream
        c.k.copy_(src)
        c.run()
    assert (c.k_out == want.k_out).all() and (c.kp == want.kp).all()


def test_pages_beyond_32_bits_of_elements():
    """Physical pages whose offsets pass 2^31 and 2^32 bytes."""
    from paper_2604_12056_b200 import binding as B
    g, d, hkv, far = 32, 128, 1, 2 ** 30
    k = torch.randn(40, hkv, d, device="cuda").bfloat16()
    v = torch.randn(40, hkv, d, device="cuda").bfloat16()
    pools = [torch.empty(2 * far + g * d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kp, vp = (p.as_strided((3, hkv, g, d), (far, g * d, d, 1)) for p in pools)
    table, kv_len = torch.tensor([[2, 1]], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx = B.Context(1, 1, hkv, d, 1, g, 2, B.LOSA_BF16, 0.1)
    kv = B.make_kv(kp, vp, None, None, table, kv_len)
    cu, st = torch.tensor([0, 40], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    B.losa_rope_append(ctx, kv, None, B.make_new_tokens(None, k, v, cu, st))
    assert ctx.poll_status() == 0
    assert (kp[2, 0] == k[:32, 0]).all() and (vp[2, 0] == v[:32, 0]).all() and (kp[1, 0, :8] == k[32:, 0]).all() and int(kv_len[0]) == 40


@pytest.mark.parametrize("g,d", [(16, 64), (32, 128), (64, 128)])
def test_block_finalisation_of_a_4_bit_cache_is_an_append_without_rotation(g, d):
    B_blk, lens = 24, [5, 0, 3 * g, 2 * g - 1]
    c = Case([B_blk] * 4, lens, kv="int4", g=g, d=d, rot=0, packed=False)
    B = c.B
    ctx = B.Context(4, c.hq, c.hkv, d, B_blk, g, c.table.shape[1], B.LOSA_BF16, 0.1)
    one = torch.ones(4, dtype=torch.int32, device="cuda")
    state = B.make_state(c.q_out, c.q_out.float(), one.float(), one)
    c.kv_len.copy_(c.st)
    B.losa_update_prefix_cache(ctx, c.kv, state, None, c.k, c.v, True)
    assert ctx.poll_status() == 0 and (one == 0).all()
    c.q_out = c.k_out = None
    c.check()


@pytest.mark.parametrize("g,d,token_major", [(16, 64, False), (32, 128, True), (64, 128, False), (64, 64, True)])
def test_a_bf16_cache_turned_into_4_bits(g, d, token_major):
    from paper_2604_12056_b200 import binding as B
    lens, hkv = [3 * g + 1, 0, 1, 2 * g], 3
    c = Case([1] * 4, lens, kv="native", g=g, d=d, hkv=hkv, hq=3, token_major=token_major)
    n_phys = c.kp.shape[0]
    codes = [torch.full((n_phys, hkv, g, d // 2), 77, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.full((n_phys, hkv, g, d // 32), 255, dtype=torch.uint8, device="cuda") for _ in range(2)]
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    src = B.make_kv(c.kp, c.vp, c.kmin, c.kmax, c.table, kv_len)
    dst = B.make_kv(*codes, c.kmin, c.kmax, c.table, kv_len, *scales)
    for build in (False, True):                       # the summaries once by the quantiser, once on their own
        c.kmin.fill_(9)
        c.kmax.fill_(-9)
        (B.losa_build_page_summaries(c.ctx, dst) if build else B.losa_quantize_kv_pages(c.ctx, src, dst))
        assert c.ctx.poll_status() == 0
        kmin, kmax = torch.full_like(c.kmin, 9).cpu(), torch.full_like(c.kmax, -9).cpu()
        for s, L in enumerate(lens):
            for p in range(-(-L // g)):
                phys, n = int(c.table[s, p]), min(g, L - p * g)
                for pool, code, sc in ((c.kp, codes[0], scales[0]), (c.vp, codes[1], scales[1])):
                    want, byte = ref.int4_encode(pool[phys, :, :n].cpu().double())
                    assert (code[phys, :, :n].cpu() == ref.int4_pack(want)).all() and (sc[phys, :, :n].cpu() == byte).all()
                    assert (sc[phys, :, n:] == 255).all()
                    if pool is c.kp:
                        x = ref.int4_value(want, byte)
                        kmin[phys], kmax[phys] = x.amin(1).bfloat16(), x.amax(1).bfloat16()
        assert (c.kmin.cpu() == kmin).all() and (c.kmax.cpu() == kmax).all()


def test_refusals():
    from paper_2604_12056_b200 import binding as B
    c = Case([4], [0], kv="int4")

    def refused(code, kv=c.kv, rope=c.rope, **kw):
        t = B.make_new_tokens(c.q, c.k, c.v, c.cu, c.st, None, c.q_out, c.k_out, c.v_out)
        for k, v in kw.items():
            setattr(t, k, v)
        with pytest.raises(B.LosaError) as e:
            B.losa_rope_append(c.ctx, kv, rope, t)
        assert e.value.code == code, kw

    launched = c.ctx.launch_count()
    refused(B.LOSA_ERR_INVALID_ARG, cu=None)
    refused(B.LOSA_ERR_INVALID_ARG, start=None)
    refused(B.LOSA_ERR_INVALID_ARG, start=c.kv_len.data_ptr())
    refused(B.LOSA_ERR_INVALID_ARG, k=None)
    refused(B.LOSA_ERR_INVALID_ARG, v=None)
    refused(B.LOSA_ERR_INVALID_ARG, q=None)
    refused(B.LOSA_ERR_INVALID_ARG, n_tokens=-1)
    refused(B.LOSA_ERR_INVALID_ARG, q_stride=8)
    refused(B.LOSA_ERR_INVALID_ARG, kv=None, q_out=None, k_out=None)
    refused(B.LOSA_ERR_UNSUPPORTED, k_stride=c.hkv * c.d + 4)
    refused(B.LOSA_ERR_UNSUPPORTED, k=c.k.data_ptr() + 2)
    refused(B.LOSA_ERR_UNSUPPORTED, v_out=c.v_out.data_ptr() + 8)
    for field, value, code in (("rot_dim", 24, B.LOSA_ERR_UNSUPPORTED), ("rot_dim", 144, B.LOSA_ERR_INVALID_ARG), ("n_pos", 0, B.LOSA_ERR_INVALID_ARG),
                               ("cos_table", None, B.LOSA_ERR_INVALID_ARG), ("sin_table", c.sin.data_ptr() + 4, B.LOSA_ERR_UNSUPPORTED)):
        rope = B.make_rope(c.cos, c.sin)
        setattr(rope, field, value)
        refused(code, rope=rope)
    half = B.make_kv(c.kp, c.vp, c.kmin, c.kmax, c.table, c.kv_len, c.ks, c.vs)
    half.kmax = None
    refused(B.LOSA_ERR_INVALID_ARG, kv=half)
    half.kmax, half.k_scale = half.kmin, c.ks.data_ptr() + 8
    refused(B.LOSA_ERR_UNSUPPORTED, kv=half)
    half.k_scale = None
    refused(B.LOSA_ERR_INVALID_ARG, kv=half)
    f32 = B.Context(1, c.hq, c.hkv, c.d, 1, c.g, c.table.shape[1], B.LOSA_F32, 0.1)
    with pytest.raises(B.LosaError) as e:
        B.losa_rope_append(f32, c.kv, c.rope, c.tokens)
    assert e.value.code == B.LOSA_ERR_UNSUPPORTED
    assert c.ctx.launch_count() == launched
    B.losa_rope_append(c.ctx, c.kv, c.rope, B.make_new_tokens(c.q[:0], c.k[:0], c.v[:0], c.cu, c.st))       # no tokens: nothing to do
    assert c.ctx.launch_count() == launched
