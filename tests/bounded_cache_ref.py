"""Plain 64-bit forms of windowed attention, the keys' weights and eviction, from their definitions, and caches to try them on.

Nothing here is used by the product path.
"""
from __future__ import annotations

import torch

import cache_ops_ref as ref


def visible(start, n, length, window, sinks, span):
    """[n, length]: which keys the tokens at places start .. start + n - 1 see."""
    p = torch.arange(start, start + n)[:, None]
    j = torch.arange(length)[None]
    ok = j < (p // span + 1) * span
    if window:
        ok = ok & ((j > p - window) | (j < sinks))
    return ok


def attention(q, k, v, ok, scale, mma):
    """q [n, G, d], k / v [t, d] in float64, ok [n, t]: output, log-sum-exp, and bounds of what they may be off by.

    Scores: on the tensor cores (mma) operands are exact and each of the d / 16 partial sums is rounded or cut by at most 2^-22 of the
    sum of |q||k|; in fp32 a chain of d fused operations is off by at most d 2^-24 of it.  The exponential's argument has 2^-23 of
    the score's and the reference's size on top, the exponential 2^-22.  Weights are bf16 on the tensor cores: half a step is 2^-8 of the weight.
    Sums: at most t + 64 additions in a chain (2^-24 of the sum of absolute terms each)."""
    n, t = ok.shape
    d = q.shape[-1]
    if t == 0 or n == 0:
        z = torch.zeros_like(q)
        return z, torch.full(q.shape[:2], -float("inf"), dtype=torch.float64), z, torch.zeros(q.shape[:2], dtype=torch.float64)
    s = torch.einsum("ngd,td->ngt", q, k) * scale
    s = torch.where(ok[:, None], s, -float("inf"))
    lse = torch.logsumexp(s, -1)
    none = lse == -float("inf")
    p = torch.exp(s - torch.where(none, 0.0, lse)[..., None])
    size = (torch.einsum("ngd,td->ngt", q.abs(), k.abs()) * scale * ok[:, None]).amax(-1)
    ds = size * ((d / 16 * 2.0 ** -22) if mma else d * 2.0 ** -24) + size * 2.0 ** -21 + 2.0 ** -21
    vs = torch.where(ok.any(0)[:, None], v, 0.0)      # (a key nobody sees may hold anything)
    around = torch.einsum("ngt,td->ngd", p, vs.abs())
    do = around * (2 * ds[..., None] + (2.0 ** -8 if mma else 0.0) + 2.0 ** -19 + (t + 64) * 2.0 ** -24)
    dl = 2 * ds + 2.0 ** -22 * torch.where(none, 0.0, lse).abs() + (t + 64) * 2.0 ** -24
    return torch.einsum("ngt,td->ngd", p, vs), lse, do, dl


def weights(q, k, ok, lse, scale, mma):
    """Sums over tokens and heads of exp(scale q.k - lse), and what they may be off by (arguments as in `attention`)."""
    n, t = ok.shape
    d = q.shape[-1]
    on = ok[:, None] & (lse != -float("inf"))[..., None]
    s = torch.einsum("ngd,td->ngt", q, k) * scale
    l = torch.where(lse == -float("inf"), 0.0, lse)
    p = torch.where(on, torch.exp(s - l[..., None]), 0.0)
    size = torch.einsum("ngd,td->ngt", q.abs(), k.abs()) * scale
    rel = size * ((d / 16 * 2.0 ** -22) if mma else d * 2.0 ** -24) + (size + l.abs()[..., None]) * 2.0 ** -22 + 2.0 ** -21
    return p.sum((0, 1)), (p * (2 * rel + (n * q.shape[1] + 64) * 2.0 ** -24)).sum((0, 1))


def stays(w, budget, sinks, recent):
    """Former places of what stays of a sequence with weights w (a list), ascending."""
    L = len(w)
    first = min(sinks, budget)
    last = min(recent, budget - first)
    order = lambda j: (0, 0.0) if w[j] != w[j] else (1, -w[j])          # noqa: E731  (a NaN is larger than any number)
    middle = sorted(range(first, L - last), key=lambda j: (*order(j), j))[:budget - first - last]
    return sorted([*range(first), *middle, *range(L - last, L)])


class Cache:
    """A random paged cache of any format; what lies behind the lengths is NaN, or codes that stand for it."""

    def __init__(self, lens, *, fmt="bf16", g=32, d=128, hkv=2, G=4, seed=0, token_major=False, extra=1, block=1, batch=None):
        from paper_2604_12056_b200 import binding as B
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.gen = gen
        self.B, self.lens, self.fmt, self.g, self.d, self.hkv, self.G = B, list(lens), fmt, g, d, hkv, G
        self.hq = hkv * G
        self.dtype = torch.float32 if fmt == "f32" else torch.bfloat16
        N = len(lens)
        self.pmax = pmax = max(1, max(-(-L // g) for L in lens)) + extra
        n_phys = N * pmax + 2
        self.table = torch.randperm(n_phys, generator=gen, device="cuda")[:N * pmax].view(N, pmax).int()
        self.live = torch.zeros(n_phys, g, dtype=torch.bool, device="cuda")
        for s, L in enumerate(lens):
            at = torch.arange(pmax * g, device="cuda").view(pmax, g) < L
            self.live[self.table[s].long()] = at

        def pool():
            x = torch.randn(n_phys, hkv, g, d, generator=gen, device="cuda")
            if fmt == "fp8":                          # (random codes are as good as quantised values)
                scale = torch.exp2(torch.randint(-6, -3, (n_phys, hkv), generator=gen, device="cuda").float())
                code = (x * 50).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
                return torch.where(self.live[:, None, :, None], code, torch.full_like(code, 0x7f)), scale
            if fmt == "int4":
                code = torch.randint(0, 256, (n_phys, hkv, g, d // 2), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
                byte = torch.randint(96, 112, (n_phys, hkv, g, d // 32), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
                return code, torch.where(self.live[:, None, :, None], byte, torch.full_like(byte, 255))
            return torch.where(self.live[:, None, :, None], x, float("nan")).to(self.dtype), None

        (self.kp, self.ks), (self.vp, self.vs) = pool(), pool()
        if token_major:
            self.kp, self.vp = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (self.kp, self.vp))
        self.kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.kmin = self.kmax = None
        self.ctx = B.Context(N, self.hq, hkv, d, block, g, pmax, B.LOSA_F32 if fmt == "f32" else B.LOSA_BF16, d ** -0.5)
        self.describe()

    def describe(self):
        self.kv = self.B.make_kv(self.kp, self.vp, self.kmin, self.kmax, self.table, self.kv_len, self.ks, self.vs)

    def values(self, pool, scale):
        """A pool as float64 on the CPU."""
        if self.fmt == "fp8":
            return pool.view(torch.float8_e4m3fn).cpu().double() * scale.cpu().double()[..., None, None]
        if self.fmt == "int4":
            return ref.int4_value(ref.int4_unpack(pool.cpu()), scale.cpu())
        return pool.cpu().double()

    def rows(self, what):
        """Per sequence [L, H_kv, d] float64 of "k" or "v"."""
        x = self.values(self.kp, self.ks) if what == "k" else self.values(self.vp, self.vs)
        table = self.table.cpu().long()
        return [x[table[s]].transpose(1, 2).flatten(0, 1)[:L] for s, L in enumerate(self.lens)]

    def tokens(self, new, start, strided=False, extra=0, amp=1.5):
        """Queries of `new` tokens per sequence (and `extra` that no sequence owns)."""
        T = sum(new) + extra
        self.new, self.start = list(new), list(start)
        width = self.hq + (2 * self.hkv if strided else 0)
        row = (torch.randn(T, width, self.d, generator=self.gen, device="cuda") * amp).to(self.dtype)
        self.q = row[:, :self.hq]
        self.cu = torch.tensor([0, *new], device="cuda").cumsum(0).int()
        self.start_t = torch.tensor(start, dtype=torch.int32, device="cuda")
        self.out = torch.full((T, self.hq, self.d), 55.0, device="cuda").to(self.dtype)
        self.lse = torch.full((T, self.hq), 55.0, device="cuda")

    def queries(self, window=0, sinks=0, span=1, max_tokens=None):
        self.mask = (window, sinks, span)
        return self.B.make_queries(self.q, self.cu, self.start_t, max(1, max(self.new)) if max_tokens is None else max_tokens, window, sinks, span)

    def attend(self, *mask, lse=True, max_tokens=None):
        self.B.losa_window_attn(self.ctx, self.queries(*mask, max_tokens=max_tokens), self.kv, self.out, self.lse if lse else None)
        return self.ctx.poll_status()

    def each(self):
        """(sequence, head, its tokens, which keys they see)"""
        at = 0
        for s, (n, a, L) in enumerate(zip(self.new, self.start, self.lens)):
            yield s, slice(at, at + n), visible(a, n, L, *self.mask)
            at += n

    def check(self):
        k, v = self.rows("k"), self.rows("v")
        q, out, lse = self.q.cpu().double(), self.out.cpu().double(), self.lse.cpu().double()
        mma = self.fmt != "f32"
        for s, tokens, ok in self.each():
            for h in range(self.hkv):
                heads = slice(h * self.G, (h + 1) * self.G)
                o, l, do, dl = attention(q[tokens, heads], k[s][:, h], v[s][:, h], ok, self.d ** -0.5, mma)
                tol = do + (2.0 ** -8 if mma else 2.0 ** -24) * (o.abs() + do)
                far = (out[tokens, heads] - o).abs() / tol.clamp_min(1e-300)
                assert not far.numel() or far.max() <= 1, (s, h, float(far.max()))
                none = l == -float("inf")
                assert (lse[tokens, heads][none] == -float("inf")).all() and (out[tokens, heads][none] == 0).all()
                far = ((lse[tokens, heads] - l).abs() / dl)[~none]
                assert not far.numel() or far.max() <= 1, (s, h, "lse", float(far.max()))
