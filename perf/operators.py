"""Work of the cache operators, as cases that are timed and compared: appending rotated keys and values to the paged
cache, and attention over a cache held in 4 bits.

An engine keeps one paged cache per attention layer.  It appends the tokens of prompts, of finished blocks and of
decoding steps (`losa_rope_append`), in the cache's own format, and attends to the cache (`losa_int4_attn` over all of
it, `losa_sparse_prefix_attn` over listed pages).  A case is one such call:

  op = "append"  new tokens of every sequence: queries and keys rotated, keys and values written into their pages
       "attn"    all `block` query tokens of every sequence over their whole 4-bit cache
       "listed"  `active` query tokens of every sequence over the `pages` listed pages of each KV head

With `own` false, `run` computes the same in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

QWEN = {"q_heads": 32, "kv_heads": 8, "dim": 128}


def _append(name, new, start, *, page=32, dtype="bf16", kv="native", rot=128, pairs="split", **heads):
    c = {"name": name, "op": "append", "new": new, "start": start, "page": page, "dtype": dtype, "kv": kv, "rot": rot, "pairs": pairs}
    c.update(heads or QWEN)
    return c


def _attn(name, lens, *, page=32, block=1, **heads):
    c = {"name": name, "op": "attn", "lens": lens, "page": page, "block": block}
    c.update(heads or QWEN)
    return c


def _text(values):
    return ",".join(str(v) for v in values)


def listed():
    return [
        # one token for each of 64 running sequences of any length, as every decoding step appends them: latency
        _append("append_tokens_int4", _text([1] * 64), _text((i * 577 + 31) % 4096 for i in range(64)), kv="int4"),
        # the finished block of one interactive sequence, at a length inside a page
        _append("append_block_bf16", "32", "8201"),
        # a serving batch's finished blocks: pages that are touched twice are quantised again
        _append("append_blocks_fp8", _text([32] * 8), "32768,16381,24571,32003,8191,0,20000,11", kv="fp8"),
        # fp32 model check: small heads, half of each head rotated in neighbouring pairs
        _append("append_prompts_f32", "1024,777", "0,5", page=16, dtype="f32", rot=32, pairs="neighbours", q_heads=4, kv_heads=1, dim=64),
        # prompts of a ragged batch into a 4-bit cache, two of them behind earlier turns
        _append("append_prompts_int4", "8191,4097,1,2875", "0,0,511,1000", kv="int4"),
        # one long prompt into a bf16 cache
        _append("append_prompt_32k", "32768", "0"),
        # one interactive sequence, one token: latency
        _attn("attn_one_8k", "8192"),
        # decoding step of 64 short ragged sequences, an empty one and one of a single token among them
        _attn("attn_batch_short", _text([0, 1] + [(i * 577 + 31) % 4096 for i in range(62)])),
        # decoding step of eight 32K sequences: bandwidth
        _attn("attn_8x32k", _text([32768] * 8)),
        # four query tokens a sequence (16 rows a KV head), ragged long prompts
        _attn("attn_4_tokens", "16381,24571,32768,32003", block=4),
        # a whole block of 32 tokens over eight 32K prompts, 128 rows a KV head: the tensor cores' work
        _attn("attn_block_8x32k", _text([32768] * 8), block=32),
        # sparse step of the same batch: three active tokens, the union of their pages
        {"name": "listed_8x32k", "op": "listed", "lens": _text([32768] * 8), "page": 32, "block": 32, "active": 3, "pages": 330, **QWEN},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hkv, G, d = rng.choice([(8, 4, 128), (8, 4, 128), (4, 8, 64), (2, 5, 128), (1, 4, 64), (4, 1, 128), (2, 16, 128)])
    heads = {"q_heads": hkv * G, "kv_heads": hkv, "dim": d}
    page = rng.choice([16, 32, 32, 64])
    op = rng.choice(["append", "append", "attn", "attn", "listed"])
    if op == "append":
        dtype, kv = rng.choice([("bf16", "native"), ("bf16", "int4"), ("bf16", "int4"), ("bf16", "fp8"), ("f32", "native")])
        n = rng.choice([1, 2, 3, 8, 17])
        total = _log_int(rng, n, 24000)
        new = [max(0, int(total / n * rng.uniform(0.2, 1.8))) for _ in range(n)]
        new[0] = max(1, new[0])
        start = [rng.choice([0, rng.randrange(4096)]) for _ in range(n)]
        rot = rng.choice([d, d, d // 2, 16])
        c = _append("", _text(new), _text(start), page=page, dtype=dtype, kv=kv, rot=rot, pairs=rng.choice(["split", "split", "neighbours"]), **heads)
        del c["name"]
        return c
    n = rng.choice([1, 2, 3, 8, 17])
    total = _log_int(rng, 16 * n, 160000)
    lens = [max(0, int(total / n * rng.uniform(0.2, 1.8))) for _ in range(n)]
    block = rng.choice([1, 1, 2, 5, 8, 16, 32])
    c = {"op": op, "lens": _text(lens), "page": page, "block": block, **heads}
    if op == "listed":
        c["active"] = rng.randint(1, block)
        c["pages"] = max(1, int(max(lens) / page * rng.uniform(0.1, 0.6)))
    return c


# ---------------------------------------------------------------- inputs
def _ints(text):
    return [int(v) for v in text.split(",")]


def _scale_values(b):
    """The numbers that scale bytes stand for: a byte, moved seven places up, is an fp16 number."""
    return (b.to(torch.int16) << 7).view(torch.float16).float()


def _int4_encode(x):
    """fp32 rows [.., d] -> (packed codes [.., d/2], scale bytes [.., d/32])."""
    g = x.unflatten(-1, (-1, 32))
    amax = g.abs().amax(-1)
    bits = (amax / torch.full_like(amax, 7.0)).view(torch.int32)                # (a plain number would be multiplied by as its reciprocal)
    up = ((bits + 0xFFFFF) & ~0xFFFFF).view(torch.float32)                      # four significant bits, upwards
    byte = (up.clamp(2.0 ** -12, 960.0).half().view(torch.int16) >> 7).to(torch.uint8)
    y = g / _scale_values(byte)[..., None]
    c = (torch.sign(y) * torch.floor(y.abs() + 0.5)).clamp(-7, 7).flatten(-2).to(torch.int16) + 8
    return (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8), byte


def _int4_decode(codes, byte):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8.0
    return (c.unflatten(-1, (-1, 32)) * _scale_values(byte)[..., None]).flatten(-2)


def _table(gen, counts, page):
    """A shuffled page table [N, P_max] for `counts` tokens per sequence, and the pool's size."""
    pmax = max(1, max(-(-c // page) for c in counts))
    n_phys = len(counts) * pmax
    return torch.randperm(n_phys, generator=gen, device="cuda").view(len(counts), pmax).int(), n_phys


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 17)
    hkv, d, g = case["kv_heads"], case["dim"], case["page"]
    st = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    # keys have channels that stand out, as rotated keys of trained models do
    channel = 1.0 + 2.0 * (torch.rand(hkv, d, generator=gen, device="cuda") > 0.94)

    if case["op"] == "append":
        new, start = _ints(case["new"]), _ints(case["start"])
        N, T, dt = len(new), sum(new), torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        st["page_table"], n_phys = _table(gen, [a + b for a, b in zip(new, start)], g)
        # projections arrive as one row per token: queries, keys, values side by side
        hq = case["q_heads"]
        row = normal(T, hq + 2 * hkv, d)
        row[:, hq:hq + hkv] *= channel
        row = row.to(dt)
        st["q"], st["k"], st["v"] = row[:, :hq], row[:, hq:hq + hkv], row[:, hq + hkv:]
        st["start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
        st["cu"] = torch.tensor([0] + new, dtype=torch.int64, device="cuda").cumsum(0).int()
        half, n_pos = case["rot"] // 2, max(a + b for a, b in zip(new, start))
        angle = torch.arange(n_pos, device="cuda").double()[:, None] * 1e6 ** (-torch.arange(half, device="cuda").double() / half)
        st["cos"], st["sin"] = angle.cos().float(), angle.sin().float()
        # what the cache holds already, and the pages that the tokens fall into, as the engine that handed them out knows them
        pairs = [(s, p) for s in range(N) for p in range(start[s] // g, -(-(start[s] + new[s]) // g) if new[s] else 0)]
        ts, tp = (torch.tensor(x, dtype=torch.int64, device="cuda") for x in zip(*pairs))
        first = [sum(1 for s, _ in pairs if s < k) - start[k] // g for k in range(N)]
        st["touched"] = (ts, tp, torch.tensor(first, dtype=torch.int64, device="cuda"))
        st["kv_len"] = st["start"].clone()
        st["kmin"] = torch.zeros(n_phys, hkv, d, dtype=dt, device="cuda")
        st["kmax"] = torch.zeros_like(st["kmin"])
        if case["kv"] == "native":
            st["kp"], st["vp"] = (normal(n_phys, hkv, g, d).to(dt) for _ in range(2))
            st["ks"] = st["vs"] = None
        elif case["kv"] == "fp8":
            st["kp"], st["vp"] = (normal(n_phys, hkv, g, d).mul_(100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2))
            st["ks"], st["vs"] = (torch.full((n_phys, hkv), 2.0 ** -6, device="cuda") for _ in range(2))
        else:
            (st["kp"], st["ks"]), (st["vp"], st["vs"]) = (_int4_encode(normal(n_phys, hkv, g, d)) for _ in range(2))
        st["q_out"] = torch.zeros(T, hq, d, dtype=dt, device="cuda")
        st["k_out"] = st["v_out"] = None
        if case["kv"] == "int4":                      # the values the codes stand for: what the prompt's own attention goes on with
            st["k_out"], st["v_out"] = (torch.zeros(T, hkv, d, dtype=dt, device="cuda") for _ in range(2))
    else:
        lens = _ints(case["lens"])
        N, B, hq = len(lens), case["block"], case["q_heads"]
        st["page_table"], n_phys = _table(gen, lens, g)
        kp, ks, vp, vs = [], [], [], []
        for at in range(0, n_phys, 2048):
            n = min(2048, n_phys - at)
            for x, codes, scales in ((normal(n, hkv, g, d) * channel[:, None], kp, ks), (normal(n, hkv, g, d), vp, vs)):
                c, b = _int4_encode(x.bfloat16().float())
                codes.append(c)
                scales.append(b)
        st["kp"], st["ks"], st["vp"], st["vs"] = (torch.cat(x) for x in (kp, ks, vp, vs))
        st["kv_len"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        st["q"] = (normal(N, B, hq, d) * 1.5).bfloat16()
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(N, B, hq, device="cuda")
        if case["op"] == "listed":
            m, pmax = case["active"], st["page_table"].shape[1]
            pick = torch.rand(N, B, generator=gen, device="cuda").argsort(1)[:, :m].sort(1).values
            st["active_idx"] = torch.full((N, B), -1, dtype=torch.int32, device="cuda")
            st["active_idx"][:, :m] = pick.int()
            st["n_active"] = torch.full((N,), m, dtype=torch.int32, device="cuda")
            have = (st["kv_len"].long() + g - 1) // g
            rank = torch.rand(N, hkv, pmax, generator=gen, device="cuda") + 2.0 * (torch.arange(pmax, device="cuda") >= have[:, None, None])
            count = have.clamp_max(case["pages"])[:, None].expand(N, hkv)
            order = rank.argsort(-1)
            keep = torch.arange(pmax, device="cuda") < count[..., None]
            st["union_pages"] = torch.where(keep, order, pmax).sort(-1).values.int()
            st["union_pages"][st["union_pages"] == pmax] = -1
            st["union_count"] = count.int().contiguous()
    if own:
        _bind(st)
    return st


def _bind(st):
    """The handles an engine keeps: a context, the cache's description, the call's arguments."""
    from paper_2604_12056_b200 import binding as B
    c = st["case"]
    N, pmax = st["page_table"].shape
    dtype = B.LOSA_F32 if c.get("dtype") == "f32" else B.LOSA_BF16
    st["B"] = B
    st["ctx"] = B.Context(N, c["q_heads"], c["kv_heads"], c["dim"], c.get("block", 1), c["page"], pmax, dtype, c["dim"] ** -0.5)
    st["kv"] = B.make_kv(st["kp"], st["vp"], st.get("kmin"), st.get("kmax"), st["page_table"], st["kv_len"], st["ks"], st["vs"])
    if c["op"] == "append":
        st["rope"] = B.make_rope(st["cos"], st["sin"], interleaved=c["pairs"] == "neighbours")
        st["tokens"] = B.make_new_tokens(st["q"], st["k"], st["v"], st["cu"], st["start"], q_out=st["q_out"], k_out=st["k_out"], v_out=st["v_out"])
    elif c["op"] == "listed":
        unused = torch.zeros(1, device="cuda")
        st["state"] = B.make_state(unused, st["out"], st["lse"], unused)


def run(state):
    op = state["case"]["op"]
    if own:
        B = state["B"]
        if op == "append":
            B.losa_rope_append(state["ctx"], state["kv"], state["rope"], state["tokens"])
            return _appended(state)
        if op == "attn":
            B.losa_int4_attn(state["ctx"], state["q"], state["kv"], state["out"], state["lse"])
        else:
            B.losa_sparse_prefix_attn(state["ctx"], state["q"], state["kv"], state["active_idx"], state["n_active"],
                                      state["union_pages"], state["union_count"], state["state"])
        return state["out"], state["lse"]
    if op == "append":
        return _plain_append(state)
    return _plain_attn(state)


# ---------------------------------------------------------------- the plain forms
def _appended(st):
    out = {"q": st["q_out"], "kmin": st["kmin"], "kmax": st["kmax"], "kv_len": st["kv_len"]}
    kind = st["case"]["kv"]
    if kind == "int4":
        out |= {"k": st["k_out"], "v": st["v_out"]}
    elif kind == "fp8":
        out |= {"k": st["kp"].view(torch.float8_e4m3fn), "v": st["vp"].view(torch.float8_e4m3fn), "ks": st["ks"], "vs": st["vs"]}
    else:
        out |= {"k": st["kp"], "v": st["vp"]}
    return out


def _rotate(x, cos, sin, rot, pairs):
    """x [T, H, d] in 32 bits, cos / sin [T, 1, rot/2]."""
    r, rest = x[..., :rot], x[..., rot:]
    if pairs == "split":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = r[..., 0::2], r[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _plain_append(st):
    c, g = st["case"], st["case"]["page"]
    T, dt = st["q"].shape[0], st["q"].dtype
    t = torch.arange(T, device="cuda")
    seq = torch.searchsorted(st["cu"][1:].long(), t, right=True)
    pos = st["start"].long()[seq] + t - st["cu"].long()[seq]
    cos, sin = st["cos"][pos][:, None], st["sin"][pos][:, None]
    st["q_out"].copy_(_rotate(st["q"].float(), cos, sin, c["rot"], c["pairs"]).to(dt))
    k, v = _rotate(st["k"].float(), cos, sin, c["rot"], c["pairs"]).to(dt), st["v"]
    phys, at = st["page_table"].long()[seq, pos // g], pos % g
    ts, tp, first = st["touched"]
    pages = st["page_table"].long()[ts, tp]                     # touched pages
    end = (st["start"] + st["cu"][1:] - st["cu"][:-1]).long()
    valid = (tp[:, None] * g + torch.arange(g, device="cuda") < end[ts][:, None])[:, None, :, None]
    if c["kv"] == "native":
        st["kp"][phys, :, at] = k
        st["vp"][phys, :, at] = v
        rows = st["kp"][pages].float()
    elif c["kv"] == "int4":
        for x, codes, scales, out in ((k, st["kp"], st["ks"], st["k_out"]), (v, st["vp"], st["vs"], st["v_out"])):
            code, byte = _int4_encode(x.float())
            codes[phys, :, at] = code
            scales[phys, :, at] = byte
            out.copy_(_int4_decode(code, byte).to(dt))
        rows = _int4_decode(st["kp"][pages], st["ks"][pages])
    else:
        item = first[seq] + pos // g                            # which touched page a token falls into
        rows = None
        for x, codes, scales in ((k, st["kp"], st["ks"]), (v, st["vp"], st["vs"])):
            page = codes[pages].view(torch.float8_e4m3fn).float() * scales[pages][..., None, None]
            page[item, :, at] = x.float()
            page = torch.where(valid, page, 0.0)
            amax = page.abs().amax((2, 3), keepdim=True)
            bits = amax.contiguous().view(torch.int32)
            e = ((bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(-6, 7)
            scale = torch.exp2(e.float())
            code = (page / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
            codes[pages] = code.view(torch.uint8)
            scales[pages] = scale[..., 0, 0]
            if rows is None:
                rows = code.float() * scale
    st["kmin"][pages] = torch.where(valid, rows, math.inf).amin(2).to(dt)
    st["kmax"][pages] = torch.where(valid, rows, -math.inf).amax(2).to(dt)
    st["kv_len"].copy_(end.int())
    return _appended(st)


def _plain_attn(st):
    c, g = st["case"], st["case"]["page"]
    hkv, d, B = c["kv_heads"], c["dim"], c["block"]
    G = c["q_heads"] // hkv
    N, pmax = st["page_table"].shape
    table, within = st["page_table"].long(), torch.arange(g, device="cuda")
    q, tokens = st["q"], None
    if c["op"] == "listed":
        m = c["active"]
        tokens = st["active_idx"][:, :m].long()
        q = q.gather(1, tokens[:, :, None, None].expand(-1, -1, c["q_heads"], d))
        pages = st["union_pages"].long()[..., :min(c["pages"], pmax)]                     # [N, Hkv, P]
        kv_page = table.gather(1, pages.clamp_min(0).flatten(1)).view_as(pages)
        head = torch.arange(hkv, device="cuda")[None, :, None]
        k, v = (_int4_decode(p[kv_page, head], s[kv_page, head]).flatten(2, 3) for p, s in ((st["kp"], st["ks"]), (st["vp"], st["vs"])))
        at = (pages[..., None] * g + within).flatten(2)
        valid = (at < st["kv_len"][:, None, None]) & (pages >= 0).repeat_interleave(g, -1)       # [N, Hkv, t]
    else:
        k, v = (_int4_decode(p[table], s[table]).transpose(1, 2).flatten(2, 3) for p, s in ((st["kp"], st["ks"]), (st["vp"], st["vs"])))
        valid = (torch.arange(pmax * g, device="cuda") < st["kv_len"][:, None])[:, None]         # [N, 1, t]
    rows = q.float().unflatten(2, (hkv, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)                 # [N, Hkv, m G, d]
    s = (rows @ k.transpose(-1, -2)) * d ** -0.5
    s = torch.where(valid[:, :, None], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, 1.0)
    lse = (torch.log(total) + top)[..., 0]
    o = o.unflatten(2, (-1, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    lse = lse.unflatten(2, (-1, G)).permute(0, 2, 1, 3).flatten(2, 3)
    if tokens is None:
        st["out"].copy_(o.bfloat16())
        st["lse"].copy_(lse)
    else:
        st["out"].scatter_(1, tokens[:, :, None, None].expand_as(o), o.bfloat16())
        st["lse"].scatter_(1, tokens[:, :, None].expand_as(lse), lse)
    return st["out"], st["lse"]


# ---------------------------------------------------------------- the same in 64 bits, sequence by sequence from the definitions
_NIBBLE = [i - 8 for i in range(16)]


def _exact_int4(codes, byte):
    """Values of packed rows, by tables."""
    scale = torch.tensor([2.0 ** ((b >> 3) - 15) * (1 + (b & 7) / 8) if b >> 3 else 2.0 ** -14 * (b & 7) / 8 for b in range(256)], dtype=torch.float64, device="cuda")
    value = torch.tensor(_NIBBLE, dtype=torch.float64, device="cuda")
    x = torch.empty(*codes.shape[:-1], codes.shape[-1] * 2, dtype=torch.float64, device="cuda")
    x[..., 0::2], x[..., 1::2] = value[(codes % 16).long()], value[(codes // 16).long()]
    return x * scale[byte.long()].repeat_interleave(32, -1)


def _exact_quantise(x):
    """What a 4-bit cache holds for rows x."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    m, e = torch.frexp(g.abs().amax(-1, keepdim=True) / 7)
    s = torch.ldexp(torch.ceil(m * 16) / 16, e).clamp(2.0 ** -12, 960)
    return (torch.floor(g.abs() / s + 0.5).clamp_max(7) * torch.sign(g) * s).reshape(x.shape)


def _exact_fp8(page):
    """What an FP8 page [.., g, d] holds."""
    amax = page.abs().amax((-1, -2), keepdim=True)
    m, e = torch.frexp(amax / 448.0)                            # m 2^e, m from 0.5 up
    scale = torch.exp2((e - (m == 0.5).int()).clamp(-6, 7).double())
    code = (page / scale).clamp(-448, 448)
    step = torch.exp2((torch.frexp(code.abs().clamp_min(2.0 ** -6))[1] - 4).double())
    return torch.round(code / step) * step, scale


def exact(case, seed):
    st = prepare(case, seed)
    hkv, d, g = case["kv_heads"], case["dim"], case["page"]
    if case["op"] == "append":
        return _exact_append(case, st)
    out, lse = st["out"].double(), st["lse"].double()
    G = case["q_heads"] // hkv
    for s, L in enumerate(_ints(case["lens"])):
        tokens = torch.arange(case["block"], device="cuda") if case["op"] == "attn" else st["active_idx"][s, :case["active"]].long()
        for h in range(hkv):
            pages = torch.arange(-(-L // g), device="cuda")
            if case["op"] == "listed":
                pages = st["union_pages"][s, h, :int(st["union_count"][s, h])].long()
            t = (pages[:, None] * g + torch.arange(g, device="cuda")).reshape(-1)
            phys = st["page_table"][s, pages].long()
            k, v = (_exact_int4(p[phys, h], b[phys, h]).reshape(-1, d)[t < L] for p, b in ((st["kp"], st["ks"]), (st["vp"], st["vs"])))
            for heads in (slice(h * G, (h + 1) * G),):
                q = st["q"][s, tokens, heads].double().reshape(-1, d)
                sc = q @ k.T / math.sqrt(d)
                l = torch.logsumexp(sc, -1)
                o = torch.exp(sc - l[:, None]) @ v if k.shape[0] else torch.zeros_like(q)
                out[s, tokens, heads] = o.reshape(-1, G, d)
                lse[s, tokens, heads] = l.reshape(-1, G)
    return out, lse


def _exact_append(case, st):
    g, hkv, d, half = case["page"], case["kv_heads"], case["dim"], case["rot"] // 2
    new, start = _ints(case["new"]), _ints(case["start"])
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    pos = torch.cat([torch.arange(a, a + n, device="cuda") for a, n in zip(start, new)])
    turn = torch.complex(st["cos"].double(), st["sin"].double())[pos][:, None]
    for x in (q, k):
        i, j = (slice(0, half), slice(half, 2 * half)) if case["pairs"] == "split" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
        y = torch.complex(x[..., i], x[..., j]) * turn
        x[..., i], x[..., j] = y.real, y.imag
    elem = k.bfloat16().double() if case["dtype"] == "bf16" else k.float().double()        # as the quantised formats take it
    kmin, kmax = st["kmin"].double(), st["kmax"].double()
    if case["kv"] == "native":
        kp, vp = st["kp"].double(), st["vp"].double()
    elif case["kv"] == "fp8":
        kp, vp = (p.view(torch.float8_e4m3fn).double() for p in (st["kp"], st["vp"]))
        ks, vs = st["ks"].double(), st["vs"].double()
    else:
        k, v = _exact_quantise(elem), _exact_quantise(v)
    first = 0
    for s, (a, n) in enumerate(zip(start, new)):
        for p in range(a // g, -(-(a + n) // g) if n else 0):
            phys = int(st["page_table"][s, p])
            lo, hi = max(a, p * g), min(a + n, (p + 1) * g)
            src, dst = slice(first + lo - a, first + hi - a), slice(lo - p * g, hi - p * g)
            if case["kv"] == "native":
                kp[phys, :, dst], vp[phys, :, dst] = k[src].transpose(0, 1), v[src].transpose(0, 1)
                rows = kp[phys]
            elif case["kv"] == "fp8":
                for x, pool, scales in ((elem, kp, ks), (v, vp, vs)):
                    page = pool[phys] * scales[phys][:, None, None]
                    page[:, dst] = x[src].transpose(0, 1)
                    page[:, hi - p * g:] = 0
                    pool[phys], sc = _exact_fp8(page)
                    scales[phys] = sc[:, 0, 0]
                rows = kp[phys] * ks[phys][:, None, None]
            else:
                rows = _exact_int4(st["kp"][phys], st["ks"][phys])
                rows[:, dst] = k[src].transpose(0, 1)
            kmin[phys], kmax[phys] = rows[:, :hi - p * g].amin(1), rows[:, :hi - p * g].amax(1)
        first += n
    out = {"q": q, "kmin": kmin, "kmax": kmax, "kv_len": None}
    if case["kv"] == "int4":
        return out | {"k": k, "v": v}
    if case["kv"] == "fp8":
        return out | {"k": kp, "v": vp, "ks": ks, "vs": vs}
    return out | {"k": kp, "v": vp}


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    hq, hkv, d, g = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    row4 = d // 2 + d // 32                                     # a 4-bit row and its scales
    if case["op"] == "append":
        new, start = _ints(case["new"]), _ints(case["start"])
        T, es = sum(new), 2 if case["dtype"] == "bf16" else 4
        kept = {"native": d * es, "fp8": d, "int4": row4}[case["kv"]]
        old = sum(a % g for a, n in zip(start, new) if n) * hkv * kept * (3 if case["kv"] == "fp8" else 1)   # (FP8: keys and values, read; written again)
        touched = sum(-(-(a + n) // g) - a // g for a, n in zip(start, new) if n)
        b = T * d * es * (2 * hq + 2 * hkv) + 2 * T * hkv * kept + old + touched * hkv * 2 * d * es + T * case["rot"] * 4
        if case["kv"] == "int4":
            b += 2 * T * hkv * d * es
        return {"bytes": b, "flops": 3 * T * (hq + hkv) * case["rot"] + 2 * T * hkv * d}
    lens, B = _ints(case["lens"]), case["block"]
    m = case.get("active", B)
    tokens = sum(min(L, case["pages"] * g) if case["op"] == "listed" else L for L in lens)
    return {"bytes": tokens * hkv * 2 * row4 + len(lens) * m * hq * (4 * d + 4), "flops": 4.0 * m * hq * d * tokens}
