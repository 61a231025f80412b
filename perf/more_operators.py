"""Work of the operators that keep a paged cache bounded, as cases that are timed and compared: attention with a sliding
window and a few first tokens that stay visible, the softmax weight that every cached token receives, and eviction by it.

An engine keeps one paged cache per attention layer.  New tokens attend to it (`losa_window_attn`: prompts, blocks that
are not in it yet, single tokens), the weight that each cached token gets is added up (`losa_kv_weights`), and when a
sequence outgrows its budget its tokens of least weight leave (`losa_kv_evict`).  A case is one such call:

  op = "window"   new tokens of every sequence over the keys that each of them sees
       "weights"  the keys' weights from the same tokens, added to those that were there
       "evict"    sequences cut down to their budgets, head by head

With `own` false, `run` computes the same in elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import torch

own = False

QWEN = {"q_heads": 32, "kv_heads": 8, "dim": 128}


def _attn(name, op, new, start, *, stored=True, window=0, sinks=0, span=1, page=32, dtype="bf16", kv="native", **heads):
    c = {"name": name, "op": op, "new": new, "start": start, "stored": stored, "window": window, "sinks": sinks, "span": span, "page": page, "dtype": dtype, "kv": kv}
    c.update(heads or QWEN)
    return c


def _evict(name, lens, budgets, *, sinks=4, recent=32, page=32, dtype="bf16", kv="native", **heads):
    c = {"name": name, "op": "evict", "lens": lens, "budgets": budgets, "sinks": sinks, "recent": recent, "page": page, "dtype": dtype, "kv": kv}
    c.update(heads or QWEN)
    return c


def _text(values):
    return ",".join(str(v) for v in values)


def listed():
    short = _text((i * 577 + 31) % 4096 for i in range(64))
    return [
        # decoding step of 64 short ragged sequences, few keys each: latency
        _attn("window_tokens_64", "window", _text([1] * 64), short, window=512, sinks=4),
        # decoding step of eight 32K sequences with a long window: bandwidth
        _attn("window_tokens_8x32k", "window", _text([1] * 8), _text([32768] * 8), window=8192, sinks=4),
        # decoding step over the whole of an 8-bit cache, a scale for each page and head
        _attn("tokens_fp8_8x16k", "window", _text([1] * 8), "16383,12001,16000,9999,16383,777,15000,16383", kv="fp8"),
        # a block that is being denoised, not in the cache yet, over the window before it
        _attn("window_blocks", "window", _text([32] * 8), "32768,16381,24571,32003,8191,0,20000,11", stored=False, window=4096, sinks=16),
        # prompts of a ragged batch, two of them behind earlier turns
        _attn("window_prompts", "window", "8191,4097,1,2875", "0,0,511,1000", window=1024, sinks=4),
        # a long prompt
        _attn("window_prompt_16k", "window", "16384", "0", window=4096, sinks=4),
        # fp32 model check: small heads, blocks of 16 that see themselves whole
        _attn("window_prompts_f32", "window", "1024,777", "0,5", window=333, sinks=3, span=16, page=16, dtype="f32", q_heads=4, kv_heads=1, dim=64),
        # what a decoding step of eight 16K sequences gives to the cached tokens: the keys' bandwidth
        _attn("weights_tokens", "weights", _text([1] * 8), "16383,12001,16000,9999,16383,777,15000,16383"),
        # what the last 64 tokens of a long prompt look at
        _attn("weights_last_64", "weights", "64,64", "32704,20001"),
        # what all tokens of a prompt look at
        _attn("weights_prompt_8k", "weights", "8192", "0"),
        # one interactive sequence in 8 bits outgrows its budget
        _evict("evict_one_fp8", "8201", "2048", kv="fp8"),
        # a serving batch cut to a quarter, one sequence that is within its budget
        _evict("evict_8x16k", "16384,16384,12001,16000,4000,15555,16384,9999", _text([4096] * 8)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max((work(c) for c in listed()), key=lambda w: w["flops"])["flops"]
    while True:
        c = _drawn(rng)
        w = work(c)
        if w["flops"] <= most and w["bytes"] <= 1.5e9:
            return c


def _drawn(rng):
    hkv, G, d = rng.choice([(8, 4, 128), (8, 4, 128), (4, 8, 64), (2, 5, 128), (1, 4, 64), (4, 1, 128), (2, 16, 128)])
    heads = {"q_heads": hkv * G, "kv_heads": hkv, "dim": d}
    page = rng.choice([16, 32, 32, 64])
    dtype, kv = rng.choice([("bf16", "native"), ("bf16", "native"), ("bf16", "native"), ("bf16", "fp8"), ("f32", "native")])
    op = rng.choice(["window", "window", "weights", "evict"])
    n = rng.choice([1, 2, 3, 8, 17])
    if op == "evict":
        total = _log_int(rng, 64 * n, 100000)
        lens = [max(1, int(total / n * rng.uniform(0.2, 1.8))) for _ in range(n)]
        budgets = [max(1, int(L * rng.uniform(0.1, 1.1))) for L in lens]
        c = _evict("", _text(lens), _text(budgets), sinks=rng.choice([0, 1, 4, 16]), recent=rng.choice([0, 1, 32, 100]), page=page, dtype=dtype, kv=kv, **heads)
    else:
        # as many tokens as a decoding step, a block, or prompts have
        kind = rng.choice(["token", "block", "prompt"])
        if kind == "token":
            new = [1] * n
        elif kind == "block":
            new = [rng.choice([2, 4, 8, 16, 32])] * n
        else:
            total = _log_int(rng, 8 * n, 4000 if dtype == "f32" else 12000)
            new = [max(0, int(total / n * rng.uniform(0.2, 1.8))) for _ in range(n)]
            new[0] = max(1, new[0])
        start = [rng.choice([0, rng.randrange(4096)]) if kind == "prompt" else rng.randrange(_log_int(rng, 16, 30000)) for _ in range(n)]
        window = rng.choice([0, 0, 128, 333, 1024, 4096])
        c = _attn("", op, _text(new), _text(start), stored=kind != "block", window=window, sinks=rng.choice([0, 4, 16, 100]) if window else 0,
                  span=rng.choice([1, 1, 32]), page=page, dtype=dtype, kv=kv, **heads)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs
def _ints(text):
    return [int(v) for v in text.split(",")]


def _lengths(case):
    """Tokens in the cache."""
    if case["op"] == "evict":
        return _ints(case["lens"])
    return [a + (b if case["stored"] else 0) for a, b in zip(_ints(case["start"]), _ints(case["new"]))]


def _fp8_page(x):
    """fp32 pages [.., g, d] -> (codes as float8, scales [..])."""
    bits = x.abs().amax((-1, -2)).view(torch.int32)
    e = ((bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(-6, 7)
    scale = torch.exp2(e.float())
    return (x / scale[..., None, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 17)
    hq, hkv, d, g = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    lens = _lengths(case)
    N, pmax = len(lens), max(1, max(-(-L // g) for L in lens))
    n_phys = N * pmax
    st = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    st["page_table"] = torch.randperm(n_phys, generator=gen, device="cuda").view(N, pmax).int()
    st["kv_len"] = ints(lens)
    # keys have channels that stand out, as rotated keys of trained models do
    channel = 1.0 + 2.0 * (torch.rand(hkv, 1, d, generator=gen, device="cuda") > 0.94)
    k, v = (normal(n_phys, hkv, g, d) * channel).to(dt), normal(n_phys, hkv, g, d).to(dt)
    st["ks"] = st["vs"] = None
    if case["kv"] == "fp8":
        # slots behind a sequence's end hold zeros
        page_len = torch.zeros(n_phys, dtype=torch.int64, device="cuda")
        page_len[st["page_table"].long()] = st["kv_len"].long()[:, None] - torch.arange(pmax, device="cuda") * g
        live = torch.arange(g, device="cuda") < page_len[:, None]
        (k, st["ks"]), (v, st["vs"]) = (_fp8_page(torch.where(live[:, None, :, None], x.float(), 0.0)) for x in (k, v))
        k, v = k.view(torch.uint8), v.view(torch.uint8)
    st["kp"], st["vp"] = k.contiguous(), v.contiguous()
    if case["op"] == "evict":
        # weights as they add up over many steps: a few tokens have most of them
        st["weights"] = torch.exp(2.0 * normal(n_phys, hkv, g))
        st["kmin"], st["kmax"] = (torch.zeros(n_phys, hkv, d, dtype=dt, device="cuda") for _ in range(2))
        st["length"], st["budget"] = ints(lens), ints(_ints(case["budgets"]))
        st["kept"] = torch.full((N, hkv, max(min(b, L) for b, L in zip(_ints(case["budgets"]), lens))), -1, dtype=torch.int32, device="cuda")
    else:
        new = _ints(case["new"])
        T = sum(new)
        st["q"] = (normal(T, hq, d) * 1.5).to(dt)
        st["cu"] = torch.tensor([0] + new, device="cuda").cumsum(0).int()
        st["start"] = ints(_ints(case["start"]))
        st["max_tokens"] = max(new)
        st["out"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(T, hq, device="cuda")
        if case["op"] == "weights":
            _plain_window(st)                                   # the attention before it leaves its log-normalisers
            st["weights"] = torch.rand(n_phys, hkv, g, generator=gen, device="cuda")
    if own:
        _bind(st)
    return st


def _bind(st):
    """The handles an engine keeps: a context, the cache's description, the call's arguments."""
    from paper_2604_12056_b200 import binding as B
    c = st["case"]
    N, pmax = st["page_table"].shape
    st["B"] = B
    st["ctx"] = B.Context(N, c["q_heads"], c["kv_heads"], c["dim"], 1, c["page"], pmax, B.LOSA_F32 if c["dtype"] == "f32" else B.LOSA_BF16, c["dim"] ** -0.5)
    st["cache"] = B.make_kv(st["kp"], st["vp"], st.get("kmin"), st.get("kmax"), st["page_table"], st["kv_len"], st["ks"], st["vs"])
    if c["op"] == "evict":
        st["eviction"] = B.make_eviction(st["length"], st["budget"], st["kept"], sinks=c["sinks"], recent=c["recent"])
    else:
        st["queries"] = B.make_queries(st["q"], st["cu"], st["start"], st["max_tokens"], window=c["window"], sinks=c["sinks"], span=c["span"])


def run(state):
    op = state["case"]["op"]
    if own:
        B = state["B"]
        if op == "window":
            B.losa_window_attn(state["ctx"], state["queries"], state["cache"], state["out"], state["lse"])
        elif op == "weights":
            B.losa_kv_weights(state["ctx"], state["queries"], state["cache"], state["lse"], state["weights"])
        else:
            B.losa_kv_evict(state["ctx"], state["cache"], state["weights"], state["eviction"])
    elif op == "window":
        _plain_window(state)
    elif op == "weights":
        _plain_weights(state)
    else:
        _plain_evict(state)
    if op == "window":
        return state["out"], state["lse"]
    if op == "weights":
        return state["weights"]
    fp8 = state["case"]["kv"] == "fp8"
    out = {n: state[n].view(torch.float8_e4m3fn) if fp8 else state[n] for n in ("kp", "vp")}
    out |= {n: state[n] for n in ("kmin", "kmax", "weights", "kept", "kv_len")}
    return out | {"ks": state["ks"], "vs": state["vs"]} if fp8 else out


# ---------------------------------------------------------------- the plain forms
def _dense(st, pool, scale):
    """A paged tensor as fp32 [N, P g, H, ..]."""
    x = pool[st["page_table"].long()]                           # [N, P, H, g, d]
    if scale is not None:
        x = x.view(torch.float8_e4m3fn).float() * scale[st["page_table"].long()][..., None, None]
    return x.float().transpose(2, 3).flatten(1, 2)


def _bands(st):
    """Queries in runs of c tokens and the keys that each run may see: q [N, R, H, c G, d], the query's token (T: none) [N, R, c], keys'
    places [N, R, K], and which row sees which [N, R, c, K]."""
    c, lens = st["case"], _lengths(st["case"])
    new, T, L = _ints(c["new"]), st["q"].shape[0], max(1, max(lens))
    m, W, span = st["max_tokens"], c["window"], c["span"]
    run = min(m, 512 if not W else max(64, min(512, W)))
    R = -(-m // run)
    i = torch.arange(R * run, device="cuda").view(R, run)
    count = st["cu"][1:] - st["cu"][:-1]
    token = torch.where(i < count[:, None, None], st["cu"][:-1, None, None] + i, T).long()
    place = st["start"].long()[:, None, None] + i                                            # [N, R, c]
    if W:
        K = min(L, W + run + span - 1)
        band = (place[..., :1] + 1 - W).clamp_min(0) + torch.arange(K, device="cuda")
        first = torch.arange(c["sinks"], device="cuda").expand(*band.shape[:2], c["sinks"])
        at = torch.cat([first, band], -1)
        fresh = torch.cat([torch.ones_like(first, dtype=torch.bool), band >= c["sinks"]], -1)         # (each key once)
    else:
        at = torch.arange(L, device="cuda").expand(len(new), R, L)
        fresh = torch.ones_like(at, dtype=torch.bool)
    end = torch.minimum((place // span + 1) * span, st["kv_len"].long()[:, None, None])
    sees = (at[:, :, None] < end[..., None]) & fresh[:, :, None] & (token < T)[..., None]
    if W:
        sees &= (at[:, :, None] > place[..., None] - W) | (at < c["sinks"])[:, :, None]
    hkv, d = c["kv_heads"], c["dim"]
    q = torch.cat([st["q"].float(), torch.zeros_like(st["q"][:1]).float()])[token]                    # [N, R, c, Hq, d]
    q = q.unflatten(3, (hkv, -1)).transpose(2, 3).flatten(3, 4)
    return q, token, at, sees


def _scores(st):
    """Scores [N, R, H, c, G, K] of _bands, -inf where a row does not see a key."""
    c = st["case"]
    q, token, at, sees = _bands(st)
    n = torch.arange(at.shape[0], device="cuda")[:, None, None]
    k = _dense(st, st["kp"], st["ks"])
    inside = at.clamp_max(k.shape[1] - 1)
    k = k[n, inside].transpose(2, 3)                            # [N, R, H, K, d]
    s = (q @ k.transpose(-1, -2)).mul_(c["dim"] ** -0.5).unflatten(3, (token.shape[2], -1))
    return s.masked_fill_(~sees[:, :, None, :, None], -math.inf), token, inside, n


def _plain_window(st):
    s, token, at, n = _scores(st)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    v = _dense(st, st["vp"], st["vs"])[n, at].transpose(2, 3)
    o = (p.flatten(3, 4) @ v).unflatten(3, p.shape[3:5]) / torch.where(total > 0, total, 1.0)      # [N, R, H, c, G, d]
    lse = (torch.log(total) + top)[..., 0]
    have = token < st["q"].shape[0]
    st["out"][token[have]] = o.transpose(2, 3).flatten(3, 4)[have].to(st["out"].dtype)
    st["lse"][token[have]] = lse.transpose(2, 3).flatten(3, 4)[have]


def _plain_weights(st):
    c, g = st["case"], st["case"]["page"]
    s, token, at, _ = _scores(st)
    N, R, H = s.shape[:3]
    lse = torch.cat([st["lse"], torch.zeros_like(st["lse"][:1])])[token].unflatten(-1, (H, -1)).transpose(2, 3)     # [N, R, H, c, G]
    p = s.sub_(torch.where(lse > -math.inf, lse, 0.0)[..., None]).exp_().sum((3, 4))                                # [N, R, H, K]
    table = st["page_table"].long()
    L = table.shape[1] * g
    got = torch.zeros(N, H, L, device="cuda").scatter_add_(2, at.flatten(1)[:, None].expand(-1, H, -1), p.transpose(1, 2).flatten(2))
    place = torch.arange(L, device="cuda")
    old = st["weights"][table].transpose(1, 2).flatten(2)                                                           # [N, H, L]
    kept = torch.where((place < st["start"][:, None])[:, None], old, 0.0) + got
    kept = torch.where((place < st["kv_len"][:, None])[:, None], kept, old)
    st["weights"][table] = kept.unflatten(2, (-1, g)).transpose(1, 2)


def _plain_evict(st):
    c, g = st["case"], st["case"]["page"]
    table, length, budget = st["page_table"].long(), st["length"].long(), st["budget"].long()
    N, pmax = table.shape
    L, b = pmax * g, st["kept"].shape[2]
    hkv = c["kv_heads"]
    goes = budget < length                                      # sequences that lose tokens
    place = torch.arange(L, device="cuda")
    w = st["weights"][table].transpose(1, 2).flatten(2)         # [N, H, L]
    sinks = torch.minimum(torch.full_like(budget, c["sinks"]), budget)
    recent = torch.minimum(torch.full_like(budget, c["recent"]), budget - sinks)
    always = (place < sinks[:, None]) | (place >= (length - recent)[:, None])
    w = torch.where(always[:, None], math.inf, w)
    w = torch.where((place < length[:, None])[:, None], w, -math.inf)
    order = w.sort(dim=2, descending=True, stable=True).indices
    taken = torch.where((place < budget[:, None])[:, None], order, L).sort(2).values[..., :b]       # [N, H, b], L: none
    real = (taken < L) & goes[:, None, None]
    st["kept"].copy_(torch.where(real, taken, st["kept"]).int())
    s, h, to = torch.nonzero(real, as_tuple=True)
    src = taken[s, h, to]
    from_page, from_slot, to_page, to_slot = table[s, src // g], src % g, table[s, to // g], to % g
    st["weights"][to_page, h, to_slot] = st["weights"][from_page, h, from_slot]
    ps, pp = torch.nonzero(goes[:, None] & (torch.arange(pmax, device="cuda") * g < budget[:, None]), as_tuple=True)
    pages = table[ps, pp]                                       # what the sequences that lose tokens keep
    live = (pp[:, None] * g + torch.arange(g, device="cuda") < budget[ps][:, None])[:, None, :, None]
    if c["kv"] == "fp8":
        item = (torch.cumsum(goes * ((budget + g - 1) // g), 0) - (budget + g - 1) // g)[s] + to // g      # which of these pages a token goes to
        rows = None
        for pool, scales in ((st["kp"], st["ks"]), (st["vp"], st["vs"])):
            page = torch.zeros(len(pages), hkv, g, c["dim"], device="cuda")
            page[item, h, to_slot] = pool[from_page, h, from_slot].view(torch.float8_e4m3fn).float() * scales[from_page, h][:, None]
            code, scale = _fp8_page(page)
            pool[pages], scales[pages] = code.view(torch.uint8), scale
            rows = code.float() * scale[..., None, None] if rows is None else rows
    else:
        for pool in (st["kp"], st["vp"]):
            pool[to_page, h, to_slot] = pool[from_page, h, from_slot]
        rows = st["kp"][pages].float()
    st["kmin"][pages] = torch.where(live, rows, math.inf).amin(2).to(st["kmin"].dtype)
    st["kmax"][pages] = torch.where(live, rows, -math.inf).amax(2).to(st["kmax"].dtype)
    st["kv_len"].copy_(torch.where(goes, budget, st["kv_len"]).int())


# ---------------------------------------------------------------- the same in 64 bits, sequence by sequence from the definitions
def _rows64(st, pool, scales, s, h, L):
    """Rows of one sequence and head, float64."""
    g = st["case"]["page"]
    pages = st["page_table"][s, :-(-L // g)].long()
    x = pool[pages, h]
    x = x.view(torch.float8_e4m3fn).double() * scales[pages, h].double()[:, None, None] if scales is not None else x.double()
    return x.flatten(0, 1)[:L]


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "evict":
        return _exact_evict(case, st)
    hkv, d, g, span, W = case["kv_heads"], case["dim"], case["page"], case["span"], case["window"]
    G = case["q_heads"] // hkv
    new, start, lens = _ints(case["new"]), _ints(case["start"]), _lengths(case)
    out, lse = st["out"].double(), st["lse"].double()
    weights = st["weights"].double() if case["op"] == "weights" else None
    first = 0
    for s in range(len(new)):
        for h in range(hkv):
            k, v = (_rows64(st, p, b, s, h, lens[s]) for p, b in ((st["kp"], st["ks"]), (st["vp"], st["vs"])))
            got = torch.zeros(lens[s], dtype=torch.float64, device="cuda")
            for a in range(0, new[s], 512):                     # tokens a .. z - 1, and the keys from lo to hi besides the sinks
                z = min(new[s], a + 512)
                place = torch.arange(start[s] + a, start[s] + z, device="cuda")
                end = ((place // span + 1) * span).clamp_max(lens[s])
                lo = max(0, int(place[0]) + 1 - W) if W else 0
                t = torch.cat([torch.arange(0, min(lo, case["sinks"], lens[s]), device="cuda"), torch.arange(lo, max(lo, int(end[-1])), device="cuda")])
                ok = t[None] < end[:, None]
                if W:
                    ok &= (t[None] >= place[:, None] + 1 - W) | (t[None] < case["sinks"])
                q = st["q"][first + a:first + z, h * G:(h + 1) * G].double()
                sc = torch.where(ok[:, None], torch.einsum("tgd,kd->tgk", q, k[t]) / math.sqrt(d), -math.inf)
                if weights is None:
                    l = torch.logsumexp(sc, -1) if len(t) else torch.full(sc.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
                    p = torch.exp(sc - torch.where(l > -math.inf, l, 0.0)[..., None])
                    out[first + a:first + z, h * G:(h + 1) * G] = torch.einsum("tgk,kd->tgd", p, v[t])
                    lse[first + a:first + z, h * G:(h + 1) * G] = l
                else:
                    l = st["lse"][first + a:first + z, h * G:(h + 1) * G].double()
                    got[t] += torch.exp(sc - torch.where(l > -math.inf, l, 0.0)[..., None]).sum((0, 1))
            if weights is not None:
                j = torch.arange(lens[s], device="cuda")
                page, slot = st["page_table"][s].long()[j // g], j % g
                weights[page, h, slot] = torch.where(j < start[s], weights[page, h, slot], 0.0) + got
        first += new[s]
    return (out, lse) if weights is None else weights


def _exact_evict(case, st):
    g = case["page"]
    pools = {n: st[n].view(torch.float8_e4m3fn).double() if case["kv"] == "fp8" else st[n].double() for n in ("kp", "vp")}
    ks, vs = (None if x is None else x.double() for x in (st["ks"], st["vs"]))
    kmin, kmax, weights = st["kmin"].double(), st["kmax"].double(), st["weights"].double()
    for s, (L, b) in enumerate(zip(_ints(case["lens"]), _ints(case["budgets"]))):
        if b >= L:
            continue
        pages = st["page_table"][s].long()
        sinks = min(case["sinks"], b)
        recent = min(case["recent"], b - sinks)
        for h in range(case["kv_heads"]):
            w = st["weights"][pages, h].flatten()[:L].cpu().tolist()
            middle = sorted(range(sinks, L - recent), key=lambda j: (-w[j], j))[:b - sinks - recent]
            keep = torch.tensor(sorted(list(range(sinks)) + middle + list(range(L - recent, L))), device="cuda")
            to = torch.arange(b, device="cuda")
            weights[pages[to // g], h, to % g] = st["weights"][pages[keep // g], h, keep % g].double()
            for name, scales, made in (("kp", st["ks"], ks), ("vp", st["vs"], vs)):
                rows = _rows64(st, st[name], scales, s, h, L)[keep]
                for p in range(-(-b // g)):
                    r = rows[p * g:(p + 1) * g]
                    if scales is not None:
                        m, e = torch.frexp(r.abs().max() / 448.0)                                # m 2^e, m from 0.5 up
                        scale = torch.exp2((e - (m == 0.5).int()).clamp(-6, 7).double())
                        code = (r / scale).clamp(-448, 448)
                        step = torch.exp2((torch.frexp(code.abs().clamp_min(2.0 ** -6))[1] - 4).double())
                        code = torch.round(code / step) * step
                        pools[name][pages[p], h] = 0.0
                        made[pages[p], h], r, code = scale, code * scale, code
                        pools[name][pages[p], h, :len(r)] = code
                    else:
                        pools[name][pages[p], h, :len(r)] = r
                    if name == "kp":
                        kmin[pages[p], h], kmax[pages[p], h] = r.amin(0), r.amax(0)
    out = {"kp": pools["kp"], "vp": pools["vp"], "kmin": kmin, "kmax": kmax, "weights": weights, "kept": None, "kv_len": None}
    return out | {"ks": ks, "vs": vs} if case["kv"] == "fp8" else out


# ---------------------------------------------------------------- what a pass cannot do without
def _seen(case):
    """(query, key) pairs, and keys that any query of a sequence sees, over all sequences."""
    pairs = keys = 0
    W, span, sinks = case["window"], case["span"], case["sinks"]
    for a, n, L in zip(_ints(case["start"]), _ints(case["new"]), _lengths(case)):
        if n == 0:
            continue
        t = torch.arange(a, a + n)
        end = ((t // span + 1) * span).clamp_max(L)
        lo = (t + 1 - W).clamp_min(0) if W else torch.zeros_like(t)
        pairs += int((end - torch.minimum(lo, end)).sum() + torch.minimum(torch.minimum(lo, end), torch.tensor(sinks)).sum())
        first, last = int(min(lo[0], end[-1])), int(end[-1])
        keys += last - first + min(first, sinks)
    return pairs, keys


def work(case):
    hq, hkv, d, g = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    es = 2 if case["dtype"] == "bf16" else 4
    row = d if case["kv"] == "fp8" else d * es
    if case["op"] == "evict":
        b = f = 0
        for L, k in zip(_ints(case["lens"]), _ints(case["budgets"])):
            if k < L:
                pages = -(-k // g)
                b += hkv * (L * 4 + k * (2 * 2 * row + 2 * 4 + 4) + pages * 2 * d * es)
                f += hkv * (L + k * d * 2)
        return {"bytes": float(max(b, 1)), "flops": float(max(f, 1))}
    pairs, keys = _seen(case)
    T = sum(_ints(case["new"]))
    if case["op"] == "window":
        return {"bytes": float(keys * hkv * 2 * row + T * hq * (2 * d * es + 4)), "flops": max(1.0, 4.0 * pairs * hq * d)}
    held = sum(_lengths(case))
    return {"bytes": float(keys * hkv * row + held * hkv * 8 + T * hq * (d * es + 4)), "flops": max(1.0, 2.0 * pairs * hq * d)}
