"""A cache that stays bounded: prompts with a sliding window, a block denoised behind them, decoded tokens, eviction by weight.

  python examples/bounded_cache.py

One attention layer with random inputs.  Queries and keys come unrotated, as projections give them:
  1. prompts of any length go into the cache rotated and attend to it with a window and first tokens that stay visible (`losa_window_attn`);
     what the cached tokens receive of it is added up (`losa_kv_weights`);
  2. a block is denoised against the window before it: the prefix part from `losa_window_attn`, the block part and the merge from stage 5; it is finalised;
  3. single tokens are appended and attend to the whole cache; sequences above the budget lose their tokens of least weight (`losa_kv_evict`).
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_12056_b200 import binding as B  # noqa: E402
from paper_2604_12056_b200 import workloads as wl  # noqa: E402
from paper_2604_12056_b200.layer import LosaLayer  # noqa: E402


def run(prompts=(1000, 37, 2100), block=32, steps=3, decode=4, window=512, sinks=4, budget=600, seed=0):
    """Outputs of the prompts, of the last denoising step, of the decoded tokens, and the lengths that are left."""
    hq, hkv, d, page, N = 32, 8, 128, 32, len(prompts)
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def project(T):                                   # queries, keys and values of T tokens, side by side
        row = torch.randn(T, hq + 2 * hkv, d, generator=gen, device="cuda").bfloat16()
        return row[:, :hq], row[:, hq:hq + hkv], row[:, hq + hkv:]

    def ints(*v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    cfg = wl.Config("example", 9, hq, hkv, d, page, tuple(L + block + decode for L in prompts), block, steps, 16, 4, "bf16", False)
    pool = torch.zeros(2, N * cfg.max_pages_per_seq, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    table = torch.randperm(pool.shape[1], generator=gen, device="cuda").view(N, -1).int()
    layer = LosaLayer(cfg, pool[0], pool[1], table, ints(*[0] * N))               # an empty cache
    angle = torch.arange(max(prompts) + block + decode, device="cuda").double()[:, None] * 1e6 ** (-torch.arange(d // 2, device="cuda").double() / (d // 2))
    rope = B.make_rope(angle.cos().float(), angle.sin().float())

    # 1. prompts
    q, k, v = project(sum(prompts))
    cu, start = ints(0, *prompts).cumsum(0).int(), ints(*[0] * N)
    rotated, out = (torch.empty(q.shape, dtype=q.dtype, device="cuda") for _ in range(2))
    lse = torch.empty(q.shape[:2], device="cuda")
    layer.append(B.make_new_tokens(q, k, v, cu, start, q_out=rotated), rope)
    queries = B.make_queries(rotated, cu, start, max(prompts), window=window, sinks=sinks)
    layer.attend(queries, out, lse)
    layer.add_weights(queries, lse)

    # 2. one block, which is not in the cache: its part of the softmax is merged by stage 5
    lens = layer.kv_len.clone()
    cu = torch.arange(N + 1, device="cuda").int() * block
    prefix, prefix_lse = torch.empty(N, block, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(N, block, hq, device="cuda")
    merged, merged_lse = torch.empty_like(prefix), torch.empty_like(prefix_lse)
    state = B.make_state(layer.q_prev, prefix, prefix_lse, layer.step)
    for _ in range(steps):
        q, k, v = project(N * block)
        qb, kb, vb = (torch.empty(N, block, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
        layer.rotate(B.make_new_tokens(q, k, None, cu, lens, q_out=qb, k_out=kb), rope)
        vb.copy_(v.view_as(vb))
        queries = B.make_queries(qb.view(-1, hq, d), cu, lens, block, window=window, sinks=sinks)
        layer.attend(queries, prefix, prefix_lse)
        B.losa_block_attn_merge(layer.ctx, qb, kb, vb, state, merged, merged_lse)
    layer.add_weights(queries, merged_lse)            # (shares of the whole softmax, the block's own keys in it)
    place = layer.kv_len.clone()
    layer.finalize_block(kb, vb)
    last = torch.arange(block, device="cuda")
    for s in range(N):                                # a finalised block begins without any weight
        at = place[s].long() + last
        layer.kv_weights[table[s].long()[at // page], :, at % page] = 0.0

    # 3. tokens, one for each sequence at a time, over all that is left
    cu = torch.arange(N + 1, device="cuda").int()
    position = layer.kv_len.clone()                   # of the text; places in the cache fall behind when tokens leave
    kept = torch.empty(N, hkv, budget, dtype=torch.int32, device="cuda")
    decoded = torch.empty(decode, N, hq, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(N, hq, device="cuda")
    for i in range(decode):
        layer.evict(B.make_eviction(layer.kv_len.clone(), torch.full_like(position, budget), kept, sinks=sinks, recent=64))
        q, k, v = project(N)
        start, rotated = layer.kv_len.clone(), torch.empty(N, hq, d, dtype=torch.bfloat16, device="cuda")
        layer.append(B.make_new_tokens(q, k, v, cu, start, pos=position + i, q_out=rotated), rope)
        queries = B.make_queries(rotated, cu, start, 1)
        layer.attend(queries, decoded[i], lse)
        layer.add_weights(queries, lse)
    status = layer.ctx.poll_status()
    if status != B.LOSA_OK:
        raise B.LosaError("example", status)
    return out, merged, decoded, layer.kv_len.tolist()


if __name__ == "__main__":
    out, merged, decoded, left = run()
    print("prompts", tuple(out.shape), "block", tuple(merged.shape), "decoded", tuple(decoded.shape), "tokens left", left)
