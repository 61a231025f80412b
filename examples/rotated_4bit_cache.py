"""The cache operators together, as an engine uses them: prompts into a 4-bit cache, a block denoised and appended, tokens decoded.

  python examples/rotated_4bit_cache.py

One attention layer with random inputs.  Queries and keys come unrotated, as projections give them:
  1. prompts of any length go into the cache rotated (`losa_rope_append`);
  2. a block is denoised by the method's steps on that cache, its queries and keys rotated to their positions, and finalised;
  3. single tokens are appended and attend to the whole cache (`losa_int4_attn`).
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_12056_b200 import binding as B  # noqa: E402
from paper_2604_12056_b200 import workloads as wl  # noqa: E402
from paper_2604_12056_b200.layer import LosaLayer  # noqa: E402


def rotation_table(n_pos, rot_dim, base=1e6, device="cuda"):
    angle = torch.arange(n_pos, device=device).double()[:, None] * base ** (-torch.arange(rot_dim // 2, device=device).double() / (rot_dim // 2))
    return B.make_rope(angle.cos().float(), angle.sin().float())


def run(prompts=(1000, 37, 4100), block=32, steps=4, decode=3, seed=0):
    """Outputs of the last denoising step [N, block, H_q, d] and of the decoded tokens [decode, N, 1, H_q, d]."""
    hq, hkv, d, page, N = 32, 8, 128, 32, len(prompts)
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def project(T):                                   # queries, keys and values of T tokens, side by side
        row = torch.randn(T, hq + 2 * hkv, d, generator=gen, device="cuda").bfloat16()
        return row[:, :hq], row[:, hq:hq + hkv], row[:, hq + hkv:]

    def ints(*v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    cfg = wl.Config("example", 9, hq, hkv, d, page, tuple(L + block + decode for L in prompts), block, steps, 16, 4, "bf16", False)
    pool = torch.zeros(N * cfg.max_pages_per_seq, hkv, page, d, dtype=torch.bfloat16, device="cuda")
    table = torch.randperm(pool.shape[0], generator=gen, device="cuda").view(N, -1).int()
    layer = LosaLayer(cfg, pool, pool, table, ints(*[0] * N), int4_kv=True)       # an empty cache
    del pool
    rope = rotation_table(max(prompts) + block + decode, d)

    # 1. prompts
    q, k, v = project(sum(prompts))
    cu = ints(0, *prompts).cumsum(0).int()
    rotated = torch.empty(q.shape, dtype=q.dtype, device="cuda")                # for the prompts' own attention
    layer.append(B.make_new_tokens(q, k, v, cu, ints(*[0] * N), q_out=rotated), rope)

    # 2. one block: the first step attends to everything, the others to the pages that four changed tokens select
    lens = layer.kv_len.clone()
    cu = torch.arange(N + 1, device="cuda").int() * block
    m = ints(*[4] * N)
    hidden = torch.randn(N * block, hq + 2 * hkv, d, generator=gen, device="cuda")
    for t in range(steps):
        changed = torch.rand(N * block, 1, 1, generator=gen, device="cuda") < 0.1
        hidden = torch.where(changed, torch.randn(hidden.shape, generator=gen, device="cuda"), hidden)
        row = hidden.bfloat16()
        qb, kb, vb = (torch.empty(N, block, h, d, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
        layer.rotate(B.make_new_tokens(row[:, :hq], row[:, hq:hq + hkv], None, cu, lens, q_out=qb, k_out=kb), rope)
        vb.copy_(row[:, hq + hkv:].view_as(vb))
        layer.run_step_fused(qb, kb, vb, m)
    layer.finalize_block(kb, vb)

    # 3. tokens, one for each sequence at a time
    single = B.Context(N, hq, hkv, d, 1, page, cfg.max_pages_per_seq, B.LOSA_BF16, cfg.sm_scale)
    out = torch.empty(decode, N, 1, hq, d, dtype=torch.bfloat16, device="cuda")
    for i in range(decode):
        q, k, v = project(N)
        rotated = torch.empty(N, 1, hq, d, dtype=torch.bfloat16, device="cuda")
        start = layer.kv_len.clone()
        B.losa_rope_append(single, layer.kv, rope, B.make_new_tokens(q, k, v, torch.arange(N + 1, device="cuda").int(), start, q_out=rotated.view(N, hq, d)))
        B.losa_int4_attn(single, rotated, layer.kv, out[i])
    for ctx in (layer.ctx, single):
        status = ctx.poll_status()
        if status != B.LOSA_OK:
            raise B.LosaError("example", status)
    assert layer.kv_len.tolist() == [L + block + decode for L in prompts]
    return layer.out, out


if __name__ == "__main__":
    block_out, decoded = run()
    print("denoised block", tuple(block_out.shape), "decoded tokens", tuple(decoded.shape), "largest value", float(decoded.abs().max()))
