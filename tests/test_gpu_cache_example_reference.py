"""The example that runs the cache operators together, against the plain 64-bit form of what it computes (needs a B200).

The example keeps its tensors to itself, so the library's calls are watched: what goes in, unrotated, is rotated, coded and attended to
again on the CPU, from the calls' inputs alone."""
import importlib.util
import os

import pytest
import torch

import cache_ops_ref as ref

pytestmark = pytest.mark.gpu


def test_decoded_tokens_are_those_of_the_rotated_and_coded_tokens_before_them(monkeypatch):
    from paper_2604_12056_b200 import binding as B
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rotated_4bit_cache.py")
    spec = importlib.util.spec_from_file_location("rotated_4bit_cache", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    appended, finals, blocks = [], [], []
    append, update, rotate_only = B.losa_rope_append, B.losa_update_prefix_cache, []

    def watch_append(ctx, kv, rope, tokens):
        append(ctx, kv, rope, tokens)
        q, k, v, cu, start = tokens._keep[:5]
        (appended if kv is not None else rotate_only).append([None if t is None else t.cpu().clone() for t in (q, k, v, cu, start)])

    def watch_update(ctx, kv, state, q, k_blk, v_blk, finalize):
        if finalize:
            finals.append([k_blk.cpu().clone(), v_blk.cpu().clone()])
        update(ctx, kv, state, q, k_blk, v_blk, finalize)

    monkeypatch.setattr(B, "losa_rope_append", watch_append)
    monkeypatch.setattr(B, "losa_update_prefix_cache", watch_update)
    prompts, block, decode, d, hq, hkv = (70, 3, 300), 32, 2, 128, 32, 8
    block_out, decoded = example.run(prompts=prompts, block=block, steps=3, decode=decode)
    assert len(appended) == 1 + decode and len(finals) == 1 and len(rotate_only) == 3
    n_pos = max(prompts) + block + decode
    angle = torch.arange(n_pos).double()[:, None] * 1e6 ** (-torch.arange(d // 2).double() / (d // 2))
    turned = lambda x, pos: ref.rotate(x.double(), angle.cos(), angle.sin(), pos, d, False)[0].bfloat16().double()
    code = lambda x: ref.int4_value(*ref.int4_encode(x))

    # the last step's keys were rotated to the block's positions before they were finalised
    q3, k3, _, cu3, start3 = rotate_only[-1]
    for s, L in enumerate(prompts):
        want = turned(k3[s * block:(s + 1) * block], torch.arange(L, L + block))
        assert int(start3[s]) == L and (finals[0][0][s].double() - want).abs().max() <= 2.0 ** -7 * want.abs().max()

    q0, k0, v0, cu, _ = appended[0]
    for s, L in enumerate(prompts):
        at = slice(int(cu[s]), int(cu[s + 1]))
        keys = [turned(k0[at], torch.arange(L)), finals[0][0][s].double()]
        values = [v0[at].double(), finals[0][1][s].double()]
        for i in range(decode):
            q, k, v = (t[s:s + 1] for t in appended[1 + i][:3])
            pos = torch.tensor([L + block + i])
            keys.append(turned(k, pos))
            values.append(v.double())
            kk, vv, qq = code(torch.cat(keys)), code(torch.cat(values)), turned(q, pos)[0]
            for h in range(hkv):
                rows = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                o, _, do, _ = ref.attention(qq[rows], kk[:, h], vv[:, h], d ** -0.5)
                got = decoded[i, s, 0, rows].cpu().double()
                # Rotated elements of queries and keys here are rounded from float64, in the library from fp32: where the two fall on either side of a
                # tie, an element is one unit of bf16 (2^-8 of it) off, and a key's code then at most one step, a seventh of its run's largest.
                # A wrong position or a wrong pair changes all of a score, of size one; one in some thousand elements
                # off by a seventh moves a score by less than 2 % of its size, and an output by as much of the values' size, about one.
                assert ((got - o).abs() <= do + 2.0 ** -8 * o.abs() + 0.02).all(), float((got - o).abs().max())
                assert float((got - o).square().mean().sqrt()) <= 2.0 ** -8
