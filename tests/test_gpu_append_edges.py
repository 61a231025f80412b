"""losa_rope_append and what goes with it where contexts, pointers or numbers are out of the ordinary (needs a B200)."""
import pytest
import torch

import cache_ops_ref as ref
from test_gpu_rope_append import KINDS, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kv,dtype", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_contexts_of_different_batches_in_turn(kv, dtype, d):
    """Contexts of 64, 2, 1000 and 1 sequences append, twice in turn: what one of them sets up must not refuse another's call."""
    cases = [Case([1 + i % 2 for i in range(n)], [i % 40 for i in range(n)], kv=kv, dtype=dtype, d=d, hq=1, hkv=1, seed=n) for n in (64, 2, 1000, 1)]
    for _ in range(2):
        for c in cases:
            assert c.run() == 0
    for c in cases[:2]:
        for t, old in zip((c.kp, c.vp, c.ks, c.vs, c.kmin, c.kmax), c.before):
            if t is not None:
                t.copy_(old)
        assert c.run() == 0
        c.check()
