"""A seeded random sweep over the attention calls of the paged cache of 16 or 8 bits: types, heads, pages, lengths, pieces."""
import random

import pytest
import torch

from tests.kv_pool import DEV, TYPES, check, decode, filled, prefill
from tests.test_gpu_kv_prefill import check_all, device, fused

pytestmark = pytest.mark.gpu
SCALE = 0.09


@pytest.mark.parametrize("seed", range(48))
def test_sweep(seed):
    r = random.Random(seed)
    dtype, coded = r.choice(TYPES), r.random() < 0.5
    hkv, share = r.choice([(1, 1), (1, 7), (1, 33), (2, 1), (2, 4), (3, 5), (4, 4), (8, 1), (8, 8), (17, 1), (17, 3)])
    hq, page = hkv * share, r.choice([16, 32, 64, 256])
    batch = r.choice([1, 2, 3, 5, 9, 40, 63, 64, 65, 70])
    longest = r.choice([5, 40, 130, 400]) if batch < 20 else r.choice([2, 6, 40])
    new = [r.choice([0, 1, 1, 2, r.randint(1, longest)]) for _ in range(batch)]
    new[0] = max(new[0], 1)
    cached = r.choice([0, 3, 60, 600, 3001 if batch < 10 else 100])
    # (some have fewer keys than new tokens, some none)
    lens = [max(0, n + r.randint(-3 if r.random() < 0.1 else 0, cached)) if n or r.random() < 0.8 else 0 for n in new]
    width = max(1, -(-max(lens) // page) + r.randint(0, 2))
    max_seq = width * page
    pool, table, k, v = filled(dtype, coded, hkv, page, lens, seed, width)
    heads = sorted({0, hq // 2, hq - 1})

    q = fused(sum(new) + 2, hq, dtype, seed=seed)
    table, dlens, starts = device(lens, table, new)
    chunk = r.choice([0, 0, 1, 2, 7, 64, 100, 500, max_seq, max_seq + 5])
    check_all(prefill(pool, table, dlens, starts, q, chunk, max_seq, SCALE), pool, lens, new, q, k, v, SCALE, heads=heads)

    q = fused(batch, hq, dtype, seed=seed + 1, extra=0).contiguous()
    got, q_cpu = decode(pool, table, dlens, q, r.choice([0, 64, 128, 512, 1024]), max_seq, SCALE).cpu(), q.cpu()
    for b, n in enumerate(lens):
        assert n or (got[b] == 0).all()
        for h in heads if n else ():
            check(got[b:b + 1, h], dtype, 2, q_cpu[b:b + 1, h], k[b][h // share], v[b][h // share], SCALE, what="sequence %d, head %d" % (b, h))
