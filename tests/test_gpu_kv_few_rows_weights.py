"""Attention of packed new tokens: in sequences of up to 16 rows a KV head the weights enter the second product as two numbers of the type, so that their
outputs are as near 64 bits as decode's.  (That the bound tells two numbers from one: tests/test_kv_bounds_host.py.)"""
import math

import pytest
import torch

from tests.kv_pool import DEV, TYPES, check, filled, prefill
from tests.test_gpu_kv_prefill import device, fused, mask

pytestmark = pytest.mark.gpu
TYPED = pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
BOTH = pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])


@TYPED
@BOTH
@pytest.mark.parametrize("scale", [1 / math.sqrt(128), 0.02])
@pytest.mark.parametrize("hq,hkv,chunk,new", [
    (1, 1, 4096, [1, 16, 7, 15]), (4, 1, 4096, [4, 1, 3, 2]), (16, 1, 4096, [1, 1, 1, 1]), (15, 3, 64, [3, 2, 1, 3]), (32, 8, 300, [1, 4, 2, 1]),
    (16, 2, 1, [2, 1, 1, 2]),
])
def test_two_numbers_a_weight(dtype, coded, scale, hq, hkv, chunk, new):
    lens, width, share = [700, 1500, 129, 64], 48, hq // hkv
    pool, table, k, v = filled(dtype, coded, hkv, 32, lens, 73, width)
    new, lens = new + [150], lens + [150]                       # ... beside a prompt without keys
    table = torch.cat([table, table[:1]])
    lens[4] = 0
    q = fused(sum(new), hq, dtype, seed=7)
    dtable, dlens, starts = device(lens, table, new)
    got = prefill(pool, dtable, dlens, starts, q, chunk, width * 32, scale).cpu()
    q, row = q.cpu(), 0
    for b, n in enumerate(new[:4]):
        assert n * share <= 16
        for h in range(hq):
            check(got[row:row + n, h], dtype, 2, q[row:row + n, h], k[b][h // share], v[b][h // share], scale, mask(lens[b], n),
                  "sequence %d, head %d" % (b, h))
        row += n
    assert (got[row:] == 0).all()
