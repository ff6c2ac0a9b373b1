"""Attention of packed new tokens in a cut launch, beside sequences that have keys and no new token: of one key, a block, more than a piece."""
import pytest
import torch

from tests.kv_pool import TYPES, filled, prefill
from tests.test_gpu_kv_prefill import check_all, device, fused

pytestmark = pytest.mark.gpu
SCALE = 0.09


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])
@pytest.mark.parametrize("chunk", [1, 3, 64, 200])
@pytest.mark.parametrize("batch", [9, 70])
def test_sequences_without_new_tokens(dtype, coded, chunk, batch):
    lens, new = [1, 64, 300, 1, 129, 1, 65, 2, 257], [0, 0, 40, 1, 0, 0, 3, 0, 200]
    lens, new = lens + [1] * (batch - 9), new + [0] * (batch - 9)
    pool, table, k, v = filled(dtype, coded, 2, 16, lens, 79, 20)
    q = fused(sum(new) + 1, 4, dtype)
    table, dlens, starts = device(lens, table, new)
    check_all(prefill(pool, table, dlens, starts, q, chunk, 320, SCALE), pool, lens, new, q, k, v, SCALE)
