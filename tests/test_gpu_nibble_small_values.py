"""Decode attention over 4-bit values that are small: the error goes with the values, whatever their size, the length of a chunk or the spread of the logits."""
import math

import pytest
import torch

from tests import cache_oracle as want
from tests import close_bounds as close
from tests import test_gpu_nibble as nibble

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rows_of(pool, table, n, head, which):
    """Values [n, 128] in 64 bits of a sequence's rows, and the largest scale of each."""
    pages = table[:-(-n // pool.page)].long()
    codes = pool.codes[which].cpu()[pages, head].reshape(-1, 64)[:n]
    scales = pool.scales[which].cpu()[pages, head].flatten(0, 1)[:n]
    return want.nibble_values(codes, scales, which), scales[:, 0].double().amax(-1)


def check_close(got, pool, table, lens, q, scale):
    share = q.shape[1] // pool.hkv
    for b, n in enumerate(lens):
        for h in range(pool.hkv):
            (k, sk), (v, sv) = (rows_of(pool, table[b], n, h, i) for i in (0, 1))
            qh = q[b, h * share:(h + 1) * share].cpu().double()
            exp, tol = close.nibble(pool.dtype, qh, k, v, sk, sv, scale)
            off = (got[b, h * share:(h + 1) * share].cpu().double() - exp).abs()
            assert (off <= tol).all(), "sequence %d (%d keys), KV head %d: %.3g of the bound, %.2g of the largest output" % (
                b, n, h, float((off / tol).max()), float(off.max() / exp.abs().max()))


@pytest.mark.parametrize("dtype", nibble.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("size", [1.0, 1e-2, 1e-3, 1e-4])
@pytest.mark.parametrize("chunk", [256, 4096, 16384])
@pytest.mark.parametrize("first", [0.0, 12.0], ids=["wide", "first_key"])
def test_small_values(dtype, size, chunk, first):
    """Logits of a standard deviation of 3, or a first key about 12 above the others."""
    lens, page, max_seq, scale = [16384, 4100], 64, 16384, 1 / math.sqrt(128)
    pool, table = nibble.filled(dtype, 32, 2, 1, page, lens, 5, max_seq // page)
    pool.scales[1] *= size
    g = torch.Generator().manual_seed(1)
    if first:
        q = 0.3 * torch.randn(2, 4, 128, generator=g)
        for b, n in enumerate(lens):
            k0 = rows_of(pool, table[b], 1, 0, 0)[0][0].float()
            q[b] += k0 * (first / scale / k0.square().sum())
    else:
        q = 2.0 * torch.randn(2, 4, 128, generator=g)
    q = q.to(dtype).to(DEV)
    got = nibble.attend(pool, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), q, chunk, max_seq, scale)
    torch.cuda.synchronize()
    check_close(got, pool, table, lens, q, scale)


@pytest.mark.parametrize("dtype", nibble.TYPES, ids=["fp16", "bf16"])
def test_small_and_large_groups_of_a_row(dtype):
    """A group of values a thousand times another's: each is as exact as alone."""
    lens, page, max_seq, scale = [5000], 64, 5056, 0.2
    pool, table = nibble.filled(dtype, 32, 1, 2, page, lens, 6, max_seq // page)
    factor = torch.tensor([1.0, 1e-3, 30.0, 0.1], dtype=dtype, device=DEV)
    pool.scales[1] *= factor
    q = torch.randn(1, 12, 128, generator=torch.Generator().manual_seed(2)).to(dtype).to(DEV)
    got = nibble.attend(pool, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), q, 8192, max_seq, scale)
    torch.cuda.synchronize()
    for h in range(2):
        k, sk = rows_of(pool, table[0], lens[0], h, 0)
        v = rows_of(pool, table[0], lens[0], h, 1)[0]
        pages = table[0, :-(-lens[0] // page)].long()
        scales = pool.scales[1].cpu()[pages, h].flatten(0, 1)[:lens[0], 0].double()
        for i in range(4):
            exp, tol = close.nibble(dtype, q[0, 6 * h:6 * h + 6].cpu().double(), k, v[:, 32 * i:32 * i + 32], sk, scales[:, i], scale)
            off = (got[0, 6 * h:6 * h + 6, 32 * i:32 * i + 32].cpu().double() - exp).abs()
            assert (off <= tol).all(), "head %d, group %d: %.3g of the bound" % (h, i, float((off / tol).max()))
