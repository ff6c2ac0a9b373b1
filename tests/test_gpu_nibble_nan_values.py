"""Value rows of the 4-bit cache with an infinite element or a NaN: their group reads as NaN, and so do that group's elements of every output over them; nothing else changes."""
import math

import pytest
import torch

from tests import test_gpu_nibble as nibble

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", nibble.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("element", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("chunk", [64, 4096])
def test_written_rows(dtype, group, element, chunk):
    tokens, hkv, hq, page = 300, 2, 10, 16
    g = torch.Generator().manual_seed(group)
    x = torch.randn(tokens, 2 * hkv, 128, generator=g).to(dtype)
    q = torch.randn(1, hq, 128, generator=g).to(dtype).to(DEV)
    table = torch.randperm(20, generator=g).to(torch.int32)[None, :19].contiguous()
    slots = (table[0].long()[:, None] * page + torch.arange(page)).flatten()[:tokens].to(torch.int32).to(DEV)
    lens = torch.tensor([tokens], dtype=torch.int32, device=DEV)
    outs = []
    for bad in (False, True):
        pool = nibble.Pool(20, page, hkv, group, dtype)
        if bad:
            x[123, hkv + 1, 70] = element                          # of V, head 1
        nibble.write(pool, x.to(DEV), 0, slots)
        outs.append(nibble.attend(pool, table.to(DEV), lens, q, chunk, 19 * page, 1 / math.sqrt(128)))
        torch.cuda.synchronize()
    clean, got = outs
    first = 70 // group * group
    assert torch.equal(got[0, :5], clean[0, :5])
    assert got[0, 5:, first:first + group].isnan().all()
    for part in (slice(0, first), slice(first + group, 128)):
        assert torch.equal(got[0, 5:, part], clean[0, 5:, part])


@pytest.mark.parametrize("dtype", nibble.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("bits", [0x7fff, 0xffff, 0x7fc1, 0xff81], ids=hex)
@pytest.mark.parametrize("which", [0, 1], ids=["scale", "lowest"])
def test_any_nan(dtype, bits, which):
    lens, page, max_seq = [200], 16, 208
    pool, table = nibble.filled(dtype, 32, 1, 1, page, lens, 4, max_seq // page)
    q = torch.randn(1, 4, 128, generator=torch.Generator().manual_seed(5)).to(dtype).to(DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    clean = nibble.attend(pool, table.to(DEV), dl, q, 64, max_seq, 0.1)
    value = torch.tensor([bits - (bits >> 15 << 16)], dtype=torch.int16).view(dtype)
    assert value.isnan().all()
    pool.scales[1][int(table[0, 7]), 0, 5, which, 2] = value.to(DEV)[0]
    assert int(pool.scales[1][int(table[0, 7]), 0, 5, which, 2].view(torch.int16)) & 0xffff == bits
    got = nibble.attend(pool, table.to(DEV), dl, q, 64, max_seq, 0.1)
    torch.cuda.synchronize()
    assert got[0, :, 64:96].isnan().all()
    assert torch.equal(got[0, :, :64], clean[0, :, :64]) and torch.equal(got[0, :, 96:], clean[0, :, 96:])
    assert torch.isfinite(clean[0]).all()
