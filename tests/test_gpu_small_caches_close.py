"""The attention calls of the smaller caches on ordinary values, within bounds near what their arithmetic loses (a hundredth of the outputs and less)."""
import math

import pytest
import torch

from tests import close_bounds as close
from tests import test_gpu_latent as latent
from tests import test_gpu_nibble as nibble
from tests import test_gpu_nibble_small_values as values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", nibble.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("hq,hkv,chunk", [(1, 1, 64), (4, 4, 256), (8, 2, 1024), (6, 1, 4096), (9, 1, 128), (16, 1, 512), (24, 1, 4096), (40, 1, 320)])
def test_nibble(dtype, group, hq, hkv, chunk):
    lens, page, max_seq, scale = [1, 200, 77, 1024, 2500], 16, 2512, 1 / math.sqrt(128)
    pool, table = nibble.filled(dtype, group, len(lens), hkv, page, lens, hq + group, max_seq // page)
    q = torch.randn(len(lens), hq, 128, generator=torch.Generator().manual_seed(hq)).to(dtype).to(DEV)
    got = nibble.attend(pool, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), q, chunk, max_seq, scale)
    torch.cuda.synchronize()
    values.check_close(got, pool, table, lens, q, scale)


@pytest.mark.parametrize("dtype", latent.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("heads,chunk", [(1, 64), (16, 1024), (17, 256), (32, 4096), (40, 128), (64, 512), (65, 64), (130, 1024), (128, 4096)])
@pytest.mark.parametrize("size", [1.0, 6.0])
def test_latent_decode(dtype, heads, chunk, size):
    lens, page, max_seq, scale = [1, 200, 77, 1500], 64, 1536, 1 / math.sqrt(192)
    rows, table = latent.filled(dtype, lens, page, max_seq // page, heads)
    ql, qr = latent.queries(heads, len(lens), heads, dtype, size)
    got = latent.decode(rows.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), ql, qr, chunk, max_seq, scale)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        k = latent.want.gather(rows, table[b], n, page).double()
        exp, tol = close.latent(dtype, 2 if heads <= 64 else 1, torch.cat([ql[b], qr[b]], -1).cpu().double(), k, k[:, :512], scale)
        off = (got[b].cpu().double() - exp).abs()
        assert (off <= tol).all(), "sequence %d: %.3g of the bound" % (b, float((off / tol).max()))


@pytest.mark.parametrize("dtype", latent.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("lens,heads,max_seq", [([1, 33, 129], 3, 129), ([300, 511], 2, 600), ([400, 333], 70, 400), ([1500], 4, 1500)])
@pytest.mark.parametrize("size", [1.0, 8.0])
def test_prompts(dtype, lens, heads, max_seq, size):
    q, kv, rope = latent.prompt(dtype, lens, heads, max_seq, 64, 3, size)
    scale = 1 / math.sqrt(192)
    got = latent.prefill(q, kv, rope, torch.tensor(lens, dtype=torch.int32, device=DEV), scale)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        below = torch.ones(n, n, dtype=torch.bool).tril()
        for h in {0, heads // 2, heads - 1}:
            x = kv[b, :n, h].cpu().double()
            exp, tol = close.latent(dtype, 1, q[b, :n, h].cpu().double(), torch.cat([x[:, :128], rope[b, :n].cpu().double()], -1), x[:, 128:], scale, below)
            off = (got[b, :n, h].cpu().double() - exp).abs()
            assert (off <= tol).all(), "sequence %d, head %d: %.3g of the bound" % (b, h, float((off / tol).max()))
