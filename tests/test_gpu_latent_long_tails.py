"""Latent attention with one key far above thousands of others, whose weights are small but many."""
import math

import pytest
import torch

from tests import close_bounds as close
from tests import test_gpu_latent as latent

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BELOW = 17.375                  # e^-17.375 = 2^-25.07: less than half of fp16's smallest number


@pytest.mark.parametrize("dtype", latent.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("heads", [4, 24, 48, 70])
@pytest.mark.parametrize("chunk", [4096, 16384])
@pytest.mark.parametrize("far", [-8.0, 1.0])                   # the others' values, beside 1 of the first key
def test_decode(dtype, heads, chunk, far):
    n, page = 16384, 64
    rows, table = latent.filled(dtype, [n], page, n // page, 3)
    flat = rows.view(-1, 576)
    at = (table[0].long()[:, None] * page + torch.arange(page)).flatten()
    flat[at, 512:] = 0
    flat[at, :512] = (far + 0.1 * torch.randn(n, 512, generator=torch.Generator().manual_seed(1))).to(dtype)
    flat[at[0], :512] = (1 + 0.1 * torch.randn(512, generator=torch.Generator().manual_seed(2))).to(dtype)
    flat[at[0], 512] = BELOW
    ql, qr = torch.zeros(1, heads, 512, dtype=dtype), torch.zeros(1, heads, 64, dtype=dtype)
    qr[:, :, 0] = 1
    got = latent.decode(rows.to(DEV), table.to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV), ql.to(DEV), qr.to(DEV), chunk, n, 1.0)
    torch.cuda.synchronize()
    k = flat[at].double()
    exp, tol = close.latent(dtype, 2 if heads <= 64 else 1, torch.cat([ql, qr], -1)[0].double(), k, k[:, :512], 1.0)
    off = (got[0].cpu().double() - exp).abs()
    assert (off <= tol).all(), "%.3g of the bound" % float((off / tol).max())


@pytest.mark.parametrize("dtype", latent.TYPES, ids=["fp16", "bf16"])
def test_prompt(dtype):
    n = 4096
    q, kv, rope = (torch.zeros(1, n, *d, dtype=dtype) for d in ((1, 192), (1, 256), (64,)))
    q[..., 128] = 1
    rope[0, 0, 0] = BELOW
    kv[0, :, 0, 128:] = (-8 + 0.1 * torch.randn(n, 128, generator=torch.Generator().manual_seed(1))).to(dtype)
    kv[0, 0, 0, 128:] = 1
    got = latent.prefill(q.to(DEV), kv.to(DEV), rope.to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV), 1.0)
    torch.cuda.synchronize()
    k = torch.cat([kv[0, :, 0, :128], rope[0]], -1).double()
    last = [1000, 2047, 4000, 4095]
    exp, tol = close.latent(dtype, 1, q[0, last, 0].double(), k, kv[0, :, 0, 128:].double(), 1.0, torch.ones(n, n, dtype=torch.bool).tril()[last])
    off = (got[0, last, 0].cpu().double() - exp).abs()
    assert (off <= tol).all(), "%.3g of the bound" % float((off / tol).max())
