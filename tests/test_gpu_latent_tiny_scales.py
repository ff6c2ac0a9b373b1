"""Scales of nothing or almost nothing beside products near the end of fp32: the logits are the products times the scale, not something larger."""
import pytest
import torch

from tests import close_bounds as close
from tests import test_gpu_latent as latent

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SCALES = [0.0, -0.0, 2.0 ** -140, -2.0 ** -112, 2.0 ** -100]


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("heads", [3, 20, 40, 70])
def test_decode(scale, heads):
    lens, max_seq = [300, 1, 65], 320
    rows, table = latent.filled(torch.bfloat16, lens, 16, max_seq // 16, 13)
    rows = rows * 2.0 ** 40
    ql, qr = (x * 2.0 ** 66 for x in latent.queries(8, 3, heads, torch.bfloat16))          # products of deviation 24 x 2^106
    got = latent.decode(rows.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), ql, qr, 64, max_seq, scale)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        k = latent.want.gather(rows, table[b], n, 16).double()
        q = torch.cat([ql[b], qr[b]], -1).cpu().double()
        exp, tol = close.latent(torch.bfloat16, 2 if heads <= 64 else 1, q, k, k[:, :512], scale)
        off = (got[b].cpu().double() - exp).abs()
        assert (off <= tol).all(), "sequence %d: %.3g of the bound" % (b, float((off / tol).max()))


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("max_seq", [200, 320])
def test_prompts(scale, max_seq):
    lens = [max_seq - 30, 33]
    q, kv, rope = latent.prompt(torch.bfloat16, lens, 3, max_seq, 64, 5)
    q, kv, rope = q * 2.0 ** 66, kv * 2.0 ** 40, rope * 2.0 ** 40
    got = latent.prefill(q, kv, rope, torch.tensor(lens, dtype=torch.int32, device=DEV), scale)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        for h in range(3):
            x = kv[b, :n, h].cpu().double()
            exp, tol = close.latent(torch.bfloat16, 1, q[b, :n, h].cpu().double(), torch.cat([x[:, :128], rope[b, :n].cpu().double()], -1), x[:, 128:], scale,
                                    torch.ones(n, n, dtype=torch.bool).tril())
            off = (got[b, :n, h].cpu().double() - exp).abs()
            assert (off <= tol).all(), "sequence %d, head %d: %.3g of the bound" % (b, h, float((off / tol).max()))
