"""Latent decode whose first keys, or whole chunks, all have logits of -inf: the softmax is over the others."""
import pytest
import torch

from tests import close_bounds as close
from tests import test_gpu_latent as latent

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", latent.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("heads", [3, 20, 40, 70])
@pytest.mark.parametrize("hidden", [(0, 32), (0, 100), (64, 200), (0, 300)], ids=lambda x: "%d-%d" % x)
@pytest.mark.parametrize("chunk", [64, 256, 512])
def test_masked_starts(dtype, heads, hidden, chunk):
    """Keys with an infinite rotary element, of the sign that makes every logit of theirs -inf; the others' logits lie near -170."""
    n, page, max_seq, scale = 300, 16, 320, 0.07
    rows, table = latent.filled(dtype, [n], page, max_seq // page, heads)
    at = (table[0, :-(-n // page)].long()[:, None] * page + torch.arange(page)).flatten()[:n]
    flat = rows.view(-1, 576)
    flat[at, 512], flat[at, 513] = 0, -30
    k = flat[at].double()
    flat[at[hidden[0]:hidden[1]], 512] = float("inf")
    ql, qr = latent.queries(heads, 1, heads, dtype)
    qr[..., 0], qr[..., 1] = -qr[..., 0].abs() - 0.1, 80
    got = latent.decode(rows.to(DEV), table.to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV), ql, qr, chunk, max_seq, scale)
    torch.cuda.synchronize()
    out = got[0].cpu().double()
    if hidden == (0, n):
        assert out.isnan().all()                                # of -inf alone the softmax is none
        return
    seen = torch.ones(heads, n, dtype=torch.bool)
    seen[:, hidden[0]:hidden[1]] = False
    exp, tol = close.latent(dtype, 2 if heads <= 64 else 1, torch.cat([ql, qr], -1)[0].cpu().double(), k, k[:, :512], scale, seen)
    off = (out - exp).abs()
    assert (off <= tol).all(), "%.3g of the bound" % float((off / tol).max())
