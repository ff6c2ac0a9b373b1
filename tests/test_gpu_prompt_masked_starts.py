"""Prompts whose queries find only logits of -inf among their first keys: the softmax is over the others."""
import pytest
import torch

from tests import close_bounds as close
from tests import test_gpu_latent as latent

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", latent.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("hidden", [(0, 32), (32, 64), (0, 64), (0, 100), (37, 200)], ids=lambda x: "%d-%d" % x)
@pytest.mark.parametrize("max_seq", [224, 420])               # a walk in one piece, and in two halves
def test_masked_starts(dtype, hidden, max_seq):
    """Keys with an infinite element, of the sign that makes every logit of theirs -inf; the others' logits lie near -170, far below where e^x ends."""
    n, heads, scale = max_seq - 5, 3, 0.07
    q, kv, rope = latent.prompt(dtype, [n], heads, max_seq, 64, 4)
    q[0, :n, :, 0] = -q[0, :n, :, 0].abs() - 0.1
    kv[0, :n, :, 0] = 0
    kv[0, hidden[0]:hidden[1], :, 0] = float("inf")
    q[0, :n, :, 1], kv[0, :n, :, 1] = 80, -30
    got = latent.prefill(q, kv, rope, torch.tensor([n], dtype=torch.int32, device=DEV), scale)
    torch.cuda.synchronize()
    below = torch.ones(n, n, dtype=torch.bool).tril()
    seen = below.clone()
    seen[:, hidden[0]:hidden[1]] = False
    some = seen.any(1)
    for h in range(heads):
        x = kv[0, :n, h].cpu().double()
        x[hidden[0]:hidden[1], 0] = 0                           # (what they are worth is in `seen`)
        k = torch.cat([x[:, :128], rope[0, :n].cpu().double()], -1)
        exp, tol = close.latent(dtype, 1, q[0, :n, h].cpu().double()[some], k, x[:, 128:], scale, seen[some])
        out = got[0, :n, h].cpu().double()
        off = (out[some] - exp).abs()
        assert (off <= tol).all(), "head %d: %.3g of the bound" % (h, float((off / tol).max()))
        assert out[~some].isnan().all()                         # of -inf alone the softmax is none
