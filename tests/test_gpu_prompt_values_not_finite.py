"""Infinite and NaN values reach the outputs of their own token and of those behind it, in their own element, and nothing else."""
import pytest
import torch

from tests import test_gpu_latent as latent

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype", latent.TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("max_seq", [224, 420])               # a walk in one piece, and in two halves
@pytest.mark.parametrize("where", [
    [(40, 3, INF)], [(63, 127, NAN)], [(64, 16, -INF), (70, 16, INF)], [(0, 5, NAN)], [(31, 0, INF), (32, 0, INF), (95, 64, NAN)],
    [(k, (7 * k) % 128, (INF, -INF, NAN)[k % 3]) for k in range(128, 160)], [(130, d, -INF) for d in range(128)], [(219, 9, NAN), (218, 9, INF)],
    [(129, 1, INF), (140, 1, NAN), (150, 1, -INF), (141, 2, -INF), (157, 2, INF)]], ids=lambda w: "%d-%d" % (w[0][0], len(w)))
def test_values_that_are_not_finite(dtype, max_seq, where):
    n, heads = max_seq - 4, 2
    q, kv, rope = latent.prompt(dtype, [n], heads, max_seq, 64, 9)
    lens = torch.tensor([n], dtype=torch.int32, device=DEV)
    clean = latent.prefill(q, kv, rope, lens, 0.07)
    for t, d, x in where:
        kv[0, t, 0, 128 + d] = x
    got = latent.prefill(q, kv, rope, lens, 0.07)
    torch.cuda.synchronize()
    exp = clean[0].cpu().clone()
    for t, d, x in where:                                       # inf and -inf add up to NaN, as do NaN and anything
        exp[t:n, 0, d] = torch.where(exp[t:n, 0, d].isinf(), exp[t:n, 0, d] + x, torch.where(exp[t:n, 0, d].isnan(), exp[t:n, 0, d], x))
    x = got[0].cpu()
    changed = torch.zeros(128, dtype=torch.bool)
    changed[[d for _, d, _ in where]] = True
    assert torch.equal(x[:, 1], exp[:, 1]) and torch.equal(x[:, 0, ~changed], exp[:, 0, ~changed])
    # (of a changed element the finite outputs in front of it are as they were)
    assert torch.equal(x.isnan(), exp.isnan()) and torch.equal(x.nan_to_num(0.0, 1e4, -1e4), exp.nan_to_num(0.0, 1e4, -1e4))
