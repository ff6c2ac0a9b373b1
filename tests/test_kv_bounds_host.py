"""What the bound of the attention tests over the paged cache of 16 or 8 bits tells apart: weights as two numbers of the type from weights as one."""
import pytest
import torch

from tests.kv_pool import TYPES, check


def attention(q, k, v, scale, dtype, parts):
    """In 64 bits but for the weights, the sum of `parts` numbers of the type; the denominator is that of the unrounded ones, the output of the type."""
    x = scale * (q.double() @ k.t())
    p = torch.exp(x - x.amax(-1, keepdim=True))
    w = torch.zeros_like(p)
    for _ in range(parts):
        w += (p - w).to(dtype).double()
    return ((w @ v) / p.sum(-1, keepdim=True)).to(dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("scale", [128 ** -0.5, 0.02])
@pytest.mark.parametrize("keys", [129, 700, 1500])
def test_one_number_a_weight_is_outside(dtype, scale, keys):
    g = torch.Generator().manual_seed(keys)
    q, k, v = (torch.randn(n, 128, generator=g).to(dtype) for n in (1, keys, keys))
    k, v = k.double(), v.double()
    check(attention(q, k, v, scale, dtype, 2), dtype, 2, q, k, v, scale)
    with pytest.raises(AssertionError):
        check(attention(q, k, v, scale, dtype, 1), dtype, 2, q, k, v, scale)
