"""Attention of packed new tokens whose sequences have up to 16 rows a KV head (single tokens, short pieces), with numbers in the last block of keys that are
not finite: the rows that see them get them, the others do not."""
import math

import pytest
import torch

from tests.kv_pool import DEV, TYPES, check, decode, filled, prefill
from tests.test_gpu_kv_prefill import device, fused, mask

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)
TYPED = pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
BOTH = pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])
HEADS = pytest.mark.parametrize("hq,hkv", [(4, 1), (5, 5), (8, 2)])
LENS, NEW = [20, 100, 300, 1, 33, 129, 2], [1, 3, 3, 1, 2, 1, 2]
PLACES = {"last": 1, "last but one": 2}                         # the key, from the end of its sequence
WIDTH = 20


def place(b, back):
    return max(LENS[b] - back, 0)


@TYPED
@HEADS
@pytest.mark.parametrize("back", PLACES.values(), ids=PLACES)
@pytest.mark.parametrize("chunk", [1, 64, 4096])
def test_infinite_values(dtype, hq, hkv, back, chunk):
    """inf in element 5, -inf in element 70, both and NaN in the next ones of one key's value of every sequence."""
    inf = float("inf")
    special = {5: inf, 70: -inf, 71: float("nan")}

    def change(b, which, x):
        if which:
            for d, value in special.items():
                x[:, place(b, back), d] = value
        return x
    pool, table, k, v = filled(dtype, False, hkv, 16, LENS, 61, WIDTH, 1.0, change)
    q = fused(sum(NEW) + 1, hq, dtype, seed=3)
    table, dlens, starts = device(LENS, table, NEW)
    got = prefill(pool, table, dlens, starts, q, chunk, WIDTH * 16, SCALE).cpu()
    last = q[starts[1:].long() - 1].contiguous()
    one = decode(pool, table, dlens, last, 64, WIDTH * 16, SCALE).cpu()
    q, row, share = q.cpu(), 0, hq // hkv
    plain = [d for d in range(128) if d not in special]
    for b, (L, n) in enumerate(zip(LENS, NEW)):
        sees = mask(L, n)
        hit = sees[:, place(b, back)]
        assert hit[-1]
        part = got[row:row + n]
        assert part[~hit].isfinite().all() and part[..., plain].isfinite().all()
        for x in (part[hit], one[b:b + 1]):
            assert (x[..., 5] == inf).all() and (x[..., 70] == -inf).all() and x[..., 71].isnan().all(), "sequence %d" % b
        for h in range(hq):
            clean = v[b][h // share].clone()
            clean[place(b, back)][list(special)] = 0.0
            check(part[:, h][:, plain], dtype, 1, q[row:row + n, h], k[b][h // share], clean[:, plain], SCALE, sees, "sequence %d, head %d" % (b, h))
        row += n
    assert (got[row:] == 7.0).all()


@TYPED
@BOTH
@HEADS
@pytest.mark.parametrize("which", [0, 1], ids=["keys", "values"])
@pytest.mark.parametrize("chunk", [1, 4096])
def test_nan(dtype, coded, hq, hkv, which, chunk):
    """A NaN in a key, or a value row of NaN, of the last but one key: rows in front of it are as if it were not there."""
    def change(b, of, x):
        if of == which:
            x[:, place(b, 2)] = float("nan")
        return x
    pool, table, k, v = filled(dtype, coded, hkv, 16, LENS, 67, WIDTH, 1.0, change)
    q = fused(sum(NEW), hq, dtype, seed=4)
    table, dlens, starts = device(LENS, table, NEW)
    got = prefill(pool, table, dlens, starts, q, chunk, WIDTH * 16, SCALE).cpu()
    q, row, share = q.cpu(), 0, hq // hkv
    for b, (L, n) in enumerate(zip(LENS, NEW)):
        sees = mask(L, n)
        hit = sees[:, place(b, 2)]
        part = got[row:row + n]
        assert part[hit].isnan().all()
        for h in range(hq):
            rows = [x[b][h // share].nan_to_num(0.0) for x in (k, v)]
            check(part[~hit, h], dtype, 1, q[row:row + n, h][~hit], *rows, SCALE, sees[~hit], "sequence %d, head %d" % (b, h))
        row += n


@TYPED
def test_infinite_values_of_both_signs_and_of_masked_keys(dtype):
    """Both signs of infinity in one element are NaN; of 16 rows each sees one more infinite key than the row before."""
    L, n, inf = 50, 16, float("inf")

    def change(b, which, x):
        if which:
            for i in range(n):
                x[0, L - n + i, i] = inf if i % 2 else -inf
            x[0, L - 3, 100], x[0, L - 2, 100] = inf, -inf
        return x
    pool, table, _, _ = filled(dtype, False, 1, 16, [L], 71, 4, 1.0, change)
    q = fused(n, 1, dtype, seed=5)
    table, dlens, starts = device([L], table, [n])
    got = prefill(pool, table, dlens, starts, q, 64, 64, SCALE).cpu()[:, 0].double()
    for i in range(n):
        exp = torch.tensor([inf if j % 2 else -inf for j in range(i + 1)], dtype=torch.float64)
        assert torch.equal(got[i, :i + 1], exp) and got[i, i + 1:100].isfinite().all() and got[i, 101:].isfinite().all()
        assert got[i, 100].isfinite() if i < n - 3 else got[i, 100] == inf if i == n - 3 else got[i, 100].isnan()
