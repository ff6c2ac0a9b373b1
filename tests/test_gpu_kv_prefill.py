"""Attention of packed new tokens over the paged cache of 16 or 8 bits, against 64 bits."""
import math

import pytest
import torch

from tests import kv_oracle as want
from tests.kv_pool import DEV, TYPES, check, filled, lib, prefill, workspace

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)
BOTH = pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])
TYPED = pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])


def mask(L, n):
    """[n, L]: what each new token sees."""
    sees = torch.tensor([want.visible(L, n, i) for i in range(n)])
    return torch.arange(L)[None, :] < sees[:, None]


def starts_of(new):
    return torch.tensor([0] + torch.tensor(new).cumsum(0).tolist(), dtype=torch.int32)


def fused(tokens, hq, dtype, seed=1, size=1.0, extra=2):
    """Queries as the beginnings of a fused projection's rows."""
    x = (size * torch.randn(tokens, hq + extra, 128, generator=torch.Generator().manual_seed(seed))).to(dtype).to(DEV)
    return x[:, :hq]


def check_all(got, pool, lens, new, q, k, v, scale=SCALE, heads=None):
    share = q.shape[1] // pool.hkv
    got, q, at = got.cpu(), q.cpu(), 0
    for b, (L, n) in enumerate(zip(lens, new)):
        sees = mask(L, n)
        for h in range(q.shape[1]) if heads is None else heads:
            check(got[at:at + n, h], pool.dtype, 1, q[at:at + n, h], k[b][h // share], v[b][h // share], scale, sees, "sequence %d, head %d" % (b, h))
        at += n
    assert (got[at:] == 7.0).all()


def device(lens, table, new):
    return table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), starts_of(new).to(DEV)


@TYPED
@BOTH
@pytest.mark.parametrize("hq,hkv,page,chunk,lens,new", [
    (1, 1, 16, 4096, [1], [1]),
    (4, 4, 16, 4096, [40, 1, 129, 64], [40, 1, 129, 64]),
    (8, 2, 32, 4096, [300, 33, 500], [300, 2, 77]),
    (6, 1, 16, 64, [70, 900, 16, 333], [70, 5, 1, 200]),
    (14, 2, 128, 256, [1000, 640], [130, 640]),
    (40, 1, 64, 128, [200, 500], [31, 3]),
    (5, 5, 16, 0, [257, 0, 31, 1], [257, 0, 0, 1]),
])
def test_against_64_bits(dtype, coded, hq, hkv, page, chunk, lens, new):
    width = -(-max(lens) // page) + 1
    pool, table, k, v = filled(dtype, coded, hkv, page, lens, hq + page, width)
    tokens = sum(new) + 3                                               # three rows of no sequence
    q = fused(tokens, hq, dtype)
    table, dlens, starts = device(lens, table, new)
    got = prefill(pool, table, dlens, starts, q, chunk, width * page, SCALE)
    check_all(got, pool, lens, new, q, k, v)


@TYPED
@BOTH
@pytest.mark.parametrize("chunk", [64, 4096])
def test_every_length_around_a_block(dtype, coded, chunk):
    """Lengths and numbers of new tokens around 16, 32, 64 and 128, most pairs of them once."""
    edges = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129]
    lens = [edges[i % len(edges)] + (i // len(edges)) * 32 for i in range(42)]
    new = [min(edges[(5 * i + 3) % len(edges)], L) for i, L in enumerate(lens)]
    pool, table, k, v = filled(dtype, coded, 1, 16, lens, 5, 16)
    q = fused(sum(new), 3, dtype)
    table, dlens, starts = device(lens, table, new)
    check_all(prefill(pool, table, dlens, starts, q, chunk, 256, SCALE), pool, lens, new, q, k, v)


@TYPED
@BOTH
def test_more_new_tokens_than_keys_and_none(dtype, coded):
    """Positions below 0 have zero rows, also where a whole sequence has no key."""
    lens, new = [5, 0, 40, 100], [9, 70, 170, 0]
    pool, table, k, v = filled(dtype, coded, 2, 16, lens, 7, 7)
    q = fused(sum(new) + 1, 4, dtype)
    table, dlens, starts = device(lens, table, new)
    for chunk in (64, 128):
        check_all(prefill(pool, table, dlens, starts, q, chunk, 112, SCALE), pool, lens, new, q, k, v)


@TYPED
@BOTH
@pytest.mark.parametrize("scale,size", [(-0.2, 1.0), (0.0, 1.0), (1.0, 3.0), (1e-30, 1.0)])
def test_scales(dtype, coded, scale, size):
    lens, new = [333, 64], [200, 64]
    pool, table, k, v = filled(dtype, coded, 1, 32, lens, 9, 11, size)
    q = fused(sum(new), 2, dtype, size=size)
    table, dlens, starts = device(lens, table, new)
    for chunk in (128, 384):
        check_all(prefill(pool, table, dlens, starts, q, chunk, 352, scale), pool, lens, new, q, k, v, scale)


@TYPED
@BOTH
def test_first_keys_far_below_and_far_above(dtype, coded):
    lens, new, n = [2000, 2000, 2000], [40, 130, 70], 2000

    def change(b, which, x):
        if which == 0:
            x = x * 0.05
            x[:, n - 200 if b == 0 else 0] = 3.0 if b < 2 else -3.0
        return x
    pool, table, k, v = filled(dtype, coded, 1, 64, lens, 11, 32, 1.0, change)
    q = fused(sum(new), 2, dtype)
    q.copy_(torch.ones_like(q))
    table, dlens, starts = device(lens, table, new)
    for chunk in (512, 2048):
        check_all(prefill(pool, table, dlens, starts, q, chunk, 2048, 0.05), pool, lens, new, q, k, v, 0.05)


@TYPED
@BOTH
def test_values_that_are_not_finite(dtype, coded):
    """An infinite or NaN value of a later token does not reach those in front of it; nothing behind a sequence does."""
    lens, new, at = [300, 150], [180, 150], [220, 64]

    def change(b, which, x):
        if which:
            x[0, at[b], 5] = float("inf") if b == 0 else float("nan")
        return x
    pool, table, k, v = filled(dtype, coded, 1, 16, lens, 13, 19, 1.0, change)
    q = fused(sum(new), 2, dtype)
    table, dlens, starts = device(lens, table, new)
    for chunk in (64, 320):
        got = prefill(pool, table, dlens, starts, q, chunk, 304, SCALE).cpu()
        row = 0
        for b, (L, n) in enumerate(zip(lens, new)):
            sees = mask(L, n)
            hit = sees[:, at[b]]
            part, x = got[row:row + n], [y.clone() for y in (k[b][0], v[b][0])]
            other = [d for d in range(128) if d != 5]
            assert part[~hit].isfinite().all()
            if coded:
                assert part[hit].isnan().all()
            else:
                column = part[hit][..., 5]
                assert (column == float("inf")).all() if b == 0 else column.isnan().all()
                assert part[hit][..., other].isfinite().all()
            x[1][at[b]] = 0.0                                           # (not seen by the rows that are compared)
            for h in range(2):
                check(part[~hit, h], dtype, 1, q[row:row + n, h].cpu()[~hit], x[0], x[1], SCALE, sees[~hit])
            row += n


@TYPED
@BOTH
def test_keys_that_are_not_finite(dtype, coded):
    """A NaN in a key makes NaN of the tokens that see it and of no other; keys at minus infinity count as nothing."""
    lens, new = [200, 260], [200, 130]

    def change(b, which, x):
        if not which and b == 0:
            x[0, 75, 3] = float("nan")
        if not which and b == 1 and not coded:
            x[:, :129, 0] = float("-inf")
        return x
    pool, table, k, v = filled(dtype, coded, 1, 16, lens, 17, 17, 1.0, change)
    q = fused(sum(new), 2, dtype)
    q.copy_(q.abs())
    table, dlens, starts = device(lens, table, new)
    for chunk in (64, 320):
        got = prefill(pool, table, dlens, starts, q, chunk, 272, SCALE).cpu()
        assert got[75:200].isnan().all() and got[:75].isfinite().all()
        first = 0 if coded else 129
        sees = mask(260, 130)[:, first:]
        for h in range(2):
            rows = slice(200, 330)
            part = slice(0, 130) if coded else slice(130 - 131 + 1, 130)
            check(got[rows, h][part], dtype, 1, q[rows, h].cpu()[part], k[1][0][first:], v[1][0][first:], SCALE, sees[part])


@TYPED
@BOTH
def test_single_tokens_are_decode_steps(dtype, coded):
    from tests.kv_pool import decode
    lens = [1, 77, 640, 2000]
    pool, table, k, v = filled(dtype, coded, 2, 32, lens, 29, 63)
    q = fused(4, 8, dtype, extra=0)
    table, dlens, starts = device(lens, table, [1] * 4)
    got = prefill(pool, table, dlens, starts, q, 256, 2016, SCALE)
    check_all(got, pool, lens, [1] * 4, q, k, v)
    other = decode(pool, table, dlens, q.contiguous(), 256, 2016, SCALE)
    check_all(other, pool, lens, [1] * 4, q, k, v)


@BOTH
def test_many_sequences(coded):
    """More sequences than lanes, most of one token, many of none."""
    dtype, g = torch.bfloat16, torch.Generator().manual_seed(3)
    new = [int(x) for x in torch.randint(0, 3, (333,), generator=g)]
    new[70], new[250], new[332] = 150, 33, 129
    lens = [n + int(x) for n, x in zip(new, torch.randint(0, 60, (333,), generator=g))]
    pool, table, k, v = filled(dtype, coded, 1, 16, lens, 31, 14)
    q = fused(sum(new) + 2, 4, dtype)
    table, dlens, starts = device(lens, table, new)
    check_all(prefill(pool, table, dlens, starts, q, 0, 224, SCALE), pool, lens, new, q, k, v)


@BOTH
def test_starts_that_are_no_partition(coded):
    """Starts beyond the tokens and below zero are clamped, a descending pair is a sequence of no token; lengths beyond the table end with it."""
    dtype, lens = torch.float16, [64, 64, 64]
    pool, table, k, v = filled(dtype, coded, 1, 16, lens, 37, 4)
    q = fused(40, 2, dtype)
    starts = torch.tensor([-3, 20, 10, 1000], dtype=torch.int32, device=DEV)
    # tokens 0 .. 19 and, of the third sequence, 10 .. 39: the second has none; 10 .. 19 would belong to two, so the first has no keys
    # and the third's rows are looked at from token 20 on
    dlens = torch.tensor([-1, 64, 1 << 30], dtype=torch.int32, device=DEV)
    got = prefill(pool, table.to(DEV), dlens, starts, q, 64, 64, SCALE).cpu()
    assert (got[:10] == 0).all()
    sees = mask(64, 30)[10:]
    for h in range(2):
        check(got[20:, h], dtype, 1, q[20:, h].cpu(), k[2][0], v[2][0], SCALE, sees)


@TYPED
@BOTH
def test_repeats_bit_for_bit(dtype, coded):
    lens, new = [700, 65, 1, 1500], [700, 1, 1, 300]
    pool, table, k, v = filled(dtype, coded, 2, 16, lens, 23, 94)
    q = fused(sum(new), 8, dtype)
    table, dlens, starts = device(lens, table, new)
    fd = lib()
    for chunk in (256, 1536):
        shape = fd.make_shape(4, 8, 2, 128, 94 * 16, chunk, SCALE)
        ws = workspace(fd.fd_kv_prefill_workspace_bytes(shape, sum(new)))
        outs = [prefill(pool, table, dlens, starts, q, chunk, 94 * 16, SCALE, ws) for _ in range(4)]
        assert all(torch.equal(outs[0], x) for x in outs[1:])
        assert (ws[:1 << 14] == 0).all()


@TYPED
@BOTH
@pytest.mark.parametrize("hq,hkv,chunk,lens,new", [
    (20, 5, 1, [64 * 139 + 7, 500, 4160], [1, 4, 3]),                   # few rows: pieces of 64 keys
    (20, 5, 30, [64 * 139 + 7, 500, 4160], [40, 9, 1]),                 # two tiles: pieces of 64; one: 64
    (18, 1, 20, [128 * 70 + 1, 64], [20, 64]),                          # three tiles of 18 heads: pieces of 64; nine: 192
])
def test_many_pieces(dtype, coded, hq, hkv, chunk, lens, new):
    """More pieces of a row than lanes; the largest logits behind the first 64 pieces."""
    def change(b, which, x):
        if which == 0:
            x = x * 0.05
            x[:, -200:-100] = 2.0
        return x
    width = -(-max(lens) // 64) + 1
    pool, table, k, v = filled(dtype, coded, hkv, 64, lens, 43, width, 1.0, change)
    q = fused(sum(new), hq, dtype)
    q[:, ::2] = 1.0
    table, dlens, starts = device(lens, table, new)
    got = prefill(pool, table, dlens, starts, q, chunk, width * 64, 0.05)
    check_all(got, pool, lens, new, q, k, v, 0.05, heads=sorted({0, 1, hq // 2, hq - 2, hq - 1}))


@TYPED
@BOTH
@pytest.mark.parametrize("hq,hkv", [(24, 12), (300, 300), (33, 11)])
def test_launches_of_up_to_two_workgroups_a_compute_unit(dtype, coded, hq, hkv):
    """257 to 512 workgroups, also of head numbers that do not divide 256 or are larger."""
    batch = 360 // hkv
    g = torch.Generator().manual_seed(batch)
    new = [int(x) for x in torch.randint(0, 30, (batch,), generator=g)]
    new[0] = max(new[0], 2)
    lens = [n + int(x) for n, x in zip(new, torch.randint(0, 200, (batch,), generator=g))]
    assert 256 < (sum(new) * hq // hkv // 128 + batch) * hkv <= 512
    pool, table, k, v = filled(dtype, coded, hkv, 16, lens, 47, 15)
    q = fused(sum(new), hq, dtype)
    table, dlens, starts = device(lens, table, new)
    got = prefill(pool, table, dlens, starts, q, 240, 240, SCALE)
    check_all(got, pool, lens, new, q, k, v, heads=sorted({0, hq // 2, hq - 1}))
