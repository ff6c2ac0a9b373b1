"""Decode attention over the paged cache of 16 or 8 bits, against 64 bits."""
import math

import pytest
import torch

from tests.kv_pool import DEV, TYPES, check, decode, filled, lib, workspace

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)
BOTH = pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])
TYPED = pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])


def check_all(got, pool, lens, q, k, v, scale=SCALE):
    share = q.shape[1] // pool.hkv
    got, q = got.cpu(), q.cpu()
    for b, n in enumerate(lens):
        if n <= 0:
            assert (got[b] == 0).all()
            continue
        for h in range(pool.hkv):
            of = slice(h * share, (h + 1) * share)
            check(got[b, of], pool.dtype, 2, q[b, of], k[b][h], v[b][h], scale, what="sequence %d, KV head %d" % (b, h))


def queries(batch, hq, dtype, seed=1, size=1.0):
    return (size * torch.randn(batch, hq, 128, generator=torch.Generator().manual_seed(seed))).to(dtype).to(DEV)


def device(lens, table):
    return table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)


@TYPED
@BOTH
@pytest.mark.parametrize("hq,hkv,page,chunk,max_seq", [
    (1, 1, 16, 64, 2512), (4, 4, 16, 256, 2512), (8, 2, 32, 1024, 2528), (6, 1, 256, 4096, 2560), (9, 1, 16, 128, 2512), (16, 1, 64, 512, 2560),
    (28, 4, 128, 0, 2560), (40, 1, 16, 320, 2512), (35, 5, 16, 16384, 2512),
])
def test_against_64_bits(dtype, coded, hq, hkv, page, chunk, max_seq):
    lens = [1, 200, 0, 77, 31, 1024, 2500]
    pool, table, k, v = filled(dtype, coded, hkv, page, lens, hq + page, max_seq // page)
    q = queries(len(lens), hq, dtype)
    table, dlens = device(lens, table)
    check_all(decode(pool, table, dlens, q, chunk, max_seq, SCALE), pool, lens, q, k, v)


@TYPED
@BOTH
def test_every_length_around_a_block(dtype, coded):
    lens = list(range(0, 70)) + [127, 128, 129, 160]
    pool, table, k, v = filled(dtype, coded, 1, 16, lens, 5, 10)
    q = queries(len(lens), 3, dtype)
    table, dlens = device(lens, table)
    check_all(decode(pool, table, dlens, q, 64, 160, SCALE), pool, lens, q, k, v)


@TYPED
@BOTH
@pytest.mark.parametrize("scale,size", [(-0.2, 1.0), (0.0, 1.0), (1.0, 3.0), (1e-30, 1.0)])
def test_scales(dtype, coded, scale, size):
    lens = [333, 64]
    pool, table, k, v = filled(dtype, coded, 2, 32, lens, 9, 11, size)
    q = queries(2, 8, dtype, size=size)
    table, dlens = device(lens, table)
    check_all(decode(pool, table, dlens, q, 128, 352, scale), pool, lens, q, k, v, scale)


@TYPED
@BOTH
def test_first_keys_far_below_and_far_above(dtype, coded):
    """A running maximum that grows late, one that never does, and thousands of small weights beside a large one."""
    lens, n = [3000, 3000, 3000], 3000

    def change(b, which, x):
        if which == 0:
            x = x * 0.05
            x[:, n - 1 if b == 0 else 0] = 3.0 if b < 2 else -3.0
        return x
    pool, table, k, v = filled(dtype, coded, 1, 64, lens, 11, 47, 1.0, change)
    q = torch.ones(3, 4, 128, dtype=dtype, device=DEV)
    table, dlens = device(lens, table)
    for chunk in (64, 1024, 16384):
        check_all(decode(pool, table, dlens, q, chunk, 47 * 64, 0.05), pool, lens, q, k, v, 0.05)


@TYPED
@BOTH
def test_values_that_are_not_finite(dtype, coded):
    """What is not finite behind a sequence does not matter (the pool is garbage there); within it an infinite value (of 8 bits: the row is NaN)
    reaches its own head's elements and no other head or sequence."""
    lens = [100, 90, 33]

    def change(b, which, x):
        if which and b == 1:
            x[0, 89, 5] = float("inf")
        return x
    pool, table, k, v = filled(dtype, coded, 2, 16, lens, 13, 7, 1.0, change)
    q = queries(3, 4, dtype)
    table, dlens = device(lens, table)
    got = decode(pool, table, dlens, q, 64, 112, SCALE).cpu()
    odd = got[1, :2].clone()
    got[1, :2] = 0
    assert got.isfinite().all()
    if coded:
        assert odd.isnan().all()
    else:
        assert (odd[:, 5] == float("inf")).all() and odd[:, :5].isfinite().all() and odd[:, 6:].isfinite().all()


@TYPED
@BOTH
def test_rows_without_a_number_and_infinite_logits(dtype, coded):
    """NaN in a key is NaN in the output; keys at minus infinity count as nothing."""
    lens = [70, 130]

    def change(b, which, x):
        if not which and b == 0:
            x[0, 40, 3] = float("nan")
        if not which and b == 1 and not coded:
            x[:, :100, 0] = float("-inf")
        return x
    pool, table, k, v = filled(dtype, coded, 1, 16, lens, 17, 9, 1.0, change)
    q = queries(2, 2, dtype).abs()
    table, dlens = device(lens, table)
    got = decode(pool, table, dlens, q, 64, 144, SCALE).cpu()
    assert got[0].isnan().all()
    check(got[1], dtype, 2, q[1].cpu(), k[1][0][0 if coded else 100:], v[1][0][0 if coded else 100:], SCALE)


@BOTH
def test_lengths_beyond_the_table_and_below_zero(coded):
    dtype, lens = torch.float16, [128, 64]
    pool, table, k, v = filled(dtype, coded, 1, 16, lens, 19, 8)
    q = queries(2, 2, dtype)
    got = decode(pool, table.to(DEV), torch.tensor([1 << 30, -5], dtype=torch.int32, device=DEV), q, 64, 128, SCALE)
    check_all(got, pool, [128, 0], q, k, v)


@TYPED
@BOTH
def test_repeats_bit_for_bit_and_leaves_the_pool_alone(dtype, coded):
    lens = [2000, 900, 1, 0]
    pool, table, k, v = filled(dtype, coded, 4, 16, lens, 23, 125)
    q = queries(4, 16, dtype)
    table, dlens = device(lens, table)
    before = [x.clone() for x in pool.rows]
    fd = lib()
    for chunk in (128, 64, 2048):
        shape = fd.make_shape(4, 16, 4, 128, 2000, chunk, SCALE)
        ws = workspace(fd.fd_kv_workspace_bytes(shape))
        outs = [decode(pool, table, dlens, q, chunk, 2000, SCALE, ws) for _ in range(4)]
        assert all(torch.equal(outs[0], x) for x in outs[1:])
        assert (ws[:1 << 14] == 0).all()
    bits = torch.uint8 if coded else torch.int16
    assert all(torch.equal(a.view(bits), b.view(bits)) for a, b in zip(before, pool.rows))


@TYPED
@BOTH
@pytest.mark.parametrize("batch,hq,hkv", [(40, 8, 8), (64, 10, 5), (65, 8, 4), (33, 80, 4), (2, 130, 130), (3, 258, 86), (57, 9, 9)])
@pytest.mark.parametrize("kind", ["random", "equal", "edges"])
def test_whole_rows_sorted_by_length(dtype, coded, batch, hq, hkv, kind):
    """Launches of more workgroups than compute units in one chunk a row: a row that is done twice or not at all shows."""
    g = torch.Generator().manual_seed(batch)
    lens = [int(x) for x in torch.randint(0, 161, (batch,), generator=g)]
    if kind == "equal":
        lens = [77] * batch
    if kind == "edges":
        lens = [[0, 160, 1, 32, 33, 160][i % 6] for i in range(batch)]
    pool, table, k, v = filled(dtype, coded, hkv, 16, lens, batch, 10)
    q = queries(batch, hq, dtype)
    table, dlens = device(lens, table)
    shape = lib().make_shape(batch, hq, hkv, 128, 160, 0, SCALE)
    assert lib().fd_kv_pick_chunk(shape) >= 160
    got = decode(pool, table, dlens, q, 0, 160, SCALE)
    assert not got.isnan().any()
    few = [b for b in range(batch) if b < 6 or b > batch - 4]           # (the others by the rows without keys and by the check for NaN)
    got, qc, share = got.cpu(), q.cpu(), hq // hkv
    for b in few:
        for h in range(hkv):
            of = slice(h * share, (h + 1) * share)
            if lens[b]:
                check(got[b, of], dtype, 2, qc[b, of], k[b][h], v[b][h], SCALE, what="sequence %d, KV head %d" % (b, h))
    assert all((got[b] == 0).all() == (lens[b] == 0) for b in range(batch))


def test_agrees_with_the_calibrated_call_over_its_pool():
    """With fp16 rows the pool is that of fd_decode_attn_paged."""
    dtype = torch.float16
    from paper_2311_01282_amd import synth
    fd, lens = lib(), [700, 33, 0]
    pool, table, k, v = filled(dtype, False, 2, 32, lens, 41, 24)
    q = queries(3, 8, dtype)
    table, dlens = device(lens, table)
    got = decode(pool, table, dlens, q, 256, 768, SCALE)
    shape = fd.make_shape(3, 8, 2, 128, 768, 256, SCALE)
    ws = torch.zeros(fd.fd_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    other = torch.full_like(got, float("nan"))
    stream = torch.cuda.current_stream().cuda_stream
    fd.fd_workspace_init(shape, ws.data_ptr(), ws.numel(), stream)
    fd.fd_decode_attn_paged(shape, q.data_ptr(), pool.rows[0].data_ptr(), pool.rows[1].data_ptr(), table.data_ptr(), 32, pool.n_pages, dlens.data_ptr(),
                            synth.PHI, synth.BOUNDS, other.data_ptr(), ws.data_ptr(), ws.numel(), stream)
    check_all(got, pool, lens, q, k, v)
    check_all(other, pool, lens, q, k, v)


@TYPED
@BOTH
@pytest.mark.parametrize("hq,hkv,chunk,lens", [
    (1, 1, 64, [40000, 33000]),                                         # hundreds of pieces of a row, joined 16 at a time
    (4, 2, 64, [128 * 129, 1, 0, 128 * 64 + 1, 127]),
    (20, 1, 128, [20000, 0, 0, 19999, 5000]),                           # two tiles of heads
    (12, 12, 64, [0] * 12), (8, 8, 64, [3000] * 8),
    (3, 3, 512, [9000, 100, 4000, 8999, 1, 777, 0, 6000, 5, 4321, 8192, 2048]),
    (8, 8, 192, [100 + 37 * i for i in range(64)]),                     # four rounds of the chip
])
def test_pieces_by_the_lengths(dtype, coded, hq, hkv, chunk, lens):
    """Launches of more than 256 chunks.  The largest logits of every row at its end."""
    def change(b, which, x):
        if which == 0:
            x = x * 0.05
            x[:, -150:-90] = 2.0
        return x
    width = -(-max(max(lens), 64 * 40) // 64) + 1
    assert len(lens) * hkv * -(-hq // hkv // 16) * -(-width * 64 // chunk) > 256
    pool, table, k, v = filled(dtype, coded, hkv, 64, lens, 53, width, 1.0, change)
    q = queries(len(lens), hq, dtype)
    q[:, ::2] = 1.0
    table, dlens = device(lens, table)
    fd = lib()
    shape = fd.make_shape(len(lens), hq, hkv, 128, width * 64, chunk, 0.05)
    ws = workspace(fd.fd_kv_workspace_bytes(shape))
    got = decode(pool, table, dlens, q, chunk, width * 64, 0.05, ws)
    some = [b for b in range(len(lens)) if b < 12 or b > len(lens) - 3]
    out, qc, share = got.cpu(), q.cpu(), hq // hkv
    for b in range(len(lens)):
        assert (out[b] == 0).all() if lens[b] == 0 else not out[b].isnan().any()
        for h in range(hkv) if b in some and lens[b] else ():
            check(out[b, h * share:(h + 1) * share], dtype, 2, qc[b, h * share:(h + 1) * share], k[b][h], v[b][h], 0.05, what="sequence %d, KV head %d" % (b, h))
    assert (ws[:1 << 14] == 0).all()
    for _ in range(3):
        assert torch.equal(decode(pool, table, dlens, q, chunk, width * 64, 0.05, ws), got)
    assert (ws[:1 << 14] == 0).all()


@BOTH
def test_pieces_follow_the_lengths_of_a_replay(coded):
    """A captured call, replayed with other lengths: other pieces, other joins."""
    dtype, lens = torch.bfloat16, [9000, 200, 4097, 1, 6000, 33]
    pool, table, k, v = filled(dtype, coded, 2, 64, lens, 59, 141)
    q = queries(len(lens), 8, dtype)
    table, dlens = device(lens, table)
    fd = lib()
    shape = fd.make_shape(len(lens), 8, 2, 128, 141 * 64, 256, SCALE)
    ws = workspace(fd.fd_kv_workspace_bytes(shape))
    out = torch.full_like(q, float("nan"))
    graph = torch.cuda.CUDAGraph()
    decode(pool, table, dlens, q, 256, 141 * 64, SCALE, ws, out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        decode(pool, table, dlens, q, 256, 141 * 64, SCALE, ws, out)
    for now in ([9000, 200, 4097, 1, 6000, 33], [1, 0, 4000, 1, 128, 32], [0] * 6, [8999, 200, 1, 1, 5999, 33], [9000, 200, 4097, 1, 6000, 33]):
        dlens.copy_(torch.tensor(now, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check_all(out, pool, now, q, [x[:, :n] for x, n in zip(k, now)], [x[:, :n] for x, n in zip(v, now)])
        assert torch.equal(out, decode(pool, table, dlens, q, 256, 141 * 64, SCALE))
