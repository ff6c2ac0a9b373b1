"""Latent attention: rows into the cache, the absorbed form over the paged cache and the expanded form for prompts, against 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import cache_oracle as want

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float16, torch.bfloat16]


def lib():
    from paper_2311_01282_amd import fdattn
    return fdattn


def of(dtype):
    return lib().FD_F16 if dtype == torch.float16 else lib().FD_BF16


def filled(dtype, lens, page, width, seed):
    """A pool with NaN in every row that holds no token, and its table, with garbage in entries without tokens."""
    rng = np.random.default_rng(seed)
    n_pages = sum(-(-n // page) for n in lens) + 2
    rows = torch.full((n_pages, page, 576), float("nan"), dtype=dtype)
    order = rng.permutation(n_pages)
    table = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (len(lens), width))).to(torch.int32)
    g, at = torch.Generator().manual_seed(seed), 0
    for b, n in enumerate(lens):
        for j in range(-(-n // page)):
            table[b, j] = pg = int(order[at])
            at += 1
            live = min(page, n - j * page)
            rows[pg, :live] = torch.randn(live, 576, generator=g).to(dtype)
    return rows, table


def decode(rows, table, lens, ql, qr, chunk, max_seq, scale, out=None, ws=None):
    fd = lib()
    batch, heads = ql.shape[:2]
    shape = fd.make_shape(batch, heads, 1, 576, max_seq, chunk, scale)
    if not chunk:
        shape.chunk = fd.fd_latent_pick_chunk(shape)
        assert shape.chunk % 64 == 0 and shape.chunk >= 64
    nbytes = fd.fd_latent_workspace_bytes(shape)
    assert nbytes > 0
    if ws is None:
        ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device=DEV)
        fd.fd_cache_workspace_init(ws.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
    out = torch.full((batch + 1, heads, 512), float("nan"), dtype=rows.dtype, device=DEV) if out is None else out
    pool = fd.make_latent_pool(rows.data_ptr(), rows.shape[0], rows.shape[1], 512, 64, of(rows.dtype))
    fd.fd_latent_decode_attn(shape, pool, ql.data_ptr(), qr.data_ptr(), table.data_ptr(), lens.data_ptr(), out.data_ptr(), ws.data_ptr(),
                             ws.numel(), torch.cuda.current_stream().cuda_stream)
    return out


def tolerance(dtype, parts, products, q, k, v, scale, exp):
    """A score is an fp32 sum of `products` exact products: as many roundings of 2^-24 of at most |q| |k|; a weight carries twice that and 2^-21 of its
    exponential, and is rounded to `parts` numbers of the type.  Sums of keys / 32 terms.  One rounding at the end."""
    half = want.HALF_STEP[dtype]
    dx = products * 2.0 ** -24 * abs(scale) * float(q.norm(dim=-1).max() * k.norm(dim=-1).max())
    part = half if parts == 1 else half * half * 2
    top = float(v.abs().max())
    return exp.abs() * half * 1.01 + top * 2 * (2 * dx + 2.0 ** -21 + part + 2.0 ** -24 * (len(k) / 16 + 16)) + 2.0 ** -25


def check(got, rows, table, lens, ql, qr, scale):
    rows, ql, qr = rows.cpu(), ql.cpu().double(), qr.cpu().double()
    for b, n in enumerate(lens):
        x = got[b].cpu().double()
        if n == 0:
            assert (x == 0).all()
            continue
        k = want.gather(rows, table[b], n, rows.shape[1]).double()
        q = torch.cat([ql[b], qr[b]], -1)
        exp = want.attend(q, k, k[:, :512], scale)
        # (of more than 64 heads a weight is one number of the type: off by half a step of its own, as in the prompts)
        tol = tolerance(rows.dtype, 2 if len(q) <= 64 else 1, 576, q, k, k[:, :512], scale, exp)
        off = (x - exp).abs()
        assert torch.isfinite(x).all() and (off <= tol).all(), "sequence %d (%d keys): %.3g of the tolerance" % (b, n, float((off / tol).max()))


def queries(seed, batch, heads, dtype, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(size * torch.randn(batch, heads, d, generator=g)).to(dtype).to(DEV) for d in (512, 64)]


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("heads", [1, 3, 16, 17, 40, 64, 65, 128, 130])
def test_heads(dtype, heads):
    lens, page, max_seq = [1, 0, 200, 77], 16, 224
    rows, table = filled(dtype, lens, page, max_seq // page, heads)
    ql, qr = queries(heads, 4, heads, dtype)
    dl, dr = torch.tensor(lens, dtype=torch.int32, device=DEV), rows.to(DEV)
    for chunk in (64, 256):
        got = decode(dr, table.to(DEV), dl, ql, qr, chunk, max_seq, 0.07)
        torch.cuda.synchronize()
        check(got, rows, table, lens, ql, qr, 0.07)
        assert got[-1].isnan().all()


@pytest.mark.parametrize("page", [16, 64, 512])
@pytest.mark.parametrize("chunk", [64, 192, 320, 512, 1024, 0])
def test_lengths_pages_and_chunks(page, chunk):
    lens = [1, 15, 16, 17, 31, 32, 33, 63, 65, 127, 128, 129, 500, 1023, 0, 1024, 5000, -3]
    max_seq = 1024
    used = [min(max(n, 0), max_seq) for n in lens]
    rows, table = filled(torch.bfloat16, used, page, max_seq // page, page + chunk)
    ql, qr = queries(1, len(lens), 20, torch.bfloat16)
    got = decode(rows.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), ql, qr, chunk, max_seq, 0.07)
    torch.cuda.synchronize()
    check(got, rows, table, used, ql, qr, 0.07)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
def test_large_logits_and_growing_maxima(dtype):
    lens, max_seq = [900, 640], 1024
    rows, table = filled(dtype, lens, 32, max_seq // 32, 3)
    ql, qr = queries(2, 2, 33, dtype, 20.0)
    for chunk in (64, 256, 1024):
        got = decode(rows.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), ql, qr, chunk, max_seq, 0.07)
        torch.cuda.synchronize()
        check(got, rows, table, lens, ql, qr, 0.07)


@pytest.mark.parametrize("scale", [0.0, -0.07])
@pytest.mark.parametrize("heads", [5, 70])
def test_scales_of_zero_and_below(scale, heads):
    lens, max_seq = [300, 1, 65], 320
    rows, table = filled(torch.float16, lens, 16, max_seq // 16, 13)
    ql, qr = queries(8, 3, heads, torch.float16)
    for chunk in (64, 1024):
        got = decode(rows.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), ql, qr, chunk, max_seq, scale)
        torch.cuda.synchronize()
        check(got, rows, table, lens, ql, qr, scale)


@pytest.mark.parametrize("heads", [2, 66])
def test_rows_of_many_chunks(heads):
    lens, max_seq = [12800, 4161, 63], 12800
    rows, table = filled(torch.bfloat16, lens, 64, max_seq // 64, 14)
    ql, qr = queries(9, 3, heads, torch.bfloat16)
    got = decode(rows.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), ql, qr, 64, max_seq, 0.07)
    torch.cuda.synchronize()
    check(got, rows, table, lens, ql, qr, 0.07)


def test_nan_stays_in_its_sequence():
    lens, max_seq = [300, 300], 320
    rows, table = filled(torch.float16, lens, 16, max_seq // 16, 4)
    ql, qr = queries(5, 2, 20, torch.float16)
    dl, dt = torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV)
    clean = decode(rows.to(DEV), dt, dl, ql, qr, 128, max_seq, 0.07)
    rows[int(table[0, 5]), 3, 520] = float("nan")
    got = decode(rows.to(DEV), dt, dl, ql, qr, 128, max_seq, 0.07)
    torch.cuda.synchronize()
    assert got[0].isnan().all() and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("heads", [16, 100])
def test_pools_beyond_32_bits(heads):
    page = 256
    n_pages = (5 << 30) // (1152 * page)
    pool = torch.empty(n_pages, page, 576, dtype=torch.bfloat16, device=DEV)
    lens, max_seq = [400, 30], 512
    table = torch.tensor([[n_pages - 1, n_pages - 2], [n_pages - 3, -1]], dtype=torch.int32)
    slots = torch.tensor([int(table[b, t // page]) * page + t % page for b, n in enumerate(lens) for t in range(n)], dtype=torch.int32).to(DEV)
    x = torch.randn(sum(lens), 576, generator=torch.Generator().manual_seed(5)).bfloat16().to(DEV)
    lib().fd_latent_write(lib().make_latent_pool(pool.data_ptr(), n_pages, page, 512, 64, lib().FD_BF16), x.data_ptr(), 576, x[:, 512:].data_ptr(), 576,
                          len(x), slots.data_ptr(), torch.cuda.current_stream().cuda_stream)
    ql, qr = queries(6, 2, heads, torch.bfloat16)
    got = decode(pool, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), ql, qr, 128, max_seq, 0.07)
    torch.cuda.synchronize()
    last = pool[-3:].cpu()
    assert torch.equal(last[1, 399 - 256], x[399].cpu())
    check(got, last, torch.where(table < 0, table, table - (n_pages - 3)), lens, ql, qr, 0.07)


def test_decode_replays():
    lens, max_seq = [500, 33, 511], 512
    rows, table = filled(torch.float16, lens, 64, max_seq // 64, 3)
    ql, qr = queries(4, 3, 32, torch.float16)
    dr, dt, dl = rows.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    out = decode(dr, dt, dl, ql, qr, 128, max_seq, 0.07)
    ws = torch.zeros(lib().fd_latent_workspace_bytes(lib().make_shape(3, 32, 1, 576, max_seq, 128, 0.07)), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        decode(dr, dt, dl, ql, qr, 128, max_seq, 0.07, out, ws)
    for i in range(4):
        out.fill_(float("nan"))
        dl.copy_(torch.tensor([n - 7 * i for n in lens], dtype=torch.int32).clamp(min=0))
        graph.replay()
        torch.cuda.synchronize()
        again = decode(dr, dt, dl, ql, qr, 128, max_seq, 0.07)
        torch.cuda.synchronize()
        assert torch.equal(out[:3], again[:3])


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
def test_rows_into_the_cache(dtype):
    tokens, page, n_pages = 77, 32, 4
    g = torch.Generator().manual_seed(1)
    fused = torch.randn(tokens, 640, generator=g).to(dtype).to(DEV)
    slots = torch.randperm(n_pages * page, generator=g)[:tokens].to(torch.int32)
    slots[5], slots[6], slots[7] = -1, n_pages * page, 2 ** 31 - 1
    pool = torch.full((n_pages, page, 576), 3.0, dtype=dtype, device=DEV)
    handle = lib().make_latent_pool(pool.data_ptr(), n_pages, page, 512, 64, of(dtype))
    ds = slots.to(DEV)
    lib().fd_latent_write(handle, fused.data_ptr(), 640, fused[:, 560:].data_ptr(), 640, tokens, ds.data_ptr(),
                          torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    exp = torch.full((n_pages * page, 576), 3.0, dtype=dtype)
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < n_pages * page:
            exp[s] = torch.cat([fused[t, :512].cpu(), fused[t, 560:624].cpu()])
    assert torch.equal(pool.cpu().view(-1, 576), exp)


# ---- prompts ----

def prompt(dtype, lens, heads, max_seq, rope_stride, seed, size=1.0):
    """Operands with NaN in every row at and behind a prompt's length."""
    g = torch.Generator().manual_seed(seed)
    batch = len(lens)
    q = size * torch.randn(batch, max_seq, heads, 192, generator=g)
    kv = torch.randn(batch, max_seq, heads, 256, generator=g)
    rope = torch.randn(batch, max_seq, rope_stride, generator=g)
    for b, n in enumerate(lens):
        for x in (q, kv, rope):
            x[b, max(n, 0):] = float("nan")
    return [x.to(dtype).to(DEV) for x in (q, kv, rope)]


def prefill(q, kv, rope, lens, scale, out=None):
    fd = lib()
    batch, max_seq, heads = q.shape[:3]
    shape = fd.make_shape(batch, heads, heads, 192, max_seq, 0, scale)
    out = torch.full((batch + 1, max_seq, heads, 128), float("nan"), dtype=q.dtype, device=DEV) if out is None else out
    fd.fd_latent_prefill_attn(shape, of(q.dtype), q.data_ptr(), kv.data_ptr(), rope[..., -64:].data_ptr(), rope.stride(1), lens.data_ptr(),
                              out.data_ptr(), torch.cuda.current_stream().cuda_stream)
    return out


def check_prompt(got, q, kv, rope, lens, scale):
    dtype = q.dtype
    q, kv, rope, got = (x.cpu().double() for x in (q, kv, rope[..., -64:], got))
    max_seq = q.shape[1]
    for b, n in enumerate(lens):
        n = min(max(n, 0), max_seq)
        assert (got[b, n:] == 0).all()
        if not n:
            continue
        below = torch.ones(n, n, dtype=torch.bool).tril()
        for h in range(q.shape[2]):
            k = torch.cat([kv[b, :n, h, :128], rope[b, :n]], -1)
            v = kv[b, :n, h, 128:]
            x = torch.where(below, scale * (q[b, :n, h] @ k.t()), -math.inf)
            exp = torch.softmax(x, -1) @ v
            tol = tolerance(dtype, 1, 192, q[b, :n, h], k, v, scale, exp)
            off = (got[b, :n, h] - exp).abs()
            assert torch.isfinite(got[b, :n, h]).all() and (off <= tol).all(), "sequence %d, head %d: %.3g of the tolerance" % (
                b, h, float((off / tol).max()))


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("lens,heads,max_seq,rope_stride", [
    ([1], 1, 1, 64), ([31, 32, 33, 0], 2, 40, 576), ([127, 128, 129, 1], 3, 129, 72), ([300, -2, 511], 2, 300, 576), ([257, 640], 9, 640, 64)])
def test_prompts(dtype, lens, heads, max_seq, rope_stride):
    q, kv, rope = prompt(dtype, lens, heads, max_seq, rope_stride, heads)
    got = prefill(q, kv, rope, torch.tensor(lens, dtype=torch.int32, device=DEV), 0.0722)
    torch.cuda.synchronize()
    check_prompt(got, q, kv, rope, lens, 0.0722)
    assert got[-1].isnan().all()


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("size", [1.0, 20.0])
def test_prompts_of_many_workgroups(dtype, size):
    """Of the launches above each workgroup of prompts beyond 256 tokens is split in halves; here it is not."""
    lens, heads, max_seq = [400, 0, 333], 70, 400
    q, kv, rope = prompt(dtype, lens, heads, max_seq, 64, 7, size)
    got = prefill(q, kv, rope, torch.tensor(lens, dtype=torch.int32, device=DEV), 0.0722)
    torch.cuda.synchronize()
    few = [0, 33, 69]
    check_prompt(got[:3, :, few], q[:, :, few], kv[:, :, few], rope, lens, 0.0722)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
def test_prompts_with_large_logits(dtype):
    q, kv, rope = prompt(dtype, [400, 257], 2, 416, 576, 3, 20.0)
    got = prefill(q, kv, rope, torch.tensor([400, 257], dtype=torch.int32, device=DEV), 0.0722)
    torch.cuda.synchronize()
    check_prompt(got, q, kv, rope, [400, 257], 0.0722)


@pytest.mark.parametrize("scale", [0.0, -0.07])
@pytest.mark.parametrize("lens,max_seq", [([170, 33], 200), ([300, 64], 320)])
def test_prompts_with_scales_of_zero_and_below(scale, lens, max_seq):
    q, kv, rope = prompt(torch.float16, lens, 3, max_seq, 64, 5)
    got = prefill(q, kv, rope, torch.tensor(lens, dtype=torch.int32, device=DEV), scale)
    torch.cuda.synchronize()
    check_prompt(got, q, kv, rope, lens, scale)


def test_a_prompt_does_not_see_later_keys():
    """Infinite and NaN keys and rotary parts behind a query do not reach it, in either form of the launch."""
    for max_seq in (224, 420):
        n = max_seq - 4
        q, kv, rope = prompt(torch.bfloat16, [n], 2, max_seq, 64, 9)
        lens = torch.tensor([n], dtype=torch.int32, device=DEV)
        clean = prefill(q, kv, rope, lens, 0.07)
        kv[0, 150, 0, 5], kv[0, 170, 0, 7], rope[0, 200, 3] = float("nan"), float("inf"), float("nan")
        got = prefill(q, kv, rope, lens, 0.07)
        torch.cuda.synchronize()
        assert torch.equal(got[0, :150, 0], clean[0, :150, 0]) and torch.equal(got[0, :200, 1], clean[0, :200, 1])
        assert got[0, 150:n, 0].isnan().all() and got[0, 200:n, 1].isnan().all()


def test_prompts_beyond_32_bits():
    """The second sequence starts 4.6 GB into the keys and values."""
    heads, max_seq, n = 128, 70000, 150
    q, kv = (torch.empty(2, max_seq, heads, d, dtype=torch.bfloat16, device=DEV) for d in (192, 256))
    rope = torch.empty(2, max_seq, 64, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator().manual_seed(6)
    for x in (q, kv, rope):
        x[1, :n] = torch.randn(n, *x.shape[2:], generator=g).bfloat16().to(DEV)
    got = prefill(q, kv, rope, torch.tensor([0, n], dtype=torch.int32, device=DEV), 0.07)
    torch.cuda.synchronize()
    assert not got[0].any() and not got[1, n:].any() and got[2, :5].isnan().all()
    few = [0, 77, 127]
    check_prompt(got[1:2, :n, few], q[1:2, :n, few], kv[1:2, :n, few], rope[1:2, :n], [n], 0.07)


def test_prompt_replays():
    q, kv, rope = prompt(torch.bfloat16, [300, 200], 2, 300, 576, 4)
    lens = torch.tensor([300, 200], dtype=torch.int32, device=DEV)
    out = prefill(q, kv, rope, lens, 0.07)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        prefill(q, kv, rope, lens, 0.07, out)
    for n in (300, 100, 33):
        lens[0] = n
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        again = prefill(q, kv, rope, lens, 0.07)
        torch.cuda.synchronize()
        assert torch.equal(out[:2], again[:2])
