"""The calls over the paged cache of 16 or 8 bits as a server makes them: pages and slots for the step's tokens, rows into the cache, attention of all new
tokens at once and of the last ones again as a decode step; captured and eager; workspaces that change shapes; streams; rows beyond 4 GiB."""
import math

import pytest
import torch

from tests import kv_oracle as want
from tests import kv_pool
from tests.kv_pool import DEV, Pool, check, filled, lib, stream, workspace
from tests.test_gpu_kv_prefill import fused, starts_of
from tests.test_gpu_small_caches import Steps

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)
STEPS = [[37, 5, 0, 64, 1], [1, 1, 20, 1, 1], [1] * 5, [1, 1, 1, 90, 1], [0, 30, 1, 1, 1], [1] * 5]        # the fourth asks for more than is free


@pytest.mark.parametrize("dtype,coded,chunk", [(torch.float16, True, 16), (torch.bfloat16, True, 1024), (torch.float16, False, 1024), (torch.bfloat16, False, 32)],
                         ids=["e4m3-fp16-cut", "e4m3-bf16", "fp16", "bf16-cut"])
@pytest.mark.parametrize("captured", [False, True], ids=["eager", "captured"])
def test_steps(dtype, coded, chunk, captured):
    hkv, hq, page, width, max_tokens = 2, 8, 16, 9, 120
    st = Steps(5, page, 13, width, max_tokens)
    pool = Pool(13, page, hkv, dtype, coded)
    g = torch.Generator().manual_seed(2)
    x = torch.zeros(max_tokens, hq + 2 * hkv, 128, dtype=dtype, device=DEV)                 # queries, keys and values of a fused projection
    out = torch.zeros(max_tokens, hq, 128, dtype=dtype, device=DEV)
    last, out_last = torch.zeros(5, hq, 128, dtype=dtype, device=DEV), torch.zeros(5, hq, 128, dtype=dtype, device=DEV)
    shape, one = (lib().make_shape(5, hq, hkv, 128, page * width, c, SCALE) for c in (chunk, 64))
    ws = workspace(max(lib().fd_kv_prefill_workspace_bytes(shape, max_tokens), lib().fd_kv_workspace_bytes(one)))
    handle, apart = pool.handle(), (hq + 2 * hkv) * 128

    def step():
        s = stream()
        st.tables(s)
        lib().fd_kv_write(handle, x[:, hq:].data_ptr(), apart, x[:, hq + hkv:].data_ptr(), apart, max_tokens, st.slots.data_ptr(), s)
        lib().fd_kv_prefill_attn(shape, handle, x.data_ptr(), apart, max_tokens, st.starts.data_ptr(), st.table.data_ptr(), st.lens.data_ptr(),
                                 out.data_ptr(), ws.data_ptr(), ws.numel(), s)
        lib().fd_kv_decode_attn(one, handle, last.data_ptr(), st.table.data_ptr(), st.lens.data_ptr(), out_last.data_ptr(), ws.data_ptr(), ws.numel(), s)

    torch.cuda.synchronize()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            step()
    rows = [[torch.zeros(hkv, 0, 128, dtype=torch.float64) for _ in range(5)] for _ in range(2)]      # what the cache stands for
    refused = 0
    for new in STEPS:
        st.new.copy_(torch.tensor(new, dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=g).to(dtype))
        starts = [0] + torch.tensor(new).cumsum(0).tolist()
        for b, n in enumerate(new):
            last[b].copy_(x[max(starts[b + 1] - 1, 0), :hq])
        out.fill_(7.0)
        graph.replay() if captured else step()
        torch.cuda.synchronize()
        before = list(st.host["cached"])
        lens, _ = st.expect(new)
        host, got, got_last = x.cpu(), out.cpu(), out_last.cpu()
        for b, (n, L) in enumerate(zip(new, lens)):
            if L == before[b] + n:
                for which in range(2):
                    fresh = host[starts[b]:starts[b] + n, hq + which * hkv:hq + (which + 1) * hkv].transpose(0, 1)
                    if coded:
                        fresh = [[want.code_row(fresh[h, t]) for t in range(n)] for h in range(hkv)]
                        fresh = torch.stack([torch.stack([want.values(torch.from_numpy(c), torch.tensor(e)) for c, e in one_head]) for one_head in fresh]) \
                            if n else torch.zeros(hkv, 0, 128, dtype=torch.float64)
                    rows[which][b] = torch.cat([rows[which][b], fresh.double()], 1)
            else:
                refused += 1
                assert not got[starts[b]:starts[b] + n].isnan().any()
            for h in range(hq):
                k, v = rows[0][b][h // 4], rows[1][b][h // 4]
                if L == before[b] + n and n:
                    sees = torch.arange(L)[None, :] < torch.tensor([want.visible(L, n, i) for i in range(n)])[:, None]
                    check(got[starts[b]:starts[b] + n, h], dtype, 1, host[starts[b]:starts[b] + n, h], k, v, SCALE, sees, "request %d" % b)
                if L:
                    check(got_last[b, h:h + 1], dtype, 2, last[b, h:h + 1].cpu(), k, v, SCALE, what="request %d, last token" % b)
        assert (got[starts[-1]:] == 7.0).all() and (ws[:1 << 14] == 0).all()
        st.after()
    assert refused


@pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])
def test_one_workspace_for_every_shape(coded):
    """Prepared once, then used by the calls in turn, prompts that are cut and that are not; its counters are zero behind each."""
    dtype = torch.bfloat16
    ws = torch.full((256 << 20,), 0xFF, dtype=torch.uint8, device=DEV)
    lib().fd_cache_workspace_init(ws.data_ptr(), ws.numel(), stream())
    for i, (lens, new, hq, hkv, chunk) in enumerate([([700, 33], [40, 33], 8, 2, 64), ([256] * 70, [1] * 70, 4, 4, 64), ([1000], [1000], 6, 1, 16), ([90, 2000, 5], [1, 3, 5], 16, 1, 256)]):
        width = -(-max(lens) // 16)
        pool, table, k, v = filled(dtype, coded, hkv, 16, lens, i, width)
        q, d = fused(sum(new), hq, dtype, i), torch.tensor(lens, dtype=torch.int32, device=DEV)
        args = (pool, table.to(DEV), d, starts_of(new).to(DEV), q, chunk, 16 * width, SCALE)
        got, alone = kv_pool.prefill(*args, ws=ws), kv_pool.prefill(*args)
        assert torch.equal(got, alone) and not ws[:1 << 14].any()
        rows = q[starts_of(new)[1:].to(DEV).long() - 1].contiguous()
        args = (pool, table.to(DEV), d, rows, 64 * (1 + i), 16 * width, SCALE)
        got, alone = kv_pool.decode(*args, ws=ws), kv_pool.decode(*args)
        assert torch.equal(got, alone) and not ws[:1 << 14].any()


def test_two_streams_with_a_workspace_each():
    dtype, lens, new, width = torch.float16, [2000, 700, 1], [300, 1, 1], 63
    pool, table, _, _ = filled(dtype, True, 2, 32, lens, 1, width)
    other, table2, _, _ = filled(dtype, False, 2, 32, lens, 2, width)
    q, d, starts = fused(sum(new), 16, dtype), torch.tensor(lens, dtype=torch.int32, device=DEV), starts_of(new).to(DEV)
    last = q[starts[1:].long() - 1].contiguous()
    table, table2 = table.to(DEV), table2.to(DEV)
    first = kv_pool.prefill(pool, table, d, starts, q, 128, 32 * width, SCALE)
    second = kv_pool.decode(other, table2, d, last, 256, 32 * width, SCALE)
    spaces = [workspace(1 << 26) for _ in range(2)]
    outs, streams = [torch.full_like(first, 3.0), torch.full_like(second, 3.0)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(streams[0]):
            kv_pool.prefill(pool, table, d, starts, q, 128, 32 * width, SCALE, spaces[0], outs[0])
        with torch.cuda.stream(streams[1]):
            kv_pool.decode(other, table2, d, last, 256, 32 * width, SCALE, spaces[1], outs[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], first) and torch.equal(outs[1], second)


@pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])
def test_rows_beyond_four_gib(coded):
    """Slots up to 2^25 of a pool of more than 4 GiB: every call finds the same rows at its end as in a small pool."""
    dtype, hkv, page, lens, new, width = torch.bfloat16, 8 if coded else 4, 32, [333, 50], [100, 1], 11
    small, table, _, _ = filled(dtype, coded, hkv, page, lens, 3, width)
    n_pages = (1 << 32) // (hkv * page * (128 if coded else 256)) + 7
    big = Pool.__new__(Pool)
    big.n_pages, big.page, big.hkv, big.dtype, big.coded = n_pages, page, hkv, dtype, coded
    shift = n_pages - small.n_pages
    big.rows, big.scales = [], [None, None]
    for i in range(2):
        x = torch.empty((n_pages,) + tuple(small.rows[i].shape[1:]), dtype=small.rows[i].dtype, device=DEV)
        x[shift:] = small.rows[i]
        big.rows.append(x)
        if coded:
            s = torch.empty((n_pages,) + tuple(small.scales[i].shape[1:]), dtype=torch.uint8, device=DEV)
            s[shift:] = small.scales[i]
            big.scales[i] = s
    assert big.rows[0].numel() * big.rows[0].element_size() > 1 << 32
    far = torch.where((table >= 0) & (table < small.n_pages), table + shift, 0)
    q, d, starts = fused(sum(new), 16, dtype), torch.tensor(lens, dtype=torch.int32, device=DEV), starts_of(new).to(DEV)
    last = q[starts[1:].long() - 1].contiguous()
    for chunk in (32, 352):
        a, b = (kv_pool.prefill(p, t.to(DEV), d, starts, q, chunk, page * width, SCALE) for p, t in ((small, table), (big, far)))
        assert torch.equal(a, b)
    a, b = (kv_pool.decode(p, t.to(DEV), d, last, 64, page * width, SCALE) for p, t in ((small, table), (big, far)))
    assert torch.equal(a, b)
    x = torch.randn(40, 2 * hkv, 128, generator=torch.Generator().manual_seed(5)).to(dtype).to(DEV)
    back = torch.zeros(2, 2, 40, hkv, 128, dtype=dtype, device=DEV)
    for i, (p, first) in enumerate(((small, 0), (big, shift * page))):
        slots = (first + torch.arange(40, dtype=torch.int32)).to(DEV)
        lib().fd_kv_write(p.handle(), x.data_ptr(), 2 * hkv * 128, x[:, hkv:].data_ptr(), 2 * hkv * 128, 40, slots.data_ptr(), stream())
        lib().fd_kv_read(p.handle(), slots.data_ptr(), 40, back[i][0].data_ptr(), hkv * 128, back[i][1].data_ptr(), hkv * 128, stream())
    torch.cuda.synchronize()
    assert torch.equal(back[0], back[1]) and (back[0] != 0).any()
