"""The 4-bit cache: rows in and out bit for bit, and the decode attention against 64 bits."""
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


class Pool:
    """A pool on the GPU, garbage in every row: codes at random, scales NaN."""

    def __init__(self, n_pages, page, hkv, group, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.n_pages, self.page, self.hkv, self.group, self.dtype = n_pages, page, hkv, group, dtype
        self.codes = [torch.randint(0, 256, (n_pages, hkv, page, 64), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2)]
        self.scales = [torch.full((n_pages, hkv, page, 2, 128 // group), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]

    def handle(self):
        ptrs = [x.data_ptr() for x in (self.codes[0], self.scales[0], self.codes[1], self.scales[1])]
        return lib().make_nibble_pool(*ptrs, self.n_pages, self.page, self.hkv, 128, self.group, of(self.dtype))


def rows_like(seed, tokens, hkv, dtype, extra=0):
    """K and V as the ends of a fused projection's rows, with values of very different sizes."""
    g = torch.Generator().manual_seed(seed)
    fused = torch.randn(tokens, extra + 2 * hkv, 128, generator=g)
    fused *= 10.0 ** torch.randint(-3, 4, (tokens, extra + 2 * hkv, 1), generator=g)
    fused[:, extra] += 3.0
    fused = fused.to(dtype)
    return fused.to(DEV), fused[:, extra:extra + hkv], fused[:, extra + hkv:]


def write(pool, fused, extra, slots):
    k, v = fused[:, extra:extra + pool.hkv], fused[:, extra + pool.hkv:]
    lib().fd_nibble_write(pool.handle(), k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0), len(fused), slots.data_ptr(),
                       torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("tokens,hkv,page,extra", [(1, 1, 16, 0), (5, 3, 16, 2), (77, 8, 64, 8), (300, 2, 32, 0)])
def test_rows_in_and_out(dtype, group, tokens, hkv, page, extra):
    n_pages = -(-tokens // page) + 3
    fused, k, v = rows_like(tokens, tokens, hkv, dtype, extra)
    special = [(0, 0), (tokens // 2, hkv - 1)]
    for x, (t, h) in ((k, special[0]), (v, special[1])):
        x[t, h, :32] = 1.5                                             # a group without a range
        x[t, h, 64] = float("inf")
        x[t, h, 127] = float("nan")
    fused.copy_(fused.cpu())
    dev = fused.clone()
    dev[:, extra:extra + hkv], dev[:, extra + hkv:] = k.to(DEV), v.to(DEV)
    pool = Pool(n_pages, page, hkv, group, dtype)
    before = [x.clone() for x in pool.codes + pool.scales]
    g = torch.Generator().manual_seed(3)
    slots = torch.randperm(n_pages * page, generator=g)[:tokens].to(torch.int32)
    live = torch.ones(tokens, dtype=torch.bool)
    if tokens > 3:
        slots[1], slots[2], slots[3] = -1, n_pages * page, -2 ** 31     # padding, and slots behind the pool
        live[1:4] = False
    dslots = slots.to(DEV)
    write(pool, dev, extra, dslots)
    back = torch.full((2, tokens, hkv, 128), 7.0, dtype=dtype, device=DEV)
    lib().fd_nibble_read(pool.handle(), dslots.data_ptr(), tokens, back[0].data_ptr(), hkv * 128, back[1].data_ptr(), hkv * 128,
                      torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    exp = [x.cpu().clone() for x in before]
    for which, x in enumerate((k, v)):
        for h in range(hkv):
            codes, s, low = want.nibble_code(x[live][:, h], group)
            packed = want.nibble_pack(codes, which)
            for i, slot in enumerate(slots[live].tolist()):
                exp[which][slot // page, h, slot % page] = packed[i]
                exp[2 + which][slot // page, h, slot % page] = torch.stack([s[i], low[i]])
            values = want.nibble_values(packed, torch.stack([s, low], 1), which)
            got = back[which].cpu()[live][:, h]
            # the sum of a number of 11 (8) bits and one of 15 is rounded to 24 bits and from there to the type
            assert torch.equal(got.isnan(), values.isnan())
            off = (got.double() - values).abs()
            off, size = off[~values.isnan()], values[~values.isnan()].abs()
            assert (off <= size * want.HALF_STEP[dtype] + 2.0 ** -24 * 2 * size + 2.0 ** -25).all()
    for a, b in zip(pool.codes + pool.scales, exp):
        a = a.cpu()
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())
    assert (back[:, ~live] == 7.0).all()


def test_codes_are_ordered_and_error_is_half_a_scale():
    dtype = torch.float16
    fused, k, v = rows_like(9, 64, 4, dtype)
    pool = Pool(4, 16, 4, 32, dtype)
    slots = torch.arange(64, dtype=torch.int32, device=DEV)
    write(pool, fused, 0, slots)
    back = torch.empty(2, 64, 4, 128, dtype=dtype, device=DEV)
    lib().fd_nibble_read(pool.handle(), slots.data_ptr(), 64, back[0].data_ptr(), 512, back[1].data_ptr(), 512,
                      torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for x, y in ((k, back[0].cpu()), (v, back[1].cpu())):
        g = x.double().reshape(64, 4, 4, 32)
        span = g.amax(-1) - g.amin(-1)
        off = (g - y.double().reshape(64, 4, 4, 32)).abs().amax(-1)
        # half a step; the stored scale is off by 2^-11 of itself (15 times that at the far end), the value read by 2^-11
        assert (off <= span / 30 + 2.0 ** -11 * (span + g.abs().amax(-1)) + 1e-7).all()


def filled(dtype, group, batch, hkv, page, lens, seed, width, spread=1.0):
    """A pool whose rows in use hold coded numbers, the others garbage; its block table, with garbage for the pages without tokens."""
    rng = np.random.default_rng(seed)
    n_pages = sum(-(-n // page) for n in lens) + 2
    pool = Pool(n_pages, page, hkv, group, dtype, seed)
    order = rng.permutation(n_pages)
    table = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (batch, width))).to(torch.int32)
    at = 0
    groups = 128 // group
    g = torch.Generator().manual_seed(seed)
    scales = [x.cpu() for x in pool.scales]
    for b, n in enumerate(lens):
        for j in range(-(-n // page)):
            pg = int(order[at])
            at += 1
            table[b, j] = pg
            rows = min(page, n - j * page)
            for x in scales:
                s = spread * (0.2 + 0.15 * torch.rand(hkv, rows, groups, generator=g))
                x[pg, :, :rows, 0] = s.to(dtype)
                x[pg, :, :rows, 1] = (-7.5 * s + 0.3 * torch.randn(hkv, rows, groups, generator=g)).to(dtype)
    pool.scales = [x.to(DEV) for x in scales]
    return pool, table


def tolerance(dtype, q, k, v, sk, sv, scale, exp):
    """What the arithmetic may be off by, per output element.  A score is a sum of 128 products (16 + c) q in fp32 and 8 more with the scales: at most 160
    roundings of 2^-24, each of a partial sum of at most sum |q| (31 s + |l|), l within |k| + 15 s, with s the largest of K's (sk); a weight carries twice that (it and the sum) and 2^-21 of its own
    exponential.  Weights times s (V's, sv) are 16 (bf16) or 22 bits, times (16 + c) <= 31 of them; sums of (keys / 32 + 16) terms in fp32.  One rounding at the end."""
    dx = 160 * 2.0 ** -24 * abs(scale) * q.abs().sum(-1).max() * (46 * sk + k.abs().max())
    part = 2.0 ** -17 if dtype == torch.bfloat16 else 2.0 ** -22
    weights = 2 * dx + 2.0 ** -21
    sums = (part + 2.0 ** -24 * (len(k) / 32 + 16)) * (62 * sv + v.abs().max())
    return exp.abs() * want.HALF_STEP[dtype] * 1.01 + weights * v.abs().max() * 2 + sums + 2.0 ** -25


def attend(pool, table, lens, q, chunk, max_seq, scale, out=None, ws=None, stream=None):
    fd = lib()
    batch, hq = q.shape[:2]
    shape = fd.make_shape(batch, hq, pool.hkv, 128, max_seq, chunk, scale)
    nbytes = fd.fd_nibble_workspace_bytes(shape)
    assert nbytes > 0
    if ws is None:
        ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device=DEV)        # NaN wherever it is not written
        fd.fd_cache_workspace_init(ws.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream)
    out = torch.full((batch + 1, hq, 128), float("nan"), dtype=pool.dtype, device=DEV) if out is None else out
    fd.fd_decode_attn_nibble(shape, pool.handle(), q.data_ptr(), table.data_ptr(), lens.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel(),
                          (stream or torch.cuda.current_stream()).cuda_stream)
    return out


def check(got, pool, table, lens, q, scale):
    hq = q.shape[1]
    share = hq // pool.hkv
    q = q.cpu()
    for b, n in enumerate(lens):
        for h in range(pool.hkv):
            rows = [want.gather(x.cpu(), table[b], n, pool.page, h) for x in (pool.codes[0], pool.scales[0], pool.codes[1], pool.scales[1])]
            k, v = want.nibble_values(rows[0], rows[1], 0), want.nibble_values(rows[2], rows[3], 1)
            qh = q[b, h * share:(h + 1) * share]
            exp = want.attend(qh, k, v, scale)
            x = got[b, h * share:(h + 1) * share].cpu().double()
            if n == 0:
                assert (x == 0).all()
                continue
            sk, sv = (float(rows[i][:, 0].double().max()) for i in (1, 3))
            tol = tolerance(pool.dtype, qh.double(), k, v, sk, sv, scale, exp)
            off = (x - exp).abs()
            assert torch.isfinite(x).all() and (off <= tol).all(), "sequence %d (%d keys), KV head %d: %.3g of %.3g" % (
                b, n, h, float((off / tol).max()), 1.0)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (8, 2), (6, 1), (9, 1), (16, 1), (24, 1), (40, 1)])
def test_heads(dtype, group, hq, hkv):
    lens, page, max_seq = [1, 0, 200, 77], 16, 224
    pool, table = filled(dtype, group, len(lens), hkv, page, lens, hq, max_seq // page)
    q = torch.randn(len(lens), hq, 128, generator=torch.Generator().manual_seed(hq)).to(dtype).to(DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    scale = 1 / math.sqrt(128)
    got = attend(pool, table.to(DEV), dl, q, 64, max_seq, scale)
    torch.cuda.synchronize()
    check(got, pool, table, lens, q, scale)
    assert got[-1].isnan().all()


@pytest.mark.parametrize("page", [16, 32, 64, 512])
@pytest.mark.parametrize("chunk", [64, 128, 320, 1024, 4096])
def test_lengths_pages_and_chunks(page, chunk):
    lens = [1, 15, 16, 17, 63, 64, 65, 255, 256, 257, 700, 1023, 0, 1024, 5000, -3]       # the last two are out of range
    max_seq = 1024
    used = [min(max(n, 0), max_seq) for n in lens]
    pool, table = filled(torch.float16, 64, len(lens), 2, page, used, page + chunk, max_seq // page)
    q = torch.randn(len(lens), 8, 128, generator=torch.Generator().manual_seed(1)).half().to(DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    got = attend(pool, table.to(DEV), dl, q, chunk, max_seq, 0.09)
    torch.cuda.synchronize()
    check(got, pool, table, used, q, 0.09)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
def test_picked_chunks_and_many_rows(dtype):
    lens = [3000, 1, 2999, 1500]
    pool, table = filled(dtype, 32, 4, 4, 64, lens, 5, 47)
    q = torch.randn(4, 28, 128, generator=torch.Generator().manual_seed(2)).to(dtype).to(DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    shape = lib().make_shape(4, 28, 4, 128, 47 * 64, 0, 0.1)
    chunk = lib().fd_nibble_pick_chunk(shape)
    assert chunk % 64 == 0 and chunk >= 64
    got = attend(pool, table.to(DEV), dl, q, chunk, 47 * 64, 0.1)
    torch.cuda.synchronize()
    check(got, pool, table, lens, q, 0.1)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
def test_large_logits_and_growing_maxima(dtype):
    """Queries 30 times larger: weights down to nothing, maxima that grow along the row."""
    lens, max_seq = [900, 640], 960
    pool, table = filled(dtype, 128, 2, 1, 32, lens, 8, max_seq // 32)
    q = (30 * torch.randn(2, 5, 128, generator=torch.Generator().manual_seed(3))).to(dtype).to(DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for chunk in (64, 256, 1024):
        got = attend(pool, table.to(DEV), dl, q, chunk, max_seq, 0.1)
        torch.cuda.synchronize()
        check(got, pool, table, lens, q, 0.1)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
def test_scales_of_v_as_large_as_the_type_allows(dtype):
    """Weights times scales near the end of fp16, with maxima that grow a little at a time."""
    lens, max_seq = [2000, 999], 2048
    pool, table = filled(dtype, 32, 2, 2, 64, lens, 12, max_seq // 64)
    pool.scales[1] *= 2.0 ** 14
    assert float(pool.scales[1].float().nan_to_num().abs().max()) > 40000
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for size in (1.0, 2.0, 4.0):
        q = (size * torch.randn(2, 8, 128, generator=torch.Generator().manual_seed(int(size)))).to(dtype).to(DEV)
        got = attend(pool, table.to(DEV), dl, q, 4096, max_seq, 0.05)
        torch.cuda.synchronize()
        check(got, pool, table, lens, q, 0.05)


@pytest.mark.parametrize("scale", [0.0, -0.08])
def test_scales_of_zero_and_below(scale):
    lens, max_seq = [300, 1, 65], 320
    pool, table = filled(torch.bfloat16, 64, 3, 2, 16, lens, 13, max_seq // 16)
    q = torch.randn(3, 6, 128, generator=torch.Generator().manual_seed(8)).bfloat16().to(DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for chunk in (64, 1024):
        got = attend(pool, table.to(DEV), dl, q, chunk, max_seq, scale)
        torch.cuda.synchronize()
        check(got, pool, table, lens, q, scale)


def test_rows_of_many_chunks():
    """More chunks than the launch joins itself, and than the join reads at a time."""
    lens, max_seq = [12800, 4161, 63], 12800
    pool, table = filled(torch.float16, 32, 3, 1, 64, lens, 14, max_seq // 64)
    q = torch.randn(3, 2, 128, generator=torch.Generator().manual_seed(9)).half().to(DEV)
    got = attend(pool, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), q, 64, max_seq, 0.1)
    torch.cuda.synchronize()
    check(got, pool, table, lens, q, 0.1)


def test_groups_of_every_size_of_number():
    """Ranges from nothing to the largest of bf16: codes, scales and lowest values bit for bit."""
    g = torch.Generator().manual_seed(4)
    tokens = 64
    x = torch.randn(tokens, 2, 128, generator=g).double() * 10.0 ** torch.linspace(-41, 37, tokens).double()[:, None, None]
    x[0] = 0
    x[1, :, :32] = torch.finfo(torch.bfloat16).max * torch.tensor([-1.0, 1.0]).repeat(16)       # a range that is no number: reads as NaN
    x[2, :, 5] = -0.0
    x = x.to(torch.bfloat16)
    pool = Pool(4, 16, 1, 32, torch.bfloat16)
    dev, slots = x.to(DEV), torch.arange(tokens, dtype=torch.int32, device=DEV)
    write(pool, dev, 0, slots)
    torch.cuda.synchronize()
    for which in range(2):
        with np.errstate(all="ignore"):
            codes, s, low = want.nibble_code(x[:, which], 32)
        bad = torch.zeros_like(s, dtype=torch.bool)
        bad[1, 0] = True
        codes[1, :32] = 0
        packed = want.nibble_pack(codes, which)
        got, scales = pool.codes[which].cpu().reshape(tokens, 64), pool.scales[which].cpu().reshape(tokens, 2, 4)
        assert torch.equal(got, packed)
        assert scales[:, :, :][bad[:, None].expand(-1, 2, -1)].isnan().all()
        for i, e in enumerate((s, low)):
            assert torch.equal(scales[:, i][~bad], e[~bad])


def test_captured_rows_and_strides_beyond_32_bits():
    """A captured write and read follow the slots of each replay; two tokens 2^31 elements apart."""
    stride = 2 ** 31
    big = torch.empty(stride + 512, dtype=torch.float16, device=DEV)
    for t in range(2):
        big[t * stride:t * stride + 512] = torch.randn(512, generator=torch.Generator().manual_seed(t)).half().to(DEV)
    pool = Pool(4, 16, 2, 128, torch.float16)
    slots = torch.tensor([3, 40], dtype=torch.int32, device=DEV)
    back = torch.zeros(2, 2, 2, 128, dtype=torch.float16, device=DEV)
    handle, side, graph = pool.handle(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        s = torch.cuda.current_stream().cuda_stream
        lib().fd_nibble_write(handle, big.data_ptr(), stride, big[256:].data_ptr(), stride, 2, slots.data_ptr(), s)
        lib().fd_nibble_read(handle, slots.data_ptr(), 2, back[0].data_ptr(), 256, back[1].data_ptr(), 256, s)
    x = torch.stack([big[t * stride:t * stride + 512] for t in range(2)]).cpu().reshape(2, 2, 2, 128)      # [token, K or V, head]
    for where in ([3, 40], [63, 0], [-1, 17], [5, 6]):
        slots.copy_(torch.tensor(where, dtype=torch.int32))
        back.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for t, slot in enumerate(where):
            for which in range(2):
                if slot < 0:
                    assert (back[which, t] == 7).all()
                    continue
                codes, sc, low = want.nibble_code(x[t, which], 128)
                packed = want.nibble_pack(codes, which)
                assert torch.equal(pool.codes[which][slot // 16, :, slot % 16].cpu(), packed)
                values = want.nibble_values(packed, torch.stack([sc, low], 1), which)
                off = (back[which, t].cpu().double() - values).abs()
                assert (off <= values.abs() * (2.0 ** -11 + 2.0 ** -23) + 2.0 ** -25).all()


def test_pools_beyond_32_bits():
    page, hkv = 512, 8
    n_pages = (5 << 30) // (64 * hkv * page)                           # 5 GiB of codes, K and V each
    codes = [torch.empty(n_pages, hkv, page, 64, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = [torch.empty(n_pages, hkv, page, 2, 4, dtype=torch.float16, device=DEV) for _ in range(2)]
    pool = Pool(1, page, hkv, 32, torch.float16)
    pool.n_pages, pool.codes, pool.scales = n_pages, codes, scales
    lens, max_seq = [700, 30], 1024
    table = torch.tensor([[n_pages - 1, n_pages - 2], [n_pages - 3, -1]], dtype=torch.int32)
    slots = torch.tensor([int(table[b, t // page]) * page + t % page for b, n in enumerate(lens) for t in range(n)], dtype=torch.int32)
    x = torch.randn(sum(lens), 2 * hkv, 128, generator=torch.Generator().manual_seed(5)).half().to(DEV)
    write(pool, x, 0, slots.to(DEV))
    q = torch.randn(2, 16, 128, generator=torch.Generator().manual_seed(6)).half().to(DEV)
    got = attend(pool, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), q, 256, max_seq, 0.1)
    torch.cuda.synchronize()
    small = Pool(3, page, hkv, 32, torch.float16)
    small.codes, small.scales = [c[-3:].clone() for c in codes], [c[-3:].clone() for c in scales]
    small_table = torch.where(table < 0, table, table - (n_pages - 3))
    check(got, small, small_table, lens, q, 0.1)
    k, s, low = want.nibble_code(x[699:700, 3].cpu(), 32)               # sequence 0's last row of K, head 3
    assert torch.equal(codes[0][n_pages - 2, 3, 699 - 512].cpu(), want.nibble_pack(k, 0)[0])


def test_nan_stays_in_its_row():
    lens, max_seq = [300, 300], 320
    pool, table = filled(torch.float16, 32, 2, 2, 16, lens, 4, max_seq // 16)
    q = torch.randn(2, 4, 128, generator=torch.Generator().manual_seed(5)).half().to(DEV)
    dl = torch.tensor(lens, dtype=torch.int32, device=DEV)
    clean = attend(pool, table.to(DEV), dl, q, 128, max_seq, 0.1)
    pool.scales[0][int(table[0, 5]), 1, 3, 0, 2] = float("nan")
    got = attend(pool, table.to(DEV), dl, q, 128, max_seq, 0.1)
    torch.cuda.synchronize()
    assert got[0, 2:].isnan().all() and torch.equal(got[0, :2], clean[0, :2]) and torch.equal(got[1], clean[1])


def test_another_stream_and_replays():
    lens, max_seq = [500, 33, 511], 512
    pool, table = filled(torch.bfloat16, 64, 3, 2, 32, lens, 9, max_seq // 32)
    q = torch.randn(3, 16, 128, generator=torch.Generator().manual_seed(6)).bfloat16().to(DEV)
    dl, dt = torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV)
    eager = attend(pool, dt, dl, q, 128, max_seq, 0.1)
    torch.cuda.synchronize()
    out = torch.full_like(eager, float("nan"))
    shape = lib().make_shape(3, 16, 2, 128, max_seq, 128, 0.1)
    ws = torch.zeros(lib().fd_nibble_workspace_bytes(shape), dtype=torch.uint8, device=DEV)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        attend(pool, dt, dl, q, 128, max_seq, 0.1, out, ws)
    for i in range(4):
        out.fill_(float("nan"))
        dl.copy_(torch.tensor([n - i for n in lens], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        again = attend(pool, dt, dl, q, 128, max_seq, 0.1)
        torch.cuda.synchronize()
        assert torch.equal(out[:3], again[:3])
    assert not torch.equal(again[:3], eager[:3])
