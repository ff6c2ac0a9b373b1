"""Rows into the paged cache of 16 or 8 bits and out of it again, bit for bit."""
import pytest
import torch

from tests import kv_oracle as want
from tests.kv_pool import DEV, TYPES, Pool, lib, stream

pytestmark = pytest.mark.gpu


def rows_like(seed, tokens, hkv, dtype, extra=0):
    """Rows of a fused projection, K and V at its end, of very different sizes."""
    g = torch.Generator().manual_seed(seed)
    fused = torch.randn(tokens, extra + 2 * hkv, 128, generator=g)
    far = 4 if dtype == torch.float16 else 36
    fused *= 10.0 ** torch.randint(-far, far, (tokens, extra + 2 * hkv, 1), generator=g)
    return fused.to(dtype)


def write(pool, fused, extra, slots):
    k, v = fused[:, extra:extra + pool.hkv], fused[:, extra + pool.hkv:]
    lib().fd_kv_write(pool.handle(), k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0), len(fused), slots.data_ptr(), stream())


def read(pool, slots, back):
    lib().fd_kv_read(pool.handle(), slots.data_ptr(), len(slots), back[0].data_ptr(), back[0].stride(0), back[1].data_ptr(), back[1].stride(0), stream())


SPECIAL = [0.0, -0.0, 448.0, 449.0, 464.0, -448.0, 0.5, 2.0 ** -10, 1.75, 1.7578125, -1.9375]


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])
@pytest.mark.parametrize("tokens,hkv,page,extra", [(1, 1, 16, 0), (5, 3, 16, 2), (77, 8, 64, 8), (150, 2, 32, 0)])
def test_rows_in_and_out(dtype, coded, tokens, hkv, page, extra):
    n_pages = -(-tokens // page) + 3
    fused = rows_like(tokens, tokens, hkv, dtype, extra)
    fused[0, extra] = 0.0                                               # a row of zeros
    if tokens > 4:
        last = torch.finfo(dtype)
        fused[1, extra, :len(SPECIAL)] = torch.tensor(SPECIAL, dtype=dtype)
        fused[1, extra, len(SPECIAL):] = 0.0
        fused[2, extra, 5], fused[2, extra + hkv, 90] = float("inf"), float("nan")
        fused[3, extra, 7], fused[3, extra, 8] = last.max, -last.max    # the type's largest
        fused[4, extra] = last.smallest_normal * 2.0 ** -3              # numbers below the normal ones
        fused[4, extra, 1] = last.smallest_normal * torch.finfo(dtype).eps
    pool = Pool(n_pages, page, hkv, dtype, coded)
    before = [None if x is None else x.clone().cpu() for x in pool.rows + pool.scales]
    g = torch.Generator().manual_seed(3)
    slots = torch.randperm(n_pages * page, generator=g)[:tokens].to(torch.int32)
    live = torch.ones(tokens, dtype=torch.bool)
    if tokens > 10:
        slots[7], slots[8], slots[9] = -1, n_pages * page, -2 ** 31     # padding, and slots behind the pool
        live[7:10] = False
    dev, dslots = fused.to(DEV), slots.to(DEV)
    write(pool, dev, extra, dslots)
    wide = torch.full((2, tokens, hkv + 1, 128), 7.0, dtype=dtype, device=DEV)      # a stride of its own
    read(pool, dslots, wide[:, :, :hkv])
    torch.cuda.synchronize()
    back = wide.cpu()
    assert (back[:, :, hkv] == 7.0).all() and (back[:, ~live] == 7.0).all()
    for which in range(2):
        x = fused[:, extra + which * hkv:extra + (which + 1) * hkv]
        rows, scales = before[which], before[2 + which]
        for t in range(tokens):
            if not live[t]:
                continue
            page_of, row = int(slots[t]) // page, int(slots[t]) % page
            for h in range(hkv):
                if coded:
                    c, byte = want.code_row(x[t, h])
                    rows[page_of, h, row], scales[page_of, h, row] = torch.from_numpy(c), byte
                    exp = want.values(torch.from_numpy(c), torch.tensor(byte))
                    got = back[which, t, h].double()
                    assert torch.equal(got.isnan(), exp.isnan()) and torch.equal(got.nan_to_num(), exp.nan_to_num()), (which, t, h)
                else:
                    rows[page_of, h, row] = x[t, h]
                    assert torch.equal(back[which, t, h].view(torch.int16), x[t, h].view(torch.int16))
        got = pool.rows[which].cpu()
        if coded:
            assert torch.equal(got, rows) and torch.equal(pool.scales[which].cpu(), scales)
        else:
            assert torch.equal(got.view(torch.int16), rows.view(torch.int16))


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
def test_error_is_half_a_step_of_four_bits(dtype):
    fused = rows_like(9, 64, 4, dtype)
    pool = Pool(4, 16, 4, dtype, True)
    slots = torch.arange(64, dtype=torch.int32, device=DEV)
    write(pool, fused.to(DEV), 0, slots)
    back = torch.empty(2, 64, 4, 128, dtype=dtype, device=DEV)
    read(pool, slots, back)
    torch.cuda.synchronize()
    for x, y in ((fused[:, :4], back[0].cpu()), (fused[:, 4:], back[1].cpu())):
        x, y = x.double(), y.double()
        top = x.abs().amax(-1, keepdim=True)
        # half a step of a normal code; of the others half of 2^-9, which is at most 2^-10 / 224 of the largest, or, where the scale is the
        # smallest, 2^-10 of that
        assert ((x - y).abs() <= torch.maximum(x.abs() * 2.0 ** -4, (top / 224).clamp(min=2.0 ** want.LOWEST) * 2.0 ** -10)).all()


def test_a_step_is_captured_and_replayed():
    dtype, tokens, hkv = torch.bfloat16, 33, 4
    pool = Pool(8, 16, hkv, dtype, True)
    x = torch.zeros(tokens, 2 * hkv, 128, dtype=dtype, device=DEV)
    slots = torch.arange(tokens, dtype=torch.int32, device=DEV)
    back = torch.empty(2, tokens, hkv, 128, dtype=dtype, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        write(pool, x, 0, slots)
        read(pool, slots, back)
    for seed in range(3):
        x.copy_(rows_like(seed, tokens, hkv, dtype).to(DEV))
        slots.copy_(torch.randperm(128, generator=torch.Generator().manual_seed(seed))[:tokens].to(torch.int32).to(DEV))
        back.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        replayed = back.clone()
        back.fill_(7.0)
        write(pool, x, 0, slots)
        read(pool, slots, back)
        torch.cuda.synchronize()
        assert torch.equal(back, replayed) and (back != 7.0).any()
