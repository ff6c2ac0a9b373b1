"""Test-side plumbing of the paged cache of 16 or 8 bits: pools on the GPU whose rows in use hold numbers and all others garbage."""
import numpy as np
import torch

from tests import close_bounds as close
from tests import kv_oracle as want

DEV = "cuda:0"
TYPES = [torch.float16, torch.bfloat16]


def lib():
    from paper_2311_01282_amd import fdattn
    return fdattn


def stream():
    return torch.cuda.current_stream().cuda_stream


def of(dtype):
    return lib().FD_F16 if dtype == torch.float16 else lib().FD_BF16


class Pool:
    """rows[which], scales[which] (8 bits): NaN and garbage to begin with."""

    def __init__(self, n_pages, page, hkv, dtype, coded, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.n_pages, self.page, self.hkv, self.dtype, self.coded = n_pages, page, hkv, dtype, coded
        if coded:
            self.rows = [torch.randint(0, 256, (n_pages, hkv, page, 128), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2)]
            self.scales = [torch.randint(0, 256, (n_pages, hkv, page), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2)]
        else:
            self.rows = [torch.full((n_pages, hkv, page, 128), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
            self.scales = [None, None]

    def handle(self):
        ptr = [None if x is None else x.data_ptr() for x in self.rows + self.scales]
        store = lib().FD_E4M3 if self.coded else of(self.dtype)
        return lib().make_kv_pool(*ptr, self.n_pages, self.page, self.hkv, 128, store, of(self.dtype))


def filled(dtype, coded, hkv, page, lens, seed, width, size=1.0, change=None):
    """(pool, table, keys, values): a pool whose rows in use hold numbers; its block table, with garbage for the pages without tokens;
    the rows of every sequence as 64-bit numbers [hkv, L, 128].  change(b, which, x): the rows [hkv, L, 128] of a sequence before
    they are put there."""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    n_pages = sum(-(-n // page) for n in lens) + 2
    pool = Pool(n_pages, page, hkv, dtype, coded, seed)
    rows, scales = [x.cpu() for x in pool.rows], [None if x is None else x.cpu() for x in pool.scales]
    order, at = rng.permutation(n_pages), 0
    table = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (len(lens), width))).to(torch.int32)
    numbers = [[], []]
    for b, n in enumerate(lens):
        pages = order[at:at + -(-n // page)]
        at += len(pages)
        table[b, :len(pages)] = torch.from_numpy(pages.astype(np.int32))
        for which in range(2):
            x = (size * torch.randn(hkv, n, 128, generator=g)).to(dtype)
            if change is not None:
                x = change(b, which, x).to(dtype)
            if coded:
                c = torch.empty(hkv, n, 128, dtype=torch.uint8)
                s = torch.empty(hkv, n, dtype=torch.uint8)
                for h in range(hkv):
                    bad = ~torch.isfinite(x[h]).all(-1)
                    ok = torch.where(bad[:, None], 0.0, x[h]).double()
                    e = torch.ceil(torch.log2(ok.abs().amax(-1).clamp(min=2.0 ** -100) / 448))
                    c[h] = (ok * torch.exp2(-e)[:, None]).float().to(torch.float8_e4m3fn).view(torch.uint8)
                    c[h][bad] = 127
                    s[h] = torch.where(bad, 255.0, e + 127).to(torch.uint8)
                numbers[which].append(want.values(c, s))
            else:
                numbers[which].append(x.double())
            for j, pg in enumerate(pages):
                m = min(page, n - j * page)
                rows[which][pg, :, :m] = (c if coded else x)[:, j * page:j * page + m]
                if coded:
                    scales[which][pg, :, :m] = s[:, j * page:j * page + m]
    pool.rows = [x.to(DEV) for x in rows]
    pool.scales = [None if x is None else x.to(DEV) for x in scales]
    return pool, table, numbers[0], numbers[1]


def workspace(nbytes, fill=0xA5):
    """Garbage but for the arrival counters, which begin it."""
    ws = torch.full((max(nbytes, 1 << 14),), fill, dtype=torch.uint8, device=DEV)
    lib().fd_cache_workspace_init(ws.data_ptr(), ws.numel(), stream())
    return ws


def decode(pool, table, lens, q, chunk, max_seq, scale, ws=None, out=None):
    """table, lens and q on the GPU."""
    fd, (batch, hq, _) = lib(), q.shape
    shape = fd.make_shape(batch, hq, pool.hkv, 128, max_seq, chunk, scale)
    if chunk == 0:
        shape.chunk = fd.fd_kv_pick_chunk(shape)
    if ws is None:
        ws = workspace(fd.fd_kv_workspace_bytes(shape))
    if out is None:
        out = torch.full_like(q, float("nan"))
    fd.fd_kv_decode_attn(shape, pool.handle(), q.data_ptr(), table.data_ptr(), lens.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel(), stream())
    return out


def prefill(pool, table, lens, starts, q, chunk, max_seq, scale, ws=None, out=None):
    """q [tokens, hq, 128], its tokens apart by any stride."""
    fd, (tokens, hq, _) = lib(), q.shape
    shape = fd.make_shape(len(lens), hq, pool.hkv, 128, max_seq, chunk, scale)
    if chunk == 0:
        shape.chunk = fd.fd_kv_prefill_pick_chunk(shape, tokens)
    if ws is None:
        ws = workspace(fd.fd_kv_prefill_workspace_bytes(shape, tokens))
    if out is None:
        out = torch.full((tokens, hq, 128), 7.0, dtype=q.dtype, device=DEV)
    fd.fd_kv_prefill_attn(shape, pool.handle(), q.data_ptr(), q.stride(0), tokens, starts.data_ptr(), table.data_ptr(), lens.data_ptr(),
                          out.data_ptr(), ws.data_ptr(), ws.numel(), stream())
    return out


def check(got, dtype, parts, q, k, v, scale, visible=None, what=""):
    """got, q [rows, 128] of one KV head, k, v [keys, 128] in 64 bits; visible [rows, keys].

    Scores are fp32 sums of exact products whose partial sums stay within |q| |k|; a weight enters as `parts` numbers of the type: the bound is that of
    the other 16-bit attention over rows as they are."""
    if visible is not None:
        some = visible.any(-1)
        assert (got[~some] == 0).all(), what + ": rows without a key"
        got, q, visible = got[some], q[some], visible[some]
    if not len(got):
        return
    exp, tol = close.latent(dtype, parts, q.double(), k, v, scale, visible)
    off = (got.double() - exp).abs()
    assert (off <= tol).all(), "%s: %.3g of the bound" % (what, float((off / tol).max()))
