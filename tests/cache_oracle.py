"""Plain implementations, on the CPU and in 64 bits, of the calls around the smaller paged caches: loops over requests, rows and keys,
written from the definitions in the header and sharing nothing with the library."""
import numpy as np
import torch

HALF_STEP = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}     # a rounding, relative to the value


def page_tables(page, n_pages, width, max_tokens, cached, new, free, n_free, table):
    """(table, seq_lens, starts, slots, n_left), one request after the other."""
    table = [list(r) for r in table]
    n_free = min(max(n_free, 0), n_pages)
    at = taken = asked = 0
    lens, starts, slots = [], [], [-1] * max_tokens
    for b, (c, n) in enumerate(zip(cached, new)):
        c, n = min(max(c, 0), width * page), max(n, 0)
        starts.append(min(at, max_tokens))
        held, upto = -(-c // page), -(-(c + n) // page)
        served = c + n <= width * page and at + n <= max_tokens
        need = upto - held if served else 0
        asked += need
        if served and need:
            served = asked <= n_free
        if served and need:
            for j in range(held, upto):
                table[b][j] = free[n_free - 1 - (asked - need + j - held)]
            taken = asked
        if served:
            for t in range(n):
                entry = table[b][(c + t) // page]
                if 0 <= entry < n_pages:
                    slots[at + t] = entry * page + (c + t) % page
        lens.append(c + n if served else c)
        at += n
    starts.append(min(at, max_tokens))
    return table, lens, starts, slots, n_free - taken


def nibble_code(x, group):
    """Codes [rows, 128] (numbers 0 .. 15), scales and lowest values [rows, 128 / group] of rows x [rows, 128] of fp16 or bf16."""
    f = x.float().numpy().reshape(len(x), 128 // group, group)
    finite = np.isfinite(f).all(-1)
    f = np.where(finite[..., None], f, np.float32(0))
    low, high = f.min(-1), f.max(-1)
    step = torch.from_numpy((high - low) / np.float32(15)).to(x.dtype)
    s = step.float().numpy()[..., None]
    c = np.where(s > 0, np.clip(np.rint((f - low[..., None]) / np.where(s > 0, s, np.float32(1))), 0, 15), 0).astype(np.int64)
    nan = torch.tensor(float("nan"), dtype=x.dtype)
    bad = torch.from_numpy(~finite)
    return c.reshape(len(x), 128), torch.where(bad, nan, step), torch.where(bad, nan, torch.from_numpy(low).to(x.dtype))


def nibble_place(which):
    """(byte, half) of element d of a row: `which` 0 for K, 1 for V."""
    res = []
    for d in range(128):
        nibble = d if which else (4 * ((d % 32) // 8) + d // 32) * 8 + d % 8
        res.append((nibble // 2, nibble % 2))
    return res


def nibble_pack(codes, which):
    out = np.zeros((len(codes), 64), dtype=np.uint8)
    for d, (byte, half) in enumerate(nibble_place(which)):
        out[:, byte] |= (codes[:, d] << (4 * half)).astype(np.uint8)
    return torch.from_numpy(out)


def nibble_values(codes, scales, which):
    """64-bit values of rows codes [rows, 64] bytes, scales [rows, 2, groups]."""
    byte, half = (torch.tensor(x) for x in zip(*nibble_place(which)))
    c = ((codes[:, byte].to(torch.int64) >> (4 * half)) & 15).double()
    of = torch.arange(128) // (128 // scales.shape[-1])
    return scales[:, 1, of].double() + scales[:, 0, of].double() * c


def gather(pool, table, n, page, head=None):
    """The first n rows of a sequence: pool [pages, heads, page, ..] or, without heads, [pages, page, ..]."""
    rows = [pool[int(table[t // page])][t % page] if head is None else pool[int(table[t // page])][head][t % page] for t in range(n)]
    return torch.stack(rows) if n else pool.new_zeros((0,) + tuple(pool.shape[(2 if head is None else 3):]))


def attend(q, k, v, scale):
    """softmax(scale q k^T) v of q [heads, d], in 64 bits; zeros where there is no key."""
    if not len(k):
        return torch.zeros(len(q), v.shape[-1], dtype=torch.float64)
    return torch.softmax(scale * (q.double() @ k.double().t()), -1) @ v.double()
