"""The calls around a paged cache that keeps less than fp16 keys and values, as measurable cases.

``listed`` gives the fixed cases, ``draw`` more of the same ranges; ``prepare`` builds what the program
holds before the call, ``run`` is one pass (the framework's entry points where ``own`` is true, elementary
torch operations in 32 bits where it is not), ``exact`` the same result from the definition in 64 bits,
``work`` the bytes and operations the pass cannot do without.

Kinds of case
    tables   fd_page_tables: pages for a step's new tokens, the block table, the slot of every token
    kv4      fd_nibble_write + fd_nibble_read: K and V rows into the 4-bit cache and, as the values they stand for,
             out of it again
    attn4    fd_decode_attn_nibble: one query token a sequence over the paged 4-bit cache
    latent   fd_latent_write + fd_latent_decode_attn: a decode step over a paged cache of latent rows (the absorbed form)
    prompt   fd_latent_prefill_attn: all tokens of a batch of prompts, with the keys and values that the latent rows
             stand for (the expanded form)

The 4-bit cache.  A group of ``group`` neighbouring elements of a row (128 elements of one token and KV head)
shares a scale s and a lowest value l, both of the cache's type, and an element is l + s c with a code c of 0 .. 15:
l = min x, s = (max x - min x) / 15 rounded to the type, c = (x - l) / s rounded to nearest (ties to even), between
0 and 15; c = 0 where s is 0.  codes [n_pages, n_kv_heads, page, 64] bytes, the lower half of a byte first; scales
[n_pages, n_kv_heads, page, 2, 128 / group], the s of all groups and then the l.  V's codes lie in order; K's 16
words of eight elements lie transposed as a 4 x 4 matrix: elements 32 t + 8 c .. + 7 are word 4 c + t.
"""
import math

import torch

own = False

D = 128
LATENT, ROPE = 512, 64
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def listed():
    return [
        # A decode step of a few users: launch latency and nothing else.
        dict(name="tables_b8_step_p16", kind="tables", batch=8, page=16, max_cached=2000, max_new=1, short=False, lens_seed=1),
        # Prompts of many requests admitted at once, some of which find no page left: over half a million slots.
        dict(name="tables_b300_prompts_p64", kind="tables", batch=300, page=64, max_cached=500, max_new=4001, short=True, lens_seed=3),
        # The rows of one decode step.
        dict(name="kv4_t32_h8_g32_bf16", kind="kv4", tokens=32, hkv=8, page=64, group=32, dtype="bf16", padded=0),
        # The rows of a batch of prompts, cut out of a fused projection; the last slots are padding.
        dict(name="kv4_t16001_h8_g64_fp16", kind="kv4", tokens=16001, hkv=8, page=128, group=64, dtype="fp16", padded=37),
        # One user, a short conversation: latency.
        dict(name="attn4_b1_gqa32x8_1k_fp16", kind="attn4", batch=1, hq=32, hkv=8, min_len=1000, max_len=1000, page=16, group=32,
             dtype="fp16", lens_seed=4),
        # A KV head for each query head, ragged lengths, finest groups.
        dict(name="attn4_b16_h32_ragged4k_fp16", kind="attn4", batch=16, hq=32, hkv=32, min_len=512, max_len=4096, page=64, group=32,
             dtype="fp16", lens_seed=5),
        # Grouped heads at a full serving batch.
        dict(name="attn4_b32_gqa64x8_4k_bf16", kind="attn4", batch=32, hq=64, hkv=8, min_len=4096, max_len=4096, page=64, group=64,
             dtype="bf16", lens_seed=6),
        # Latent attention: one user, the heads of one of eight GPUs.
        dict(name="latent_b1_h16_2k_bf16", kind="latent", batch=1, heads=16, min_len=2001, max_len=2001, page=64, dtype="bf16", lens_seed=8),
        # A few long ragged sequences.
        dict(name="latent_b8_h32_ragged32k_fp16", kind="latent", batch=8, heads=32, min_len=3000, max_len=32768, page=64, dtype="fp16",
             lens_seed=9),
        # A serving batch with all heads on one GPU: as much arithmetic as memory traffic.
        dict(name="latent_b64_h128_4k_bf16", kind="latent", batch=64, heads=128, min_len=4096, max_len=4096, page=64, dtype="bf16",
             lens_seed=10),
        # A batch of ordinary prompts, the heads of one of eight GPUs.
        dict(name="prompt_b3_h16_ragged1k_bf16", kind="prompt", batch=3, heads=16, min_len=150, max_len=1000, dtype="bf16", lens_seed=11),
        # One long prompt of an odd length.
        dict(name="prompt_b1_h64_4001_fp16", kind="prompt", batch=1, heads=64, min_len=4001, max_len=4001, dtype="fp16", lens_seed=12),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    kind = rng.choice(["tables", "kv4", "attn4", "attn4", "latent", "latent", "prompt"])
    seed, page = rng.randrange(1 << 20), rng.choice([16, 32, 64, 128, 256])
    dtype = rng.choice(["fp16", "bf16"])
    if kind == "tables":
        batch = _log(rng, 1, 4096)
        return dict(kind=kind, batch=batch, page=page, max_cached=_log(rng, 1, 8000), max_new=_log(rng, 1, min(8000, 1000000 // batch)),
                    short=rng.random() < 0.3, lens_seed=seed)
    if kind == "kv4":
        tokens = _log(rng, 1, 16000)
        return dict(kind=kind, tokens=tokens, hkv=rng.choice([1, 2, 4, 5, 8]), page=page, group=rng.choice([32, 64, 128]), dtype=dtype,
                    padded=rng.randrange(0, tokens // 8 + 1))
    if kind == "attn4":
        hq, hkv = rng.choice([(8, 8), (16, 16), (32, 32), (32, 8), (64, 8), (28, 4), (40, 20), (16, 1), (24, 1), (8, 1)])
        max_len = _log(rng, 1, 32768)
        batch = _log(rng, 1, max(1, min(64, 1000000 // (max_len * hkv))))
        return dict(kind=kind, batch=batch, hq=hq, hkv=hkv, min_len=max(1, max_len // rng.choice([1, 2, 8])), max_len=max_len, page=page,
                    group=rng.choice([32, 64, 128]), dtype=dtype, lens_seed=seed)
    heads = rng.choice([8, 16, 20, 32, 40, 64, 128])
    if kind == "prompt":
        max_len = _log(rng, 1, 5000)
        batch = _log(rng, 1, max(1, min(16, 64 * 4001 ** 2 // (heads * max_len ** 2))))
        heads = min(heads, max(1, 64 * 4001 ** 2 // (batch * max_len ** 2)))
        return dict(kind=kind, batch=batch, heads=heads, min_len=max(1, max_len // rng.choice([1, 2, 8])), max_len=max_len, dtype=dtype, lens_seed=seed)
    max_len = _log(rng, 1, 32768)
    batch = _log(rng, 1, max(1, min(128, 64 * 4096 * 128 // (max_len * max(heads, 64)))))
    return dict(kind=kind, batch=batch, heads=heads, min_len=max(1, max_len // rng.choice([1, 2, 8])), max_len=max_len, page=page,
                dtype=dtype, lens_seed=seed)


def _lens(case):
    g = torch.Generator().manual_seed(case["lens_seed"])
    return torch.randint(case["min_len"], case["max_len"] + 1, (case["batch"],), generator=g, dtype=torch.int32)


def _step(case):
    """(cached, new, pages left) of a tables case: lengths from the case alone, so that `work` knows them."""
    g = torch.Generator().manual_seed(case["lens_seed"])
    cached = torch.randint(0, case["max_cached"] + 1, (case["batch"],), generator=g, dtype=torch.int32)
    new = torch.randint(0 if case["max_new"] > 1 else 1, case["max_new"] + 1, (case["batch"],), generator=g, dtype=torch.int32)
    page = case["page"]
    need = int(((cached + new + page - 1) // page - (cached + page - 1) // page).sum())
    return cached, new, (need * 3 // 4 if case["short"] else need + 5)


def _width(case):
    return -(-case["max_len"] // case["page"])


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device=dev).to(dtype)

    def table_of(batch, width, n_pages):
        return torch.randperm(n_pages, generator=g, device=dev)[:batch * width].to(torch.int32).view(batch, width)

    s = dict(case)
    kind, page = case["kind"], case.get("page")
    if kind == "tables":
        cached, new, n_free = _step(case)
        batch, width = case["batch"], -(-(case["max_cached"] + case["max_new"]) // page)
        held = (cached + page - 1) // page
        n_pages = int(held.sum()) + n_free
        order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
        table = torch.zeros(batch, width, dtype=torch.int32, device=dev)
        mine = torch.arange(width, device=dev)[None, :] < held.to(dev)[:, None]
        table[mine] = order[n_free:]
        max_tokens = int(new.sum()) + 3
        return dict(s, n_pages=n_pages, width=width, max_tokens=max_tokens, cached=cached.to(dev), new=new.to(dev),
                    free=torch.cat([order[:n_free], torch.zeros(n_pages - n_free, dtype=torch.int32, device=dev)]),
                    n_free=torch.tensor([n_free], dtype=torch.int32, device=dev), table=table,
                    seq_lens=torch.empty(batch, dtype=torch.int32, device=dev),
                    starts=torch.empty(batch + 1, dtype=torch.int32, device=dev),
                    slots=torch.empty(max_tokens, dtype=torch.int32, device=dev), n_left=torch.empty(1, dtype=torch.int32, device=dev))
    dtype = TYPES[case["dtype"]]
    if kind == "kv4":
        tokens, hkv = case["tokens"], case["hkv"]
        n_pages, per_row = -(-tokens // page) + 2, 2 * D // case["group"]
        # rows of a fused projection: two query heads a KV head in front, then the keys, then the values
        fused = randn(tokens, 4 * hkv, D, dtype=dtype)
        fused[:, 2 * hkv:3 * hkv] += 0.7 * randn(hkv, D, dtype=dtype)          # keys have means of their own by channel
        slots = torch.randperm(n_pages * page, generator=g, device=dev)[:tokens].to(torch.int32)
        slots[tokens - case["padded"]:] = -1
        pool = [torch.zeros(n_pages, hkv, page, n, dtype=t, device=dev) for n, t in ((64, torch.uint8), (per_row, dtype)) * 2]
        pool = [x.view(n_pages, hkv, page, 2, per_row // 2) if x.dtype == dtype else x for x in pool]
        return dict(s, n_pages=n_pages, k=fused[:, 2 * hkv:3 * hkv], v=fused[:, 3 * hkv:], slots=slots, pool=pool,
                    k_back=torch.zeros(tokens, hkv, D, dtype=dtype, device=dev), v_back=torch.zeros(tokens, hkv, D, dtype=dtype, device=dev))
    batch, lens = case["batch"], _lens(case).to(dev)
    if kind == "prompt":
        # token-major, as projections leave them: a head's query 128 + 64 elements, its key's 128 and value's 128 side by side, the
        # rotary part of the keys, which all heads share, at the end of the latent rows
        heads, n = case["heads"], case["max_len"]
        return dict(s, lens=lens, q=randn(batch, n, heads, D + ROPE, dtype=dtype), kv=randn(batch, n, heads, 2 * D, dtype=dtype),
                    rows=randn(batch, n, LATENT + ROPE, dtype=dtype), out=torch.empty(batch, n, heads, D, dtype=dtype, device=dev))
    width = _width(case)
    n_pages = batch * width + 3
    table = table_of(batch, width, n_pages)
    if kind == "attn4":
        hq, hkv, groups = case["hq"], case["hkv"], D // case["group"]
        pool = []
        for _ in range(2):
            pool.append(torch.randint(0, 256, (n_pages, hkv, page, 64), generator=g, device=dev, dtype=torch.uint8))
            spread = torch.rand(n_pages, hkv, page, 1, groups, generator=g, device=dev) * 0.15 + 0.2
            low = -7.5 * spread + 0.3 * torch.randn(n_pages, hkv, page, 1, groups, generator=g, device=dev)
            pool.append(torch.cat([spread, low], 3).to(dtype))
        ws = torch.zeros(batch * hq * (-(-width * page // 64)) * 1024 + (1 << 16), dtype=torch.uint8, device=dev)
        return dict(s, n_pages=n_pages, width=width, lens=lens, table=table, pool=pool, q=randn(batch, hq, D, dtype=dtype),
                    out=torch.empty(batch, hq, D, dtype=dtype, device=dev), ws=ws)
    heads = case["heads"]
    rows = torch.empty(n_pages, page, LATENT + ROPE, dtype=dtype, device=dev)
    rows.copy_(randn(n_pages, page, LATENT + ROPE))
    last = (lens - 1).long()
    slots = table.gather(1, (last // page)[:, None])[:, 0] * page + (last % page).to(torch.int32)
    new = randn(batch, LATENT + ROPE, dtype=dtype)                                # one projection's output: strided parts
    ws = torch.zeros(256 * heads * 4096 * 2 + (batch * heads * 4096 * 2) + (1 << 16), dtype=torch.uint8, device=dev)
    return dict(s, n_pages=n_pages, width=width, lens=lens, table=table, rows=rows, slots=slots, latent=new[:, :LATENT], rope=new[:, LATENT:],
                q_latent=randn(batch, heads, LATENT, dtype=dtype), q_rope=randn(batch, heads, ROPE, dtype=dtype),
                out=torch.empty(batch, heads, LATENT, dtype=dtype, device=dev), ws=ws)


# ---- the plain forms ----

def _plain_tables(s):
    page, width = s["page"], s["width"]
    cached, new = s["cached"].long(), s["new"].long()
    dev = cached.device
    held, upto = (cached + page - 1) // page, (cached + new + page - 1) // page
    ends = new.cumsum(0)
    fits = (cached + new <= width * page) & (ends <= s["max_tokens"])
    need = torch.where(fits, upto - held, 0)
    run_need = need.cumsum(0)
    n_free = s["n_free"].long()
    served = fits & ((need == 0) | (run_need <= n_free))
    taken = torch.where(run_need <= n_free, run_need, 0).max()
    s["n_left"].copy_((n_free - taken).int())
    s["seq_lens"].copy_(torch.where(served, cached + new, cached).int())
    s["starts"].copy_(torch.cat([torch.zeros_like(ends[:1]), ends]).clamp(max=s["max_tokens"]).int())
    # pages from the end of the list, in the order of the requests
    j = torch.arange(width, device=dev)[None, :]
    fresh = served[:, None] & (j >= held[:, None]) & (j < upto[:, None])
    at = n_free - 1 - ((run_need - need)[:, None] + j - held[:, None])
    s["table"].copy_(torch.where(fresh, s["free"][at.clamp(0, s["n_pages"] - 1)], s["table"]))
    t = torch.arange(s["max_tokens"], device=dev)
    b = torch.searchsorted(ends, t, right=True)
    inside = b < len(ends)
    b = b.clamp(max=len(ends) - 1)
    pos = cached[b] + t - (ends - new)[b]
    entry = s["table"][b, (pos // page).clamp(max=width - 1)].long()
    good = inside & served[b] & (entry >= 0) & (entry < s["n_pages"])
    s["slots"].copy_(torch.where(good, entry * page + pos % page, -1).int())
    return [s["table"], s["seq_lens"], s["starts"], s["slots"], s["n_left"]]


def _swap_words(x):
    return x.unflatten(-1, (4, 4, 8)).transpose(-2, -3).flatten(-3)


def _values(codes, scales, is_k):
    """32-bit values of rows of codes [.., 64] and scales [.., 2, groups]."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    if is_k:
        c = _swap_words(c)
    s = scales.float()
    g = s.shape[-1]
    return (c.float().unflatten(-1, (g, D // g)) * s[..., 0, :, None] + s[..., 1, :, None]).flatten(-2)


def _coded(x, group, is_k):
    x32 = x.float().unflatten(-1, (D // group, group))
    lo, hi = x32.amin(-1), x32.amax(-1)
    s = ((hi - lo) / 15).to(x.dtype)
    s32 = s.float()[..., None]
    c = torch.where(s32 > 0, torch.round((x32 - lo[..., None]) / s32).clamp(0, 15), 0.0).to(torch.uint8).flatten(-2)
    if is_k:
        c = _swap_words(c)
    c = c.unflatten(-1, (64, 2))
    return c[..., 0] | (c[..., 1] << 4), torch.stack([s, lo.to(x.dtype)], -2)


def _plain_kv4(s):
    slots = s["slots"].long()
    keep = slots >= 0
    page_of, row = slots[keep] // s["page"], slots[keep] % s["page"]
    for i, (x, back) in enumerate(((s["k"], s["k_back"]), (s["v"], s["v_back"]))):
        codes, scales = s["pool"][2 * i], s["pool"][2 * i + 1]
        codes[page_of, :, row], scales[page_of, :, row] = _coded(x[keep], s["group"], i == 0)
        back[keep] = _values(codes[page_of, :, row], scales[page_of, :, row], i == 0).to(back.dtype)
    return [s["k_back"], s["v_back"]]


def _sequences(pool, table):
    """[batch, heads, tokens, ..] of a pool [n_pages, heads, page, ..]."""
    return pool[table.long()].transpose(1, 2).flatten(2, 3)


def _plain_softmax(x, lens):
    x = torch.where(torch.arange(x.shape[-1], device=x.device) < lens.view(-1, 1, 1, 1), x, -math.inf)
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_attn4(s):
    k, v = (_values(_sequences(s["pool"][2 * i], s["table"]), _sequences(s["pool"][2 * i + 1], s["table"]), i == 0) for i in (0, 1))
    q = s["q"].float().unflatten(1, (s["hkv"], -1))
    p = _plain_softmax(torch.matmul(q, k.transpose(-1, -2)) * (1 / math.sqrt(D)), s["lens"])
    s["out"].copy_(torch.matmul(p, v).flatten(1, 2))
    return [s["out"]]


def _plain_latent(s):
    s["rows"].view(-1, LATENT + ROPE)[s["slots"].long()] = torch.cat([s["latent"], s["rope"]], -1)
    c = s["rows"][s["table"].long()].flatten(1, 2).float()
    q = torch.cat([s["q_latent"], s["q_rope"]], -1).float()
    p = _plain_softmax((torch.matmul(q, c.transpose(-1, -2)) * _latent_scale())[:, None], s["lens"])[:, 0]
    s["out"].copy_(torch.matmul(p, c[..., :LATENT]))
    return [s["out"], s["rows"]]


def _plain_prompt(s):
    n = s["max_len"]
    at = torch.arange(n, device=s["q"].device)
    hidden = at[None, :] > at[:, None]
    k = torch.cat([s["kv"][..., :D], s["rows"][:, :, None, LATENT:].expand(-1, -1, s["heads"], -1)], -1).float().permute(0, 2, 3, 1)
    x = torch.matmul(s["q"].float().transpose(1, 2), k).mul_(_latent_scale()).masked_fill_(hidden, -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    x = x.div_(x.sum(-1, keepdim=True))
    o = torch.matmul(x, s["kv"][..., D:].float().transpose(1, 2)).transpose(1, 2)
    s["out"].copy_(torch.where((at[None, :] < s["lens"][:, None])[:, :, None, None], o, 0.0))
    return [s["out"]]


def _latent_scale():
    return 1 / math.sqrt(D + ROPE)          # of the heads that the latent rows stand for: 128 elements and the rotary ones


# ---- the framework's calls ----

def _own(s):
    from paper_2311_01282_amd import fdattn as fd
    stream = torch.cuda.current_stream().cuda_stream
    kind, page = s["kind"], s.get("page")
    if kind == "tables":
        fd.fd_page_tables(s["batch"], page, s["n_pages"], s["width"], s["max_tokens"], s["cached"].data_ptr(), s["new"].data_ptr(),
                          s["free"].data_ptr(), s["n_free"].data_ptr(), s["table"].data_ptr(), s["seq_lens"].data_ptr(),
                          s["starts"].data_ptr(), s["slots"].data_ptr(), s["n_left"].data_ptr(), stream)
        return [s["table"], s["seq_lens"], s["starts"], s["slots"], s["n_left"]]
    dtype = fd.FD_F16 if s["dtype"] == "fp16" else fd.FD_BF16
    if kind == "prompt":
        shape = fd.make_shape(s["batch"], s["heads"], s["heads"], D + ROPE, s["max_len"], 0, _latent_scale())
        rope = s["rows"][..., LATENT:]
        fd.fd_latent_prefill_attn(shape, dtype, s["q"].data_ptr(), s["kv"].data_ptr(), rope.data_ptr(), rope.stride(1), s["lens"].data_ptr(),
                                  s["out"].data_ptr(), stream)
        return [s["out"]]
    if kind == "latent":
        pool = fd.make_latent_pool(s["rows"].data_ptr(), s["n_pages"], page, LATENT, ROPE, dtype)
        fd.fd_latent_write(pool, s["latent"].data_ptr(), s["latent"].stride(0), s["rope"].data_ptr(), s["rope"].stride(0), s["batch"],
                           s["slots"].data_ptr(), stream)
        shape = fd.make_shape(s["batch"], s["heads"], 1, LATENT + ROPE, s["width"] * page, 0, _latent_scale())
        shape.chunk = fd.fd_latent_pick_chunk(shape)
        fd.fd_latent_decode_attn(shape, pool, s["q_latent"].data_ptr(), s["q_rope"].data_ptr(), s["table"].data_ptr(), s["lens"].data_ptr(),
                                 s["out"].data_ptr(), s["ws"].data_ptr(), s["ws"].numel(), stream)
        return [s["out"], s["rows"]]
    pool = fd.make_nibble_pool(*[x.data_ptr() for x in s["pool"]], s["n_pages"], page, s["hkv"], D, s["group"], dtype)
    if kind == "kv4":
        fd.fd_nibble_write(pool, s["k"].data_ptr(), s["k"].stride(0), s["v"].data_ptr(), s["v"].stride(0), s["tokens"], s["slots"].data_ptr(), stream)
        fd.fd_nibble_read(pool, s["slots"].data_ptr(), s["tokens"], s["k_back"].data_ptr(), s["k_back"].stride(0), s["v_back"].data_ptr(),
                       s["v_back"].stride(0), stream)
        return [s["k_back"], s["v_back"]]
    shape = fd.make_shape(s["batch"], s["hq"], s["hkv"], D, s["width"] * page, 0, 1 / math.sqrt(D))
    shape.chunk = fd.fd_nibble_pick_chunk(shape)
    fd.fd_decode_attn_nibble(shape, pool, s["q"].data_ptr(), s["table"].data_ptr(), s["lens"].data_ptr(), s["out"].data_ptr(),
                          s["ws"].data_ptr(), s["ws"].numel(), stream)
    return [s["out"]]


def run(state):
    if own:
        return _own(state)
    return {"tables": _plain_tables, "kv4": _plain_kv4, "attn4": _plain_attn4, "latent": _plain_latent, "prompt": _plain_prompt}[state["kind"]](state)


def work(case):
    kind = case["kind"]
    if kind == "tables":
        cached, new, _ = _step(case)
        page = case["page"]
        tokens = int(new.sum())
        fresh = int(((cached + new + page - 1) // page - (cached + page - 1) // page).sum())
        # lengths in and out, starts, a held entry for each request, each fresh page's entry read and written, a slot for each token
        return {"bytes": 4 * (4 * case["batch"] + 2 + 2 * fresh + tokens + case["batch"]), "flops": 0}
    if kind == "kv4":
        rows = 2 * (case["tokens"] - case["padded"]) * case["hkv"]
        coded = 64 + 2 * 2 * (D // case["group"])
        return {"bytes": rows * (4 * D + 2 * coded) + 8 * case["tokens"], "flops": 8 * rows * D}
    keys, batch = int(_lens(case).sum()), case["batch"]
    if kind == "prompt":
        pairs = sum(n * (n + 1) // 2 for n in _lens(case).tolist())
        return {"bytes": 2 * keys * (case["heads"] * (D + ROPE + 2 * D) + ROPE) + 2 * batch * case["max_len"] * case["heads"] * D + 4 * batch,
                "flops": 2 * (2 * D + ROPE) * pairs * case["heads"]}
    table = 4 * batch + 4 * int(((_lens(case) + case["page"] - 1) // case["page"]).sum())
    if kind == "attn4":
        row = 64 + 2 * 2 * (D // case["group"])
        return {"bytes": 2 * keys * case["hkv"] * row + 4 * batch * case["hq"] * D + table, "flops": 4 * D * keys * case["hq"]}
    width, heads = LATENT + ROPE, case["heads"]
    # (the step's rows are read and written once; the attention's own rows include them)
    return {"bytes": 2 * keys * width + 4 * batch * width + 2 * batch * heads * (width + LATENT) + table + 4 * batch,
            "flops": 2 * (width + LATENT) * keys * heads}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    kind = case["kind"]
    if kind == "tables":
        return None
    s = prepare(case, seed)
    page = case.get("page")
    dev = torch.device("cuda:0")
    element = torch.arange(D, device=dev)
    # byte and half of a byte that hold element d of a K row and of a V row
    word_k = 4 * ((element % 32) // 8) + element // 32
    place = [(word_k * 4 + (element % 8) // 2, element % 2), (element // 2, element % 2)]

    def decoded(codes, scales, which):
        byte, half = place[which]
        code = (codes[..., byte].to(torch.int32) >> (4 * half)) & 15
        of = element // case["group"]
        return code.double() * scales[..., 0, :].double()[..., of] + scales[..., 1, :].double()[..., of]

    if kind == "kv4":
        dtype, live = TYPES[case["dtype"]], s["slots"] >= 0
        res = []
        for x in (s["k"], s["v"]):
            y = x.double().reshape(case["tokens"], case["hkv"], D // case["group"], case["group"])
            low = y.min(-1, keepdim=True).values
            step = ((y.max(-1, keepdim=True).values - low) / 15).to(dtype).double()
            code = torch.round((y - low) / torch.where(step > 0, step, 1.0)).clamp(0, 15)
            res.append((low + step * torch.where(step > 0, code, 0.0)).reshape(case["tokens"], case["hkv"], D) * live[:, None, None])
        return res
    out, lens = [], s["lens"].tolist()
    if kind == "attn4":
        share = case["hq"] // case["hkv"]
        for b, n in enumerate(lens):
            pages = s["table"][b, :-(-n // page)].long()
            rows = []
            for h in range(case["hkv"]):
                k, v = (decoded(s["pool"][2 * i][pages, h].reshape(-1, 64)[:n], s["pool"][2 * i + 1][pages, h].flatten(0, 1)[:n], i) for i in (0, 1))
                x = s["q"][b, h * share:(h + 1) * share].double() @ k.t() / D ** 0.5
                rows.append(torch.softmax(x, -1) @ v)
            out.append(torch.cat(rows))
        return [torch.stack(out)]
    if kind == "prompt":
        out = torch.zeros(case["batch"], case["max_len"], case["heads"], D, dtype=torch.float64, device=dev)
        for b, n in enumerate(lens):
            below = torch.ones(n, n, dtype=torch.bool, device=dev).tril()
            for h in range(case["heads"]):
                q, kv = s["q"][b, :n, h].double(), s["kv"][b, :n, h].double()
                x = (q[:, :D] @ kv[:, :D].t() + q[:, D:] @ s["rows"][b, :n, LATENT:].double().t()) / (D + ROPE) ** 0.5
                out[b, :n, h] = torch.softmax(torch.where(below, x, -math.inf), -1) @ kv[:, D:]
        return [out]
    for b, n in enumerate(lens):
        c = s["rows"][s["table"][b, :-(-n // page)].long()].flatten(0, 1)[:n].double()
        c[n - 1, :LATENT], c[n - 1, LATENT:] = s["latent"][b].double(), s["rope"][b].double()
        x = (s["q_latent"][b].double() @ c[:, :LATENT].t() + s["q_rope"][b].double() @ c[:, LATENT:].t()) / (D + ROPE) ** 0.5
        out.append(torch.softmax(x, -1) @ c[:, :LATENT])
    return [torch.stack(out), None]
