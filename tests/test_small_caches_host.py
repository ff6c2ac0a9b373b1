"""Refusals of the calls around the smaller paged caches: all of them come from the host before anything is enqueued, so they need no GPU
(the pointers are never followed)."""
import ctypes
import math

import pytest

from paper_2311_01282_amd import fdattn as fd

P = 1 << 20                       # an address, aligned to everything
F16, BF16 = fd.FD_F16, fd.FD_BF16
NULL, SHAPE, WORKSPACE, UNSUPPORTED = fd.FD_ERR_NULL, fd.FD_ERR_SHAPE, fd.FD_ERR_WORKSPACE, fd.FD_ERR_UNSUPPORTED


def status(call, *args):
    try:
        call(*args)
    except fd.FdError as e:
        return e.status
    return fd.FD_OK


def changed(base, **kw):
    out = dict(base)
    out.update(kw)
    return out


TABLES = dict(batch=4, page_size=16, n_pages=8, pages_per_seq=4, max_tokens=16, cached=P, new=P, free=P, n_free=P, table=P, lens=P, starts=P,
              slots=P, left=P)


@pytest.mark.parametrize("kw,want", [
    (dict(page_size=8), SHAPE), (dict(page_size=48), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=-16), SHAPE), (dict(n_pages=0), SHAPE),
    (dict(n_pages=1 << 27), SHAPE), (dict(pages_per_seq=0), SHAPE), (dict(pages_per_seq=1 << 27), SHAPE), (dict(batch=-1), SHAPE),
    (dict(max_tokens=-1), SHAPE), (dict(max_tokens=(1 << 30) + 1), UNSUPPORTED), (dict(cached=P + 2), SHAPE), (dict(slots=P + 1), SHAPE),
] + [({k: None}, NULL) for k in ("cached", "new", "free", "n_free", "table", "lens", "starts", "slots", "left")])
def test_page_tables(kw, want):
    assert status(fd.fd_page_tables, *changed(TABLES, **kw).values()) == want


NIBBLE = dict(k_codes=P, k_scales=P, v_codes=P, v_scales=P, n_pages=8, page_size=16, n_kv_heads=2, head_dim=128, group=32, dtype=F16)
BAD_NIBBLE = [
    (dict(k_codes=None), NULL), (dict(k_scales=None), NULL), (dict(v_codes=None), NULL), (dict(v_scales=None), NULL), (dict(v_codes=P + 8), SHAPE),
    (dict(k_scales=P + 4), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 27), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=8), SHAPE),
    (dict(n_kv_heads=0), SHAPE), (dict(head_dim=64), UNSUPPORTED), (dict(group=16), UNSUPPORTED), (dict(group=0), UNSUPPORTED),
    (dict(group=256), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
]
ROWS = dict(k=P, k_stride=256, v=P, v_stride=256, n_tokens=4, slots=P)
BAD_ROWS = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(slots=None), NULL), (dict(k=P + 8), SHAPE), (dict(v=P + 2), SHAPE), (dict(slots=P + 2), SHAPE),
    (dict(n_tokens=1 << 26), UNSUPPORTED),
    (dict(k_stride=255), SHAPE), (dict(k_stride=260), SHAPE), (dict(v_stride=128), SHAPE), (dict(v_stride=-256), SHAPE), (dict(n_tokens=-1), SHAPE),
]


def nibble_write(pool, r):
    return status(fd.fd_nibble_write, pool, r["k"], r["k_stride"], r["v"], r["v_stride"], r["n_tokens"], r["slots"])


def nibble_read(pool, r):
    return status(fd.fd_nibble_read, pool, r["slots"], r["n_tokens"], r["k"], r["k_stride"], r["v"], r["v_stride"])


@pytest.mark.parametrize("call", [nibble_write, nibble_read])
def test_nibble_rows(call):
    for kw, want in BAD_NIBBLE:
        assert call(fd.make_nibble_pool(**changed(NIBBLE, **kw)), ROWS) == want, kw
    for kw, want in BAD_ROWS:
        assert call(fd.make_nibble_pool(**NIBBLE), changed(ROWS, **kw)) == want, kw
    assert call(fd.make_nibble_pool(**NIBBLE), changed(ROWS, n_tokens=0)) == fd.FD_OK
    name = "fd_" + call.__name__
    none = [0 if t in (ctypes.c_int32, ctypes.c_int64) else None for t in getattr(fd._lib, name).argtypes]
    assert getattr(fd._lib, name)(*none) == NULL


SHAPE4 = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, max_seq=1024, chunk=256, scale=0.1)
CALL = dict(q=P, table=P, lens=P, out=P, ws=P)


def attn4(shape=SHAPE4, pool=NIBBLE, ws_bytes=None, **kw):
    sh = fd.make_shape(**shape)
    c = changed(CALL, **kw)
    n = fd.fd_nibble_workspace_bytes(sh) if ws_bytes is None else ws_bytes
    return status(fd.fd_decode_attn_nibble, sh, fd.make_nibble_pool(**pool), c["q"], c["table"], c["lens"], c["out"], c["ws"], n)


BAD_SHAPES = [
    (dict(batch=-1), SHAPE), (dict(n_q_heads=0), SHAPE), (dict(max_seq=0), SHAPE), (dict(chunk=0), SHAPE), (dict(chunk=-64), SHAPE),
    (dict(chunk=16385), UNSUPPORTED), (dict(chunk=32768), UNSUPPORTED), (dict(scale=math.inf), SHAPE), (dict(scale=math.nan), SHAPE),
    (dict(max_seq=1 << 30, batch=1 << 12), UNSUPPORTED), (dict(max_seq=(1 << 30) + 16, chunk=16384), UNSUPPORTED), (dict(batch=1 << 19), UNSUPPORTED),
]


def test_decode_attn_nibble():
    for kw, want in BAD_SHAPES + [(dict(n_q_heads=9), SHAPE), (dict(chunk=80), UNSUPPORTED), (dict(head_dim=64), UNSUPPORTED)]:
        assert attn4(changed(SHAPE4, **kw), ws_bytes=1 << 40) == want, kw
        assert fd.fd_nibble_workspace_bytes(fd.make_shape(**changed(SHAPE4, **kw))) == 0
    for kw, want in BAD_NIBBLE:
        assert attn4(pool=changed(NIBBLE, **kw)) == want, kw
    assert attn4(pool=changed(NIBBLE, n_kv_heads=4)) == SHAPE
    assert attn4(changed(SHAPE4, max_seq=1000)) == SHAPE                  # no multiple of the page
    for kw, want in [(dict(q=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(out=None), NULL), (dict(q=P + 8), SHAPE),
                     (dict(out=P + 4), SHAPE), (dict(table=P + 2), SHAPE), (dict(lens=P + 1), SHAPE), (dict(ws=None), WORKSPACE),
                     (dict(ws=P + 128), WORKSPACE)]:
        assert attn4(**kw) == want, kw
    assert attn4(ws_bytes=fd.fd_nibble_workspace_bytes(fd.make_shape(**SHAPE4)) - 1) == WORKSPACE
    assert attn4(changed(SHAPE4, batch=0)) == fd.FD_OK
    for kw in (dict(n_q_heads=9), dict(head_dim=64), dict(max_seq=0)):
        assert fd.fd_nibble_pick_chunk(fd.make_shape(**changed(SHAPE4, **kw))) == 0


LATENT = dict(rows=P, n_pages=8, page_size=16, latent_dim=512, rope_dim=64, dtype=BF16)
BAD_LATENT = [
    (dict(rows=None), NULL), (dict(rows=P + 8), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 27), SHAPE), (dict(page_size=8), SHAPE),
    (dict(page_size=40), SHAPE), (dict(latent_dim=0), SHAPE), (dict(latent_dim=256), UNSUPPORTED), (dict(rope_dim=32), UNSUPPORTED),
    (dict(dtype=2), UNSUPPORTED),
]


def latent_write(pool=LATENT, **kw):
    c = changed(dict(latent=P, ls=576, rope=P, rs=576, n=4, slots=P), **kw)
    return status(fd.fd_latent_write, fd.make_latent_pool(**pool), c["latent"], c["ls"], c["rope"], c["rs"], c["n"], c["slots"])


def test_latent_write():
    for kw, want in BAD_LATENT:
        assert latent_write(changed(LATENT, **kw)) == want, kw
    for kw, want in [(dict(latent=None), NULL), (dict(rope=None), NULL), (dict(slots=None), NULL), (dict(latent=P + 8), SHAPE), (dict(rope=P + 2), SHAPE),
                     (dict(slots=P + 2), SHAPE), (dict(ls=504), SHAPE), (dict(ls=516), SHAPE), (dict(rs=56), SHAPE), (dict(rs=68), SHAPE), (dict(n=-1), SHAPE),
                     (dict(n=(1 << 25) + 1), UNSUPPORTED)]:
        assert latent_write(**kw) == want, kw
    assert latent_write(n=0) == fd.FD_OK


SHAPE_L = dict(batch=2, n_q_heads=16, n_kv_heads=1, head_dim=576, max_seq=1024, chunk=256, scale=0.1)


def latent_attn(shape=SHAPE_L, pool=LATENT, ws_bytes=None, **kw):
    sh = fd.make_shape(**shape)
    c = changed(dict(ql=P, qr=P, table=P, lens=P, out=P, ws=P), **kw)
    n = fd.fd_latent_workspace_bytes(sh) if ws_bytes is None else ws_bytes
    return status(fd.fd_latent_decode_attn, sh, fd.make_latent_pool(**pool), c["ql"], c["qr"], c["table"], c["lens"], c["out"], c["ws"], n)


def test_latent_decode_attn():
    for kw, want in BAD_SHAPES + [(dict(chunk=96), UNSUPPORTED), (dict(head_dim=128), UNSUPPORTED), (dict(n_kv_heads=2), UNSUPPORTED)]:
        assert latent_attn(changed(SHAPE_L, **kw), ws_bytes=1 << 40) == want, kw
        assert fd.fd_latent_workspace_bytes(fd.make_shape(**changed(SHAPE_L, **kw))) == 0
    for kw, want in BAD_LATENT:
        assert latent_attn(pool=changed(LATENT, **kw)) == want, kw
    assert latent_attn(changed(SHAPE_L, max_seq=1000)) == SHAPE
    for kw, want in [(dict(ql=None), NULL), (dict(qr=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(out=None), NULL),
                     (dict(ql=P + 8), SHAPE), (dict(qr=P + 8), SHAPE), (dict(out=P + 4), SHAPE), (dict(table=P + 2), SHAPE), (dict(lens=P + 1), SHAPE),
                     (dict(ws=None), WORKSPACE), (dict(ws=P + 64), WORKSPACE)]:
        assert latent_attn(**kw) == want, kw
    assert latent_attn(ws_bytes=fd.fd_latent_workspace_bytes(fd.make_shape(**SHAPE_L)) - 1) == WORKSPACE
    assert latent_attn(changed(SHAPE_L, batch=0)) == fd.FD_OK
    assert fd.fd_latent_pick_chunk(fd.make_shape(**changed(SHAPE_L, n_kv_heads=2, n_q_heads=16))) == 0


SHAPE_P = dict(batch=2, n_q_heads=16, n_kv_heads=16, head_dim=192, max_seq=100, chunk=0, scale=0.1)


def test_latent_prefill_attn():
    def call(shape=SHAPE_P, **kw):
        c = changed(dict(dtype=F16, q=P, kv=P, rope=P, rs=576, lens=P, out=P), **kw)
        return status(fd.fd_latent_prefill_attn, fd.make_shape(**shape), *c.values())
    for kw, want in [(dict(batch=-1), SHAPE), (dict(n_q_heads=0), SHAPE), (dict(max_seq=0), SHAPE), (dict(head_dim=128), UNSUPPORTED),
                     (dict(n_kv_heads=8), UNSUPPORTED), (dict(scale=math.nan), SHAPE), (dict(n_q_heads=65536, n_kv_heads=65536), UNSUPPORTED),
                     (dict(batch=1 << 20, max_seq=1 << 20), UNSUPPORTED), (dict(max_seq=(1 << 30) + 1), UNSUPPORTED)]:
        assert call(changed(SHAPE_P, **kw)) == want, kw
    for kw, want in [(dict(dtype=2), UNSUPPORTED), (dict(q=None), NULL), (dict(kv=None), NULL), (dict(rope=None), NULL), (dict(lens=None), NULL),
                     (dict(out=None), NULL), (dict(q=P + 8), SHAPE), (dict(kv=P + 8), SHAPE), (dict(rope=P + 8), SHAPE), (dict(out=P + 8), SHAPE),
                     (dict(lens=P + 2), SHAPE), (dict(rs=56), SHAPE), (dict(rs=68), SHAPE), (dict(rs=(1 << 24) + 8), SHAPE), (dict(rs=-576), SHAPE)]:
        assert call(**kw) == want, kw
    assert call(changed(SHAPE_P, batch=0)) == fd.FD_OK


def test_workspace_init():
    init = lambda ptr, n: status(fd.fd_cache_workspace_init, ptr, n)      # noqa: E731
    assert init(None, 1 << 20) == WORKSPACE and init(P + 128, 1 << 20) == WORKSPACE and init(P, 4 * 4096 - 1) == WORKSPACE


def test_workspaces_grow_with_the_split():
    a, b = (fd.fd_nibble_workspace_bytes(fd.make_shape(**changed(SHAPE4, chunk=c))) for c in (1024, 64))
    assert 0 < a <= b and b >= 2 * 8 * 16 * (128 + 2) * 4
    a, b = (fd.fd_latent_workspace_bytes(fd.make_shape(**changed(SHAPE_L, chunk=c))) for c in (1024, 64))
    assert 0 < a <= b and b >= 2 * 16 * 16 * (512 + 2) * 4


@pytest.mark.parametrize("batch", [1, 3, 8, 64, 300])
@pytest.mark.parametrize("max_seq", [16, 48, 1008, 4096, 32768, 1 << 20])
def test_picked_chunks_are_accepted(batch, max_seq):
    for hq, hkv in ((1, 1), (32, 32), (64, 8), (40, 1)):
        sh = fd.make_shape(batch, hq, hkv, 128, max_seq, 0, 0.1)
        sh.chunk = fd.fd_nibble_pick_chunk(sh)
        assert fd.fd_nibble_workspace_bytes(sh) > 0
    for h in (1, 16, 64, 65, 128, 200):
        sh = fd.make_shape(batch, h, 1, 576, max_seq, 0, 0.1)
        sh.chunk = fd.fd_latent_pick_chunk(sh)
        assert fd.fd_latent_workspace_bytes(sh) > 0
