"""Refusals of the calls over the paged cache of 16 or 8 bits: all of them come from the host before anything is enqueued, so they need no GPU (the
pointers are never followed)."""
import ctypes

import pytest

from paper_2311_01282_amd import fdattn as fd

P = 1 << 20                       # an address, aligned to everything
NULL, SHAPE, WORKSPACE, UNSUPPORTED = fd.FD_ERR_NULL, fd.FD_ERR_SHAPE, fd.FD_ERR_WORKSPACE, fd.FD_ERR_UNSUPPORTED
POOL = dict(k=P, v=P, k_scales=P, v_scales=P, n_pages=8, page_size=16, n_kv_heads=2, head_dim=128, store=fd.FD_E4M3, dtype=fd.FD_F16)
BAD_POOL = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(k_scales=None), NULL), (dict(v_scales=None), NULL), (dict(k=P + 8), SHAPE), (dict(v=P + 2), SHAPE),
    (dict(k_scales=P + 4), SHAPE), (dict(v_scales=P + 1), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 27), SHAPE), (dict(page_size=24), SHAPE),
    (dict(page_size=8), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=64), UNSUPPORTED), (dict(store=3), UNSUPPORTED),
    (dict(store=-1), UNSUPPORTED), (dict(dtype=fd.FD_E4M3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(store=fd.FD_BF16), UNSUPPORTED),
    (dict(n_kv_heads=65536), UNSUPPORTED),
]
ROWS = dict(k=P, k_stride=256, v=P, v_stride=256, n_tokens=4, slots=P)
BAD_ROWS = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(slots=None), NULL), (dict(k=P + 8), SHAPE), (dict(v=P + 2), SHAPE), (dict(slots=P + 2), SHAPE),
    (dict(n_tokens=1 << 26), UNSUPPORTED), (dict(k_stride=255), SHAPE), (dict(k_stride=260), SHAPE), (dict(v_stride=128), SHAPE),
    (dict(v_stride=-256), SHAPE), (dict(n_tokens=-1), SHAPE),
]


def status(call, *args):
    try:
        call(*args)
    except fd.FdError as e:
        return e.status
    return fd.FD_OK


def changed(base, **kw):
    return dict(base, **kw)


def write(pool, r):
    return status(fd.fd_kv_write, fd.make_kv_pool(**pool), r["k"], r["k_stride"], r["v"], r["v_stride"], r["n_tokens"], r["slots"])


def read(pool, r):
    return status(fd.fd_kv_read, fd.make_kv_pool(**pool), r["slots"], r["n_tokens"], r["k"], r["k_stride"], r["v"], r["v_stride"])


def none_of(name):
    return [0 if t in (ctypes.c_int32, ctypes.c_int64) else fd.Workspace(None, 0) if t is fd.Workspace else None for t in getattr(fd._lib, name).argtypes]


@pytest.mark.parametrize("call", [write, read])
def test_rows(call):
    for kw, want in BAD_POOL:
        assert call(changed(POOL, **kw), ROWS) == want, kw
    for kw, want in BAD_ROWS:
        assert call(POOL, changed(ROWS, **kw)) == want, kw
    for store in (fd.FD_E4M3, fd.FD_F16):
        assert call(changed(POOL, store=store), changed(ROWS, n_tokens=0)) == fd.FD_OK
    # 16 bits have no scales
    assert call(changed(POOL, store=fd.FD_F16, k_scales=None, v_scales=None), changed(ROWS, n_tokens=0)) == fd.FD_OK
    name = "fd_kv_" + call.__name__
    assert getattr(fd._lib, name)(*none_of(name)) == NULL


SHAPE_OK = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, max_seq=1024, chunk=256, scale=0.1)
BAD_SHAPE = [
    (dict(batch=-1), SHAPE), (dict(n_q_heads=0), SHAPE), (dict(n_q_heads=7), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(head_dim=0), SHAPE),
    (dict(max_seq=0), SHAPE), (dict(chunk=0), SHAPE), (dict(chunk=-64), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(head_dim=64), UNSUPPORTED), (dict(max_seq=(1 << 30) + 16), UNSUPPORTED),
    (dict(batch=1 << 20, max_seq=1 << 20), UNSUPPORTED), (dict(n_q_heads=4, n_kv_heads=4), SHAPE), (dict(max_seq=1000), SHAPE),
]
CALL = dict(q=P, table=P, lens=P, out=P, ws=P, ws_bytes=1 << 40)
BAD_CALL = [
    (dict(q=None), NULL), (dict(table=None), NULL), (dict(lens=None), NULL), (dict(out=None), NULL), (dict(q=P + 8), SHAPE), (dict(out=P + 2), SHAPE),
    (dict(table=P + 2), SHAPE), (dict(lens=P + 1), SHAPE), (dict(ws=None), WORKSPACE), (dict(ws=P + 128), WORKSPACE), (dict(ws_bytes=1 << 14), WORKSPACE),
]


def decode(shape, pool, c):
    return status(fd.fd_kv_decode_attn, fd.make_shape(**shape), fd.make_kv_pool(**pool), c["q"], c["table"], c["lens"], c["out"], c["ws"], c["ws_bytes"])


def prefill(shape, pool, c):
    c = dict(dict(q_stride=1024, n_tokens=600, starts=P), **c)
    return status(fd.fd_kv_prefill_attn, fd.make_shape(**shape), fd.make_kv_pool(**pool), c["q"], c["q_stride"], c["n_tokens"], c["starts"], c["table"],
                  c["lens"], c["out"], c["ws"], c["ws_bytes"])


@pytest.mark.parametrize("call", [decode, prefill])
def test_attention(call):
    for kw, want in BAD_POOL:
        # (more KV heads than the shape has, which is seen later, have a limit of their own)
        assert call(SHAPE_OK, changed(POOL, **kw), CALL) == want, kw
    for kw, want in BAD_SHAPE:
        assert call(changed(SHAPE_OK, **kw), POOL, CALL) == want, kw
    for kw, want in BAD_CALL:
        assert call(SHAPE_OK, POOL, changed(CALL, **kw)) == want, kw
    assert call(changed(SHAPE_OK, batch=0), POOL, CALL) == fd.FD_OK
    name = "fd_kv_%s_attn" % call.__name__
    assert getattr(fd._lib, name)(*none_of(name)) == NULL


def test_decode_chunks():
    for chunk in (96, 32, 16448):
        assert decode(changed(SHAPE_OK, chunk=chunk), POOL, CALL) == UNSUPPORTED


def test_packed_tokens():
    for kw, want in [(dict(starts=None), NULL), (dict(starts=P + 2), SHAPE), (dict(q_stride=1023), SHAPE), (dict(q_stride=1028), SHAPE), (dict(q_stride=512), SHAPE),
                     (dict(q_stride=-1024), SHAPE), (dict(n_tokens=-1), SHAPE), (dict(n_tokens=(1 << 31) - 1), UNSUPPORTED)]:
        assert prefill(SHAPE_OK, POOL, changed(CALL, **kw)) == want, kw
    assert prefill(SHAPE_OK, POOL, changed(CALL, n_tokens=0)) == fd.FD_OK
    # a long cache in small pieces: more workgroups than there may be
    assert prefill(changed(SHAPE_OK, max_seq=1 << 24, chunk=1), POOL, changed(CALL, n_tokens=1 << 16)) == UNSUPPORTED


@pytest.mark.parametrize("batch", [0, 1, 7, 64, 4096])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (32, 8), (28, 4), (40, 1), (128, 8)])
@pytest.mark.parametrize("max_seq", [16, 512, 1008, 32768, 1 << 20])
def test_picked_chunks_are_taken(batch, hq, hkv, max_seq):
    shape = fd.make_shape(batch, hq, hkv, 128, max_seq, 0, 0.1)
    shape.chunk = fd.fd_kv_pick_chunk(shape)
    assert shape.chunk % 64 == 0 and 64 <= shape.chunk <= 16384
    assert fd.fd_kv_workspace_bytes(shape) > 0 or batch * hq * -(-max_seq // shape.chunk) > 1 << 23
    if batch <= 64 and max_seq <= 32768:
        assert fd.fd_kv_workspace_bytes(shape) <= 1 << 28
    for tokens in (0, 1, batch, 1000, 100000):
        shape.chunk = fd.fd_kv_prefill_pick_chunk(shape, tokens)
        assert 1 <= shape.chunk <= max_seq
        nbytes = fd.fd_kv_prefill_workspace_bytes(shape, tokens)
        assert nbytes >= 1 << 14
        assert nbytes <= 1 << 28                                        # what a serving program can set aside


@pytest.mark.parametrize("hq,tokens", [(1, (1 << 23) + 1), (16 * 65535 + 1, 1)])
def test_cut_launches_stay_within_their_grid(hq, tokens):
    # the launch that joins pieces: a token's 16 heads a workgroup of 256 threads, fewer than 2^32 threads along x, 2^16 workgroups along y
    cut, whole = (fd.make_shape(1, hq, 1, 128, 4096, chunk, 0.1) for chunk in (2048, 4096))
    assert fd.fd_kv_prefill_workspace_bytes(cut, tokens) == 0
    assert fd.fd_kv_prefill_workspace_bytes(whole, tokens) > 0
    assert fd.fd_kv_prefill_pick_chunk(whole, tokens) == 4096
    assert fd.fd_kv_prefill_workspace_bytes(fd.make_shape(1, hq - 1, 1, 128, 4096, 2048, 0.1) if hq > 1 else cut, tokens - (hq == 1)) > 0


def test_queries_of_sizes_refuse_bad_shapes():
    for call in (fd.fd_kv_workspace_bytes, fd.fd_kv_pick_chunk):
        assert call(fd.make_shape(2, 8, 2, 64, 1024, 256, 0.1)) == 0
    for call in (fd.fd_kv_prefill_workspace_bytes, fd.fd_kv_prefill_pick_chunk):
        assert call(fd.make_shape(2, 8, 2, 64, 1024, 256, 0.1), 16) == 0
        assert call(fd.make_shape(2, 8, 2, 128, 1024, 256, 0.1), -1) == 0
    assert fd._lib.fd_kv_workspace_bytes(None) == 0 and fd._lib.fd_kv_pick_chunk(None) == 0
    assert fd._lib.fd_kv_prefill_workspace_bytes(None, 4) == 0 and fd._lib.fd_kv_prefill_pick_chunk(None, 4) == 0
