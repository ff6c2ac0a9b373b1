"""Decode over the cache of 16 or 8 bits, cut by the sequences' lengths, where pieces are shorter than a chunk: as many as a row has places for their sums, and
nothing behind the workspace is written."""
import math

import pytest
import torch

from tests.kv_pool import TYPES, decode, filled, lib, workspace
from tests.test_gpu_kv_decode import check_all, device, queries

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


@pytest.mark.parametrize("dtype", TYPES, ids=["fp16", "bf16"])
@pytest.mark.parametrize("coded", [True, False], ids=["e4m3", "16"])
@pytest.mark.parametrize("chunk,lens", [
    (512, [640, 513, 1025, 1152, 512, 511, 1024, 1, 0, 897, 1151, 1152]),
    (192, [193, 385, 577, 1152, 192, 384, 576, 1, 0, 256, 257, 1152]),
    (448, [449, 897, 1152, 1152, 448, 896, 512, 640, 0, 128, 129, 1152]),
])
def test_pieces_shorter_than_a_chunk(dtype, coded, chunk, lens):
    hkv, width, fd = 12, 18, lib()
    batch, max_seq = len(lens), 64 * width
    assert batch * hkv <= 512 and batch * hkv * -(-max_seq // chunk) > 256
    pool, table, k, v = filled(dtype, coded, hkv, 64, lens, 83, width)
    q = queries(batch, hkv, dtype)
    table, dlens = device(lens, table)
    nbytes = fd.fd_kv_workspace_bytes(fd.make_shape(batch, hkv, hkv, 128, max_seq, chunk, SCALE))
    room = workspace(nbytes + 4096)
    out = decode(pool, table, dlens, q, chunk, max_seq, SCALE, room[:nbytes])
    check_all(out, pool, lens, q, k, v)
    assert (room[nbytes:] == 0xA5).all() and not room[:1 << 14].any()
