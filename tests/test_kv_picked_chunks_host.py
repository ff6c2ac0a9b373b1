"""Chunks that fd_kv_pick_chunk picks, at the largest shapes too: one that the call takes wherever it takes any."""
import pytest

from paper_2311_01282_amd import fdattn as fd


@pytest.mark.parametrize("batch", [1, 64, 65, 512, 4096])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (32, 8), (40, 1), (128, 8), (512, 512)])
def test_taken_where_any_is(batch, hq, hkv):
    for log in range(4, 31):
        shape = fd.make_shape(batch, hq, hkv, 128, 1 << log, 16384, 0.1)            # the fewest chunks
        possible = fd.fd_kv_workspace_bytes(shape) > 0
        shape.chunk = fd.fd_kv_pick_chunk(shape)
        assert shape.chunk % 64 == 0 and 64 <= shape.chunk <= 16384
        assert (fd.fd_kv_workspace_bytes(shape) > 0) == possible, (log, shape.chunk)


def test_as_before_where_the_launch_has_room():
    for batch, hq, hkv, max_seq, want in [(1, 32, 8, 1 << 20, 2048), (128, 32, 8, 131072, 2048), (65, 32, 8, 4096, 4096), (65, 32, 8, 4160, 1408), (32, 64, 8, 4096, 4096)]:
        assert fd.fd_kv_pick_chunk(fd.make_shape(batch, hq, hkv, 128, max_seq, 0, 0.1)) == want
