"""Shapes of prompts whose launch would have 2^32 threads and more are refused before anything is enqueued (the pointers are never followed)."""
import pytest

from paper_2311_01282_amd import fdattn as fd
from tests.test_small_caches_host import P, status


@pytest.mark.parametrize("batch,heads,max_seq", [(1, 1, 1 << 30), (1, 1, 1 << 28), (1, 2, (1 << 28) + 1), (3, 1, 1 << 28), (1, 4, 1 << 28), (1, 1, (1 << 28) - 127)])
def test_launches_that_are_too_large(batch, heads, max_seq):
    shape = fd.make_shape(batch, heads, heads, 192, max_seq, 0, 0.1)
    assert status(fd.fd_latent_prefill_attn, shape, fd.FD_F16, P, P, P, 64, P, P) == fd.FD_ERR_UNSUPPORTED
