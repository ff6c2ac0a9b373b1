"""fd_page_tables refuses outputs that share memory with another of its arrays: its workgroups read and write them at different times.  On the host, before anything is enqueued
(the pointers are never followed)."""
import pytest

from paper_2311_01282_amd import fdattn as fd
from tests.test_small_caches_host import status

BATCH, WIDTH, PAGES, TOKENS = 6, 5, 40, 30
SIZES = dict(cached=BATCH, new=BATCH, free=PAGES, n_free=1, table=BATCH * WIDTH, lens=BATCH, starts=BATCH + 1, slots=TOKENS, left=1)
INPUTS = ("cached", "new", "free", "n_free")
PAIRS = [(a, b) for i, a in enumerate(SIZES) for b in list(SIZES)[:i] if a not in INPUTS]


def call(at):
    return status(fd.fd_page_tables, BATCH, 16, PAGES, WIDTH, TOKENS, *at.values())


def apart():
    return {name: (1 << 20) + 4096 * i for i, name in enumerate(SIZES)}


@pytest.mark.parametrize("out,other", PAIRS, ids=lambda x: x)
def test_shared_arrays_are_refused(out, other):
    at = apart()
    at[out] = at[other]
    assert call(at) == fd.FD_ERR_SHAPE


@pytest.mark.parametrize("out,other", PAIRS, ids=lambda x: x)
def test_the_last_entry_of_one_and_the_first_of_the_other(out, other):
    for first, second in ((out, other), (other, out)):
        at = apart()
        at[second] = at[first] + 4 * (SIZES[first] - 1)
        assert call(at) == fd.FD_ERR_SHAPE
