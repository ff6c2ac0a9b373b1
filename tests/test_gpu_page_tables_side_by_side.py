"""The arrays of fd_page_tables one right behind the other in one allocation, in either order: none of them overlap."""
import pytest
import torch

from tests import cache_oracle as want
from tests import test_gpu_page_tables as tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("turned", [False, True])
def test_side_by_side(turned):
    from paper_2311_01282_amd import fdattn
    page, n_pages, width, max_tokens, cached, new, free, n_free, table = c = tables.case(3, batch=50, page=16, max_cached=90, max_new=30, n_free=60, spare_tokens=3)
    values = [cached, new, list(free) + [0] * (n_pages - len(free)), [n_free], sum(table, []), [-7] * 50, [-7] * 51, [-7] * max_tokens, [-7]]
    order = list(range(9))[::-1] if turned else list(range(9))
    buffer = torch.cat([torch.tensor(values[i], dtype=torch.int32) for i in order]).to("cuda:0")
    at, start = {}, 0
    for i in order:
        at[i] = buffer[start:start + len(values[i])]
        start += len(values[i])
    fdattn.fd_page_tables(50, page, n_pages, width, max_tokens, *[at[i].data_ptr() for i in range(9)], torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    exp = want.page_tables(*c)
    assert (at[4].view(50, width).tolist(), *[at[i].tolist() for i in (5, 6, 7)], at[8].item()) == tuple(exp)
    assert [at[i].tolist() for i in range(4)] == values[:4]
