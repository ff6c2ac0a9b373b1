"""fd_page_tables against a loop over the requests."""
import numpy as np
import pytest
import torch

from tests import cache_oracle as want

pytestmark = pytest.mark.gpu


def run(page, n_pages, width, max_tokens, cached, new, free, n_free, table):
    from paper_2311_01282_amd import fdattn
    dev = "cuda:0"
    t = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)      # noqa: E731
    batch = len(cached)
    ins = [t(cached), t(new), t(list(free) + [0] * (n_pages - len(free))), t([n_free])]
    table = t(table).reshape(batch, width) if batch else torch.zeros(0, width, dtype=torch.int32, device=dev)
    # (guards of 64 entries behind every output)
    outs = [torch.full((k + 64,), -77, dtype=torch.int32, device=dev) for k in (batch, batch + 1, max_tokens, 1)]
    one = torch.zeros(1, dtype=torch.int32, device=dev)               # an empty tensor has no address
    ptr = lambda x: (x if x.numel() else one).data_ptr()              # noqa: E731
    fdattn.fd_page_tables(batch, page, n_pages, width, max_tokens, ptr(ins[0]), ptr(ins[1]), ptr(ins[2]), ptr(ins[3]), ptr(table),
                          *[o.data_ptr() for o in outs], torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for o in outs:
        assert (o[-64:] == -77).all()
    lens, starts, slots, left = [o[:-64].tolist() for o in outs]
    return table.tolist(), lens, starts, slots, left[0]


def case(seed, batch, page, max_cached, max_new, n_free=None, spare_tokens=0, width=None):
    rng = np.random.default_rng(seed)
    cached = rng.integers(0, max_cached + 1, batch).tolist()
    new = rng.integers(0, max_new + 1, batch).tolist()
    width = width or max(1, -(-(max_cached + max_new) // page))
    held = [-(-c // page) for c in cached]
    need = sum(-(-(c + n) // page) - h for c, n, h in zip(cached, new, held))
    n_free = need if n_free is None else n_free
    n_pages = sum(held) + max(n_free, 1)
    order = rng.permutation(n_pages).tolist()
    free, rest = order[:n_free], order[n_free:]
    table = [[-5] * width for _ in range(batch)]
    for b in range(batch):
        for j in range(min(held[b], width)):
            table[b][j] = rest.pop()
    return page, n_pages, width, max(0, sum(new) + spare_tokens), cached, new, free, n_free, table


@pytest.mark.parametrize("args", [
    dict(batch=1, page=16, max_cached=0, max_new=1),
    dict(batch=3, page=16, max_cached=40, max_new=1, spare_tokens=5),
    dict(batch=7, page=32, max_cached=5, max_new=100, spare_tokens=1),
    dict(batch=63, page=16, max_cached=300, max_new=2),
    dict(batch=513, page=64, max_cached=1000, max_new=40),
    dict(batch=2049, page=16, max_cached=30, max_new=7),               # beyond one window of requests
    dict(batch=5000, page=128, max_cached=300, max_new=3, spare_tokens=9),
    dict(batch=2, page=256, max_cached=10, max_new=9000),
    dict(batch=40, page=16, max_cached=100, max_new=50, n_free=37),    # the list ends early
    dict(batch=40, page=16, max_cached=100, max_new=50, n_free=0),
    dict(batch=40, page=16, max_cached=100, max_new=50, spare_tokens=-300),    # more tokens than the slot map takes
    dict(batch=40, page=16, max_cached=100, max_new=50, width=7),      # some outgrow the table
    dict(batch=4500, page=16, max_cached=50, max_new=20, n_free=1234, spare_tokens=-9000, width=4),
], ids=lambda a: "-".join("%s%s" % (k[:3], v) for k, v in a.items()))
def test_against_the_loop(args):
    for seed in (1, 2):
        c = case(seed, **args)
        got, exp = run(*c), want.page_tables(*c)
        for name, x, y in zip(("table", "seq_lens", "starts", "slots", "n_left"), got, exp):
            assert x == y, "%s, seed %d" % (name, seed)


def test_no_requests_and_no_tokens():
    assert run(16, 4, 2, 5, [], [], [0, 1], 2, []) == ([], [], [0], [-1] * 5, 2)
    assert run(16, 4, 2, 0, [3, 0], [0, 0], [0, 1], 2, [[3, -5], [-5, -5]]) == ([[3, -5], [-5, -5]], [3, 0], [0, 0, 0], [], 2)


def test_lengths_and_counts_that_are_no_lengths():
    """Negative lengths count as none, a cached length is limited to the table, a free count to the pool; a held entry out of range gives
    no slot."""
    c = (16, 6, 3, 40, [-4, 100, 10, 5], [3, 0, 8, 4], [0, 1, 2, 3, 4, 5], 99, [[-5] * 3, [1] * 3, [-5] * 3, [99, -5, -5]])
    got = run(*c)
    assert got == tuple(want.page_tables(*c))
    assert got[3][11:15] == [-1] * 4


def test_sums_beyond_32_bits():
    c = (16, 4, 2, 8, [0] * 6, [2 ** 31 - 1, 2, 2 ** 31 - 1, 2 ** 31 - 1, 0, 1], [0, 1, 2, 3], 4, [[-5, -5]] * 6)
    got = run(*c)
    assert got[1] == [0] * 6 and got[2] == [0] + [8] * 6 and got[3] == [-1] * 8 and got[4] == 4
    c = (16, 4, 2, 8, [0] * 4, [3, 2 ** 31 - 1, 0, 1], [0, 1, 2, 3], 4, [[-5, -5]] * 4)
    got = run(*c)
    assert got[1] == [3, 0, 0, 0] and got[2] == [0, 3, 8, 8, 8] and got[3] == [48, 49, 50] + [-1] * 5 and got[4] == 3


def test_captured_and_replayed():
    """A captured call follows the lengths and the list that it finds at each replay."""
    from paper_2311_01282_amd import fdattn
    dev = "cuda:0"
    cases = [case(s, batch=20, page=16, max_cached=60, max_new=9, n_free=30, width=5) for s in (5, 6, 7)]
    page, width, n_pages, max_tokens = 16, 5, max(c[1] for c in cases), 200
    z = lambda *n: torch.zeros(*n, dtype=torch.int32, device=dev)      # noqa: E731
    cached, new, free, n_free, table = z(20), z(20), z(n_pages), z(1), z(20, width)
    outs = [z(20), z(21), z(max_tokens), z(1)]
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fdattn.fd_page_tables(20, page, n_pages, width, max_tokens, cached.data_ptr(), new.data_ptr(), free.data_ptr(), n_free.data_ptr(),
                              table.data_ptr(), *[o.data_ptr() for o in outs], torch.cuda.current_stream().cuda_stream)
    for c in cases + cases:
        for dst, src in ((cached, c[4]), (new, c[5]), (n_free, [c[7]]), (table, c[8])):
            dst.copy_(torch.tensor(src, dtype=torch.int32))
        free[:len(c[6])] = torch.tensor(c[6], dtype=torch.int32, device=dev)
        graph.replay()
        torch.cuda.synchronize()
        exp = want.page_tables(page, n_pages, width, max_tokens, *c[4:])
        assert [table.tolist()] + [o.tolist() for o in outs[:3]] + [outs[3].item()] == list(exp)
