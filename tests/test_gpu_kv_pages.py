"""baps_kv_fork and baps_kv_compact: whole numbers and copied pages equal to a plain restatement."""
import pytest
import torch

import serving
from paper_2602_02071_b200 import binding
from test_gpu_kv_append import pool

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def check_pool(state, before, copies):
    for t, b in zip(state, before):
        b = b.clone()
        if copies:
            src, dst = (torch.tensor(i).cuda() for i in zip(*copies))
            b[dst] = b[src]
        assert torch.equal(t, b)


def check_fork(state, page, table, lengths, refs, parents, reserve=0, window=serving.NONE, sinks=0):
    before = [t.clone() for t in state]
    got = binding.baps_kv_fork(binding.KvCache(*state), ints(table), ints(lengths), ints(refs), ints(parents), reserve=reserve,
                               window=window, sinks=sinks)
    want = serving.fork(table, lengths, refs, parents, page, len(refs), reserve, window, sinks)
    for g, w in zip(got, want):
        assert g.tolist() == w
    check_pool(state, before, want[3])
    return want


def batch(rows, width, page, n_pages, seed, most=None):
    """Tables with some shared full pages, their counts, lengths."""
    g = torch.Generator().manual_seed(seed)
    lengths = torch.randint(0, (most or width * page) + 1, (rows,), generator=g).tolist()
    order = torch.randperm(n_pages, generator=g).tolist()
    table = [[-1] * width for _ in range(rows)]
    for b, n in enumerate(lengths):
        for c in range(-(-n // page)):
            shared = b > 0 and c < 2 and (c + 1) * page <= min(n, lengths[b - 1])
            table[b][c] = table[b - 1][c] if shared else order.pop()
    refs = [0] * n_pages
    for row in table:
        for e in row:
            if e >= 0:
                refs[e] += 1
    return table, lengths, refs


@pytest.mark.parametrize("page,D,heads", [(16, 64, 1), (16, 128, 3), (64, 128, 8), (128, 64, 2)])
@pytest.mark.parametrize("rows,new_rows", [(1, 1), (1, 9), (5, 3), (20, 41)])
@pytest.mark.parametrize("reserve,window,sinks", [(0, serving.NONE, 0), (1, serving.NONE, 0), (70, 100, 5), (300, 1, 0), (3, 40, 200)])
def test_fork(page, D, heads, rows, new_rows, reserve, window, sinks):
    width = 8 + 300 // page
    n_pages = rows * 8 + new_rows * (reserve // page + 3)
    table, lengths, refs = batch(rows, width, page, n_pages, rows + page, most=8 * page)
    g = torch.Generator().manual_seed(new_rows)
    parents = torch.randint(-1, rows + 1, (new_rows,), generator=g).tolist()
    check_fork(pool(n_pages, heads, page, D, 1), page, table, lengths, refs, parents, reserve, window, sinks)


def test_fork_without_room():
    """A pool that runs out in the middle of the batch, and rows that the table cannot hold."""
    page, n_pages = 16, 12
    table = [[0, 1, -1, -1], [2, 3, 4, -1], [5, -1, -1, -1]]
    lengths, refs = [20, 48, 16], [1] * 6 + [0, 0, 1, 0, 0, 1]
    state = pool(n_pages, 2, page, 64, 1)
    want = check_fork(state, page, table, lengths, refs, [0, 0, 1, 2, 0, 2, -1], reserve=16)
    assert want[1] == [20, 20, 48, -1, -1, -1, 0]          # 1 + 2 + 1 of the four free pages
    want = check_fork(state, page, table, lengths, refs, [1, 0, 2], reserve=17)
    assert want[1] == [-1, 20, 16]
    assert check_fork(state, page, table, lengths, [1] * n_pages, [2, 0, 1], reserve=0)[1] == [16, 20, 48]
    assert check_fork(state, page, table, lengths, [1] * n_pages, [2, 0, 0], reserve=0)[1] == [16, 20, -1]


def test_fork_of_odd_tables():
    """Entries that name no page, lengths below zero, parents of no row, a sequence whose last page is gone."""
    page = 16
    table = [[0, -1, 2, -1], [9, 3, -1, -1], [4, -1, -1, -1], [1, 5, 6, -1]]
    check_fork(pool(9, 1, page, 64, 2), page, table, [40, 33, -4, 37], [1] * 7 + [0, 0], [0, 0, 1, 1, 2, 3, 7, -9, 3], 0)


def test_fork_of_many_rows():
    page, rows, new_rows, n_pages = 16, 700, 2500, 9000
    table, lengths, refs = batch(rows, 5, page, n_pages, 3, most=64)
    g = torch.Generator().manual_seed(1)
    parents = torch.randint(-1, rows, (new_rows,), generator=g).tolist()
    check_fork(pool(n_pages, 1, page, 64, 1), page, table, lengths, refs, parents, 5)


def test_fork_that_looks_far_for_free_pages():
    """All free pages stand behind 40000 used ones."""
    page, n_pages = 16, 40100
    table, lengths, refs = batch(4, 5, page, 60, 3, most=70)
    refs = refs + [1] * (n_pages - 60 - 37) + [0] * 37
    for i in range(60):
        refs[i] = max(refs[i], 1)
    check_fork(pool(n_pages, 1, page, 64, 1), page, table, lengths, refs, [0, 1, 2, 3, 0, 1, 2, 0], 30)


def check_compact(state, table, refs):
    before = [t.clone() for t in state]
    got = binding.baps_kv_compact(binding.KvCache(*state), ints(table).view(len(table), len(table[0]) if table else 0), ints(refs))
    want = serving.compact(table, refs)
    if table:
        assert got[0].tolist() == want[0]
    assert got[1].tolist() == want[1] and got[2].tolist() == want[2] and got[3].tolist() == [want[3]]
    check_pool(state, before, want[4])


@pytest.mark.parametrize("n_pages", [1, 2, 7, 1023, 1024, 1025, 5000])
@pytest.mark.parametrize("live", [0.0, 0.1, 0.5, 0.9, 1.0])
def test_compact(n_pages, live):
    g = torch.Generator().manual_seed(n_pages)
    refs = (torch.rand(n_pages, generator=g) < live).int() * torch.randint(1, 5, (n_pages,), generator=g)
    table = torch.randint(-2, n_pages + 1, (13, 9), generator=g).tolist()
    check_compact(pool(n_pages, 2, 16, 64, 1), table, refs.tolist())


def test_compact_large_pages_and_ends():
    """Everything in use at one end of the pool."""
    for refs in ([0] * 40 + [1] * 30, [1] * 30 + [0] * 40, [0] * 69 + [3], [2] + [0] * 69):
        check_compact(pool(70, 8, 64, 128, 1), [[0, 69, 40]], refs)
    check_compact(pool(70, 3, 128, 64, 1), [], [0, 1] * 35)


def test_compact_of_a_pool_too_large_to_be_read_by_every_block():
    n_pages = 70001
    g = torch.Generator().manual_seed(3)
    refs = (torch.rand(n_pages, generator=g) < 0.4).int()
    table = torch.randint(-1, n_pages, (50, 40), generator=g).tolist()
    check_compact(pool(n_pages, 1, 16, 64, 1), table, refs.tolist())


def test_fork_and_compact_in_a_graph():
    page, n_pages, rows = 16, 60, 4
    table, lengths, refs = batch(rows, 4, page, n_pages, 5, most=48)
    state = pool(n_pages, 2, page, 64, 1)
    cache = binding.KvCache(*state)
    t, n, r, p = ints(table), ints(lengths), ints(refs), ints([0, 0, 1, 2, 3, 3])
    binding.baps_kv_fork(cache, t, n, r, p, reserve=2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = binding.baps_kv_fork(cache, t, n, r, p, reserve=2)
        b = binding.baps_kv_compact(cache, a[0], a[2])
    p.copy_(ints([3, 3, 3, -1, 0, 1]))
    graph.replay()
    want = serving.fork(table, lengths, refs, [3, 3, 3, -1, 0, 1], page, n_pages, 2, serving.NONE, 0)
    assert [x.tolist() for x in a] == list(want[:3])
    then = serving.compact(want[0], want[2])
    assert [x.tolist() for x in b] == [then[0], then[1], then[2], [then[3]]]


def test_refusals():
    page, n_pages = 16, 20
    state = pool(n_pages, 2, page, 64, 1)
    cache = binding.KvCache(*state)
    t, n, r, p = ints([[0, 1, -1, -1]]), ints([20]), ints([1, 1] + [0] * 18), ints([0])

    def status(fn):
        with pytest.raises(binding.BapsError) as e:
            fn()
        return e.value.status

    assert status(lambda: binding.baps_kv_fork(cache, t, n, r, p, reserve=-1)) == -1
    assert status(lambda: binding.baps_kv_fork(cache, t, n, r, p, window=0)) == -1
    assert status(lambda: binding.baps_kv_fork(cache, t, n, r, p[:0])) == -1
    many = ints([[-1]] * 8193)
    assert status(lambda: binding.baps_kv_fork(cache, many, ints([0] * 8193), r, p)) == -2
    with pytest.raises(ValueError):
        binding.baps_kv_fork(cache, t, n, r[:5], p)
    with pytest.raises(ValueError):
        binding.baps_kv_fork(cache, t, n, r, p.long())
    with pytest.raises(ValueError):
        binding.baps_kv_compact(cache, t, r.float())
    with pytest.raises(ValueError):
        binding.baps_kv_compact(cache, t[:, ::2], r)


def test_counts_that_are_a_slice_of_a_larger_array():
    """refs is read 16 bytes at a time: a slice that begins on a multiple of four is taken, any other refused."""
    page, n_pages = 16, 9
    table, lengths, refs = [[0, 3]], [20], [1, 0, 0, 1, 0, 1, 0, 0, 0]
    state = pool(n_pages, 1, page, 64, 1)
    cache, parents = binding.KvCache(*state), ints([0, 0])
    want = serving.fork(table, lengths, refs, [0, 0], page, n_pages, 0, serving.NONE, 0)
    for at in range(6):
        part = ints([7] * at + refs + [7] * 5)[at:at + n_pages]
        if at % 4 == 0:
            got = binding.baps_kv_fork(cache, ints(table), ints(lengths), part, parents)
            assert [g.tolist() for g in got] == list(want[:3])
        else:
            n = binding.launch_count()
            with pytest.raises(binding.BapsError) as e:
                binding.baps_kv_fork(cache, ints(table), ints(lengths), part, parents)
            assert e.value.status == -3 and binding.launch_count() == n
        got = binding.baps_kv_compact(cache, ints(table), part)              # any alignment
        assert got[1].tolist() == serving.compact(table, refs)[1]
