"""Page tables on the device (cascade_pages_fork, cascade_pages_compact, cascade_pages_copy) against lists, number by number."""
import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2507_05228_b200 import binding as cb

pytestmark = pytest.mark.gpu


def random_state(rng, n, width, n_pages, page, shares):
    """Sequences of random lengths; some share pages with the one before, up to and including a partly filled page."""
    table, kv_len = rng.choice([-1, 2 ** 30], (n, width)).astype(np.int32), np.zeros(n, np.int32)
    free = list(rng.permutation(n_pages))
    for i in range(n):
        rows = int(rng.integers(0, width * page // 2 + 1))
        count = -(-rows // page)
        if i and rng.random() < shares:
            rows = int(kv_len[i - 1]) - int(rng.integers(0, 2)) * int(rng.integers(0, page))
            rows = max(rows, 0)
            count = -(-rows // page)
            keep = count if rng.random() < 0.5 else min(count, rows // page)
        else:
            keep = 0
        if count - keep > len(free):
            rows = count = keep = 0
        table[i, :keep] = table[i - 1, :keep]
        for c in range(keep, count):
            table[i, c] = free.pop()
        kv_len[i] = rows
    return table, kv_len


def run_fork(table, kv_len, source, add, n_pages, page):
    got = cb.cascade_pages_fork(pu.ints(table), pu.ints(kv_len), pu.ints(source), pu.ints(add), n_pages, page)
    return [t.cpu().numpy() for t in got]


def same(got, want):
    for name, g, w in zip(("table", "kv_len", "refs", "copies", "report"), got, want):
        assert np.array_equal(g, np.asarray(w)), (name, g, w)


@pytest.mark.parametrize("n,width,n_pages,page", [(1, 1, 1, 16), (3, 4, 12, 16), (8, 9, 40, 48), (65, 7, 300, 16), (300, 5, 1111, 64),
                                                  (1500, 3, 3000, 16), (40, 200, 20000, 32)])
@pytest.mark.parametrize("seed", range(3))
def test_fork(n, width, n_pages, page, seed):
    rng = np.random.default_rng([seed, n, width])
    table, kv_len = random_state(rng, n, width, n_pages, page, 0.5)
    source = rng.integers(-1, n, n) if seed else np.arange(n)
    add = rng.integers(0, 3 if seed < 2 else 2 * page, n)
    same(run_fork(table, kv_len, source, add, n_pages, page), pu.fork(table, kv_len, source, add, n_pages, page))


def test_fork_of_one_sequence_by_all_readers_and_writers():
    """Twenty rows, pages of sixteen: who writes the second page alone keeps it, a reader among its holders makes all writers copy."""
    table, kv_len = np.array([[4, 2, -1], [-1, -1, -1], [-1, -1, -1], [-1, -1, -1]], np.int32), np.array([20, 0, 0, 0], np.int32)
    for add, copies, free in (([1, 1, 1, 1], [[-1, -1], [2, 0], [2, 1], [2, 3]], 1), ([0, 1, 1, 0], [[-1, -1], [2, 0], [2, 1], [-1, -1]], 2),
                              ([0, 0, 0, 0], [[-1, -1]] * 4, 4), ([5, 0, 0, 0], [[2, 0], [-1, -1], [-1, -1], [-1, -1]], 3)):
        got = run_fork(table, kv_len, [0, 0, 0, 0], add, 6, 16)
        assert got[3].tolist() == copies and got[4].tolist() == [0, 0, 0, free]
        same(got, pu.fork(table, kv_len, np.zeros(4, int), np.array(add), 6, 16))


def test_new_and_ended_sequences():
    table, kv_len = np.array([[5, 1], [0, -1], [-1, -1]], np.int32), np.array([32, 3, 0], np.int32)
    got = run_fork(table, kv_len, [-1, 1, -1], [0, 0, 17], 6, 16)
    assert got[0].tolist() == [[-1, -1], [0, -1], [1, 2]] and got[1].tolist() == [0, 3, 17]
    assert got[2].tolist() == [1, 1, 1, 0, 0, 0] and got[4].tolist() == [0, 0, 0, 3]


@pytest.mark.parametrize("what", ["pages", "width", "source", "add", "length", "id"])
def test_a_step_that_cannot_be_done_changes_nothing(what):
    rng = np.random.default_rng(5)
    n, width, page = 20, 6, 16
    n_pages = 60 if what == "pages" else 200
    table, kv_len = random_state(rng, n, width, n_pages, page, 0.3)
    kv_len[3] = 20
    table[3, :2] = 7, 9
    source, add = np.arange(n), np.ones(n, int)
    if what == "pages":
        add = np.full(n, 3 * page)  # 60 pages more
        add[kv_len > 3 * page] = 1
    elif what == "width":
        add[3] = width * page
    elif what == "source":
        source[2], source[7] = n, -2
    elif what == "add":
        add[5] = -1
    elif what == "length":
        kv_len[3] = width * page + 1
    else:
        table[3, 1] = -5
    got = run_fork(table, kv_len, source, add, n_pages, page)
    want = pu.fork(table, kv_len, source, add, n_pages, page)
    same(got, want)
    assert got[4][:3].any() and np.array_equal(got[0], table) and np.array_equal(got[1], kv_len) and (got[3] == -1).all()


@pytest.mark.parametrize("n,width,n_pages,page", [(1, 1, 1, 16), (2, 3, 9, 16), (8, 9, 41, 48), (65, 7, 300, 16), (300, 5, 1111, 64),
                                                  (40, 200, 20000, 32), (3, 4, 100000, 16)])
@pytest.mark.parametrize("seed", range(2))
def test_compact(n, width, n_pages, page, seed):
    rng = np.random.default_rng([seed, n, width, 3])
    table, kv_len = random_state(rng, n, width, n_pages, page, 0.4)
    got = [t.cpu().numpy() for t in cb.cascade_pages_compact(pu.ints(table), pu.ints(kv_len), n_pages, page)]
    for name, g, w in zip(("table", "refs", "moves", "report"), got, pu.compact(table, kv_len, n_pages, page)):
        assert np.array_equal(g, np.asarray(w)), (name, g, w)


def test_compaction_of_a_full_an_empty_and_a_bad_table():
    table = np.array([[2, 0], [1, 3]], np.int32)
    for kv_len in ([32, 32], [0, 0]):
        got = [t.cpu().numpy() for t in cb.cascade_pages_compact(pu.ints(table), pu.ints(kv_len), 4, 16)]
        assert got[3].tolist() == [4, 0, 0, 0] if kv_len[0] else [0, 0, 0, 4]
        assert (got[2] == -1).all() and np.array_equal(got[0], table if kv_len[0] else np.full((2, 2), -1))
    table[0, 1] = 4
    got = [t.cpu().numpy() for t in cb.cascade_pages_compact(pu.ints(table), pu.ints([32, 32]), 4, 16)]
    assert got[3][2] == 1 and np.array_equal(got[0], table) and (got[2] == -1).all()


@pytest.mark.parametrize("page_bytes", [16, 48, 4096, 32768, 98320])
@pytest.mark.parametrize("n_pairs", [1, 37, 2500])
def test_copy(page_bytes, n_pairs):
    g = torch.Generator(device="cuda").manual_seed(page_bytes + n_pairs)
    n_pages = 2 * n_pairs + 5
    if n_pages * page_bytes > 1 << 28:
        pytest.skip("a pool of the larger pages is tested with fewer pairs")
    pools = [torch.randint(0, 255, (n_pages, page_bytes), generator=g, device="cuda", dtype=torch.uint8) for _ in range(3)]
    wide = torch.randint(0, 255, (n_pages, page_bytes + 32), generator=g, device="cuda", dtype=torch.uint8)
    pools.append(wide[:, 16:16 + page_bytes])  # pages further apart than they are long
    ids = torch.randperm(n_pages, generator=g, device="cuda")
    pairs = torch.stack([ids[:n_pairs], ids[n_pairs:2 * n_pairs]], 1).int()
    pairs[::3, 0] = -1
    pairs[1::5, 1] = -1
    want = [p.clone() for p in pools] + [wide.clone()]
    there = (pairs >= 0).all(1)
    for w in want[:4]:
        w[pairs[there, 1].long()] = w[pairs[there, 0].long()]
    want[4][:, 16:16 + page_bytes] = want[3]
    cb.cascade_pages_copy(pools, pairs)
    for got, w in zip(pools + [wide], want):
        assert torch.equal(got, w)


def test_copy_reports_a_bad_pair_and_copies_the_others():
    pool = torch.arange(8 * 64, device="cuda", dtype=torch.float32).reshape(8, 64)
    want = pool.clone()
    want[3] = pool[2]
    cb.cascade_pages_copy([pool], pu.ints([[0, 8], [2, 3], [-9, 1], [5, 5]]))
    with pytest.raises(cb.CascadeError, match="code 125.*pair 0, value 8|code 125.*pair 2, value -9"):
        cb.cascade_paged_status()
    assert torch.equal(pool, want) and cb.cascade_paged_status() == 0


def test_copy_beyond_32_bits_of_offset():
    pool = torch.empty((5, 1 << 30), dtype=torch.uint8, device="cuda")
    pool[0].fill_(7)
    cb.cascade_pages_copy([pool], pu.ints([[0, 4]]))
    assert (pool[4] == 7).all()


def test_a_captured_step_follows_its_tables():
    """Fork, copy and compaction in a graph, replayed on tables that have changed since."""
    rng = np.random.default_rng(9)
    n, width, n_pages, page = 12, 6, 100, 16
    state = [random_state(rng, n, width, n_pages, page, 0.5) for _ in range(3)]
    table, kv_len = pu.ints(state[0][0]), pu.ints(state[0][1])
    source, add = pu.ints(np.arange(n) // 2), pu.ints(np.ones(n))
    pool = torch.randn((n_pages, page, 2, 64), device="cuda")
    shapes = ((n, width), (n,), (n_pages,), (n, 2), (4,))
    out = tuple(torch.empty(s, dtype=torch.int32, device="cuda") for s in shapes)
    out2 = tuple(torch.empty(s, dtype=torch.int32, device="cuda") for s in ((n, width), (n_pages,), (n_pages // 2, 2), (4,)))

    def step():
        cb.cascade_pages_fork(table, kv_len, source, add, n_pages, page, out=out)
        cb.cascade_pages_copy([pool], out[3])
        cb.cascade_pages_compact(out[0], out[1], n_pages, page, out=out2)
        cb.cascade_pages_copy([pool], out2[2])

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t, k in state[1:]:
        table.copy_(pu.ints(t))
        kv_len.copy_(pu.ints(k))
        want_pool = pool.clone()
        graph.replay()
        f = pu.fork(t, k, np.arange(n) // 2, np.ones(n, int), n_pages, page)
        same([x.cpu().numpy() for x in out], f)
        c = pu.compact(f[0], f[1], n_pages, page)
        for g, w in zip(out2, c):
            assert np.array_equal(g.cpu().numpy(), np.asarray(w))
        for pairs in (f[3], c[2]):
            for a, b in pairs:
                if a >= 0:
                    want_pool[b] = want_pool[a]
        assert torch.equal(pool, want_pool)


@pytest.mark.parametrize("n_pages", [8200, 40000])
@pytest.mark.parametrize("reader", [None, 5])
def test_fork_of_one_prompt_by_as_many_sequences_as_there_may_be(n_pages, reader):
    """8192 sequences that go on writing the second page of one prompt: the first keeps it, unless one only reads."""
    n, page = 8192, 16
    table, kv_len = np.full((n, 3), -1, np.int32), np.zeros(n, np.int32)
    table[0, :2], kv_len[0] = (7, 2), 20
    add = np.ones(n, np.int32)
    if reader is not None:
        add[reader] = 0
    got = [t.cpu().numpy() for t in cb.cascade_pages_fork(pu.ints(table), pu.ints(kv_len), pu.ints(np.zeros(n)), pu.ints(add), n_pages, page)]
    copies = add == 1
    copies[0] = reader is not None
    free = np.setdiff1d(np.arange(n_pages), [7, 2])
    want, refs = np.tile([7, 2, -1], (n, 1)), np.zeros(n_pages, int)
    want[copies, 1] = free[:copies.sum()]
    refs[7], refs[2] = n, n - copies.sum()
    refs[want[copies, 1]] = 1
    pairs = np.full((n, 2), -1)
    pairs[copies] = np.stack([np.full(copies.sum(), 2), want[copies, 1]], 1)
    for g, w in zip(got, (want, 20 + add, refs, pairs, [0, 0, 0, free.size - copies.sum()])):
        assert np.array_equal(g, w)
