"""Tokens whose page was missing when they were appended: a page that the sequence gets later does not stand in for them."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as po
from tests import test_gpu_pages as T
from tests.test_gpu_pages_serving import Server

pytestmark = pytest.mark.gpu

tq = pytest.importorskip("paper_2504_19874_amd")

DEV, ints = T.DEV, T.ints


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_a_pool_that_has_pages_again(kind):
    """A sequence goes on without a page while others hold all of them; one ends, its pages are free, and the sequence goes on: it never reads
    what they hold, and has a page from the next span of tokens on."""
    s = Server(kind, n_pages=4, seed=2)
    s.step([30, 32, 0, 0])
    s.step([1, 0, 1, 0])       # row 0 has room; row 2 gets none
    assert s.pool.table[2, 0] == -1
    s.step([0, 0, 3, 0])
    s.pool.free([1])
    tq.tq_pages_free(s.p, s.table, s.lens, ints([1]))
    s.check()
    for _ in range(11):
        s.step([0, 0, 1, 0])
        assert s.pool.table[2, 0] == -1
    assert s.pool.lens[2] == 15
    s.step([0, 0, 2, 0])       # the rest of a span that has none, and the first of one that gets one
    assert s.pool.table[2, 0] == -1 and s.pool.table[2, 1] >= 0
    s.step([0, 0, 1, 0], chosen=2)


def test_a_fork_without_a_page_for_the_last_tokens():
    s = Server("int8", n_pages=3, seed=3)
    s.step([20, 8, 0, 0])
    pairs, short = s.pool.fork([0], [2])
    missing = ints([-1])
    tq.tq_pages_fork(s.p, s.table, s.lens, ints([0]), ints([2]), missing=missing)
    assert short == 1 == int(missing) and pairs == []
    s.pool.free([1])
    tq.tq_pages_free(s.p, s.table, s.lens, ints([1]))
    for _ in range(3):
        s.step([0, 0, 1, 0])
        assert s.pool.table[2, 1] == -1


def test_rows_of_different_counts():
    """With starts, a sequence's own new tokens count: the hole of one with a single token lies within the most of another."""
    s = Server("e4m3", n_pages=6, seed=4)
    s.step([64, 32, 0, 0])
    s.step([0, 0, 4, 0])
    assert s.pool.table[2, 0] == -1
    s.pool.free([1])
    tq.tq_pages_free(s.p, s.table, s.lens, ints([1]))
    new = [0, 10, 1, 0]
    for starts, page in ((s.starts(new), -1), (None, 1)):
        table, lens, missing = s.table.clone(), s.lens + ints(new), ints([-1])
        p = tq.Pages(s.p.k, s.p.v, s.p.k_scale, s.p.v_scale, refs=s.p.refs.clone())
        pool = po.Pool(s.pool.table, s.pool.lens + np.array(new), s.pool.refs, s.page)
        short = pool.reserve(20, starts)
        tq.tq_pages_reserve(p, table, lens, 20, missing=missing, starts=None if starts is None else ints(starts))
        assert T.same_pool(p, pool, table, lens) and int(missing) == short
        assert (table[2, 0].item() >= 0) == (page > 0)  # (without them all of the last 20 positions are new)


def test_forks_into_rows_of_negative_lengths():
    """They hold no tokens: the same as a length of zero, whatever its size beside the list's."""
    rng = np.random.default_rng(122)
    for below in (-1, -2, -3, -1000, -2**31):
        p, pool = T.pool_state(rng, 40, 6, 4, 16, live=2)
        pool.lens[:2], pool.table[:], pool.refs[:] = [20, 33], -1, 0
        pool.table[0, :2], pool.table[1, :3], pool.refs[:5] = [0, 1], [2, 3, 4], 1
        p.refs.copy_(ints(pool.refs))
        pool.lens[2:5] = below
        table, lens = ints(pool.table), ints(pool.lens)
        parents, children = [0, 1, 0, 4, 1], [2, 3, 3, 5, 4]
        want = T.contents(p)
        pairs, short = pool.fork(parents, children)
        missing = ints([-1])
        tq.tq_pages_fork(p, table, lens, ints(parents), ints(children), missing=missing)
        assert T.same_pool(p, pool, table, lens) and int(missing) == short, below
        assert all(torch.equal(a, b) for a, b in zip(T.contents(p), T.moved(want, pairs)))
        assert pool.lens.tolist() == [20, 33, 20, 33, 33, 0]


@pytest.mark.parametrize("seed", range(3))
def test_reserve_of_any_state(seed):
    """Random tables with holes, lengths and counts, with starts and without."""
    rng = np.random.default_rng([121, seed])
    rows, width, page, n = 1500, 7, 16, 7000
    for most, with_starts in ((1, False), (1, True), (5, True), (40, True), (40, False), (2**31 - 1, True), (0, False)):
        table = np.where(rng.random((rows, width)) < 0.5, -1, 0)
        ids = rng.permutation(n)
        used = int((table == 0).sum())
        table[table == 0] = ids[:used]
        refs = np.zeros(n, int)
        refs[ids[:used + 300]] = 1
        lens = rng.integers(0, width * page + 20, rows)
        starts = np.concatenate([[0], np.cumsum(np.minimum(rng.integers(0, 45, rows), lens))]) if with_starts else None
        pool = po.Pool(table, lens, refs, page)
        p = tq.make_pages(n, 1, 64, page, dtype=torch.int8, device=DEV)
        p.refs.copy_(ints(refs))
        t, ln, missing = ints(table), ints(lens), ints([-1])
        short = pool.reserve(most, starts)
        tq.tq_pages_reserve(p, t, ln, most, missing=missing, starts=None if starts is None else ints(starts))
        assert T.same_pool(p, pool, t, ln) and int(missing) == short
