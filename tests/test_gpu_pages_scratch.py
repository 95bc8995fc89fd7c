"""Scratch memory of the paged cache's calls: threads, streams and graphs that read one cache at the same time, and sizes that creep up."""
import threading

import numpy as np
import pytest
import torch

from tests import test_gpu_pages as T

pytestmark = pytest.mark.gpu

tq = pytest.importorskip("paper_2504_19874_amd")

DEV, ints = T.DEV, T.ints
HEADS, GROUP, D, PAGE = 4, 4, 128, 64


@pytest.fixture(scope="module")
def cache():
    """Three long sequences, whose keys are cut into ranges, and 400 pages to choose from."""
    rng = np.random.default_rng(101)
    b = T.Batch(rng, [25000, 900, 13000], [2, 1, 2], PAGE)
    p = T.filled(rng, b, HEADS, D, "e4m3")
    bounds = torch.from_numpy(np.sort(rng.standard_normal((b.n_pages, HEADS, 2, D)), 2)).to(DEV, torch.bfloat16)
    return tq.Pages(p.k, p.v, p.k_scale, p.v_scale, bounds=bounds, refs=torch.zeros(b.n_pages, dtype=torch.int32, device=DEV)), b


def queries(b, seed):
    x = np.random.default_rng([102, seed]).standard_normal((b.rows, HEADS * GROUP, D)).astype(np.float32)
    return torch.from_numpy(x).to(DEV, torch.bfloat16)


class Reader:
    """What one reader has: queries and outputs of its own."""

    def __init__(self, p, b, seed):
        self.p, self.args = p, b.args()
        self.q, self.rows = queries(b, seed), b.rows
        self.out, self.lse = torch.empty_like(self.q), torch.empty(self.q.shape[:2], device=DEV)
        self.chosen = torch.empty((b.rows, HEADS, 20), dtype=torch.int32, device=DEV)
        self.part = torch.empty_like(self.q)

    def call(self):
        tq.tq_pages_attend(self.p, self.q, *self.args, 0.1, self.out, lse=self.lse)
        tq.tq_pages_select(self.p, self.q, *self.args, self.chosen)
        tq.tq_pages_attend(self.p, self.q, *self.args, 0.1, self.part, chosen=self.chosen)

    def results(self):
        return [t.clone() for t in (self.out, self.lse, self.chosen, self.part)]

    def clear(self):
        for t in (self.out, self.lse, self.chosen, self.part):
            t.zero_()


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.fixture(scope="module")
def readers(cache):
    made = [Reader(*cache, seed) for seed in range(3)]
    want = []
    for r in made:
        r.call()
        torch.cuda.synchronize()
        want.append(r.results())
    assert not same(want[0], want[1])
    return made, want


def test_streams_of_one_thread(readers):
    made, want = readers
    streams = [torch.cuda.Stream() for _ in made]
    for r in made:
        r.clear()
    torch.cuda.synchronize()
    for _ in range(30):
        for r, s in zip(made, streams):
            with torch.cuda.stream(s):
                r.call()
    torch.cuda.synchronize()
    assert all(same(r.results(), w) for r, w in zip(made, want))
    spaces = made[0].p._scratch.spaces
    assert len({spaces[s.cuda_stream].data_ptr() for s in streams}) == len(streams)


@pytest.mark.parametrize("own_streams", [False, True])
def test_threads(readers, own_streams):
    """Each on a stream of its own, and all on the default one."""
    made, want = readers
    for r in made:
        r.clear()
    torch.cuda.synchronize()
    go, seen, errors = threading.Barrier(len(made)), [], []

    def work(r):
        try:
            go.wait(20)
            with torch.cuda.stream(torch.cuda.Stream() if own_streams else torch.cuda.default_stream()):
                for _ in range(30):
                    r.call()
            seen.append([t.data_ptr() for t in r.p._scratch.spaces.values()])
            go.wait(20)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(r,)) for r in made]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors and len({x for s in seen for x in s}) == len(made)
    assert all(same(r.results(), w) for r, w in zip(made, want))


def test_graphs_that_run_at_once(readers):
    """Captured from one cache, replayed on two streams without an order between them, with eager calls on a third."""
    made, want = readers
    graphs = []
    for r in made[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            r.call()
    streams = [torch.cuda.Stream() for _ in graphs]
    for i in range(6):
        for r in made:
            r.clear()
        torch.cuda.synchronize()
        for _ in range(10):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
            made[2].call()
        torch.cuda.synchronize()
        assert all(same(r.results(), w) for r, w in zip(made, want)), i


def test_a_stream_that_is_captured_after_eager_calls_on_it(readers):
    """The graph has scratch memory of its own, also when the stream's has been replaced since."""
    made, want = readers
    p = tq.Pages(*[getattr(made[0].p, n) for n in ("k", "v", "k_scale", "v_scale")], bounds=made[0].p.bounds)
    r = made[0]
    kept, r.p = r.p, p
    try:
        s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            r.call()
        torch.cuda.synchronize()
        before = p._scratch.spaces[s.cuda_stream].data_ptr()
        with torch.cuda.graph(graph, stream=s):
            r.call()
        assert p._scratch.spaces[s.cuda_stream].data_ptr() == before
        with torch.cuda.stream(s):
            p.reserve_bytes(64 << 20)
            del_me = torch.empty(32 << 20, dtype=torch.uint8, device=DEV).fill_(255)  # torch may give the old one away
        for _ in range(4):
            r.clear()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert same(r.results(), want[0]) and bool((del_me == 255).all())
    finally:
        r.p = kept


def test_sizes_that_creep_up(cache):
    """A call larger than the last one by a little, many times: no more is held than half as much again as the largest needs."""
    p, b = cache
    p = tq.Pages(p.k, p.v, p.k_scale, p.v_scale, bounds=p.bounds)
    table, lens, _, _ = b.args()
    q = torch.randn((3 * 40, HEADS * GROUP, D), device=DEV).to(torch.bfloat16)
    chosen = torch.empty((3 * 40, HEADS, 4), dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    from paper_2504_19874_amd import _lib
    import ctypes as C
    before, largest = torch.cuda.memory_allocated(), 0
    for new in range(1, 41):
        tq.tq_pages_select(p, q[:3 * new], table, lens, None, new, chosen[:3 * new])
        batch = _lib.TqBatch(n_seqs=3, max_new=new, n_rows=3 * new, width=table.shape[1], table_stride=table.shape[1])
        largest = max(largest, int(_lib.load().tq_pages_select_workspace_bytes(C.byref(p.c), C.byref(batch))))
    assert largest > 100000 and torch.cuda.memory_allocated() - before <= 1.5 * largest + 1024
    torch.cuda.synchronize()


def test_reserved_calls_ask_torch_for_nothing(readers):
    made, want = readers
    r = made[0]
    p = tq.Pages(r.p.k, r.p.v, r.p.k_scale, r.p.v_scale, bounds=r.p.bounds, refs=r.p.refs)
    table, _, _, most = r.args
    p.reserve_attend(r.rows, *table.shape, HEADS * GROUP, most)
    p.reserve_attend(r.rows, *table.shape, HEADS * GROUP, most, n_chosen=20)
    p.reserve_select(r.rows, *table.shape, most)
    kept, r.p = r.p, p
    try:
        count = torch.cuda.memory_stats()["allocation.all.allocated"]
        r.call()
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == count
        torch.cuda.synchronize()
        assert same(r.results(), want[0]) and p.c.workspace == p.workspace.data_ptr() and p.c.workspace_bytes == p.workspace.numel()
    finally:
        r.p = kept


def test_without_the_compiled_half(readers, cache, monkeypatch):
    from paper_2504_19874_amd import _lib
    monkeypatch.setattr(_lib, "_call", _lib._Checked())
    test_streams_of_one_thread(readers)
    test_threads(readers, False)
    test_threads(readers, True)
    test_graphs_that_run_at_once(readers)
    test_a_stream_that_is_captured_after_eager_calls_on_it(readers)
    test_sizes_that_creep_up(cache)


def test_the_pools_calls_captured():
    """Fork, free, reserve and compact in a graph: every replay against the same calls made eagerly, from states that differ."""
    rng = np.random.default_rng(103)
    heads, page, n_pages, rows, width = 1, 16, 300, 24, 8

    def state():
        p = tq.make_pages(n_pages, heads, 64, page, dtype=torch.int8, bounds=True, device=DEV)
        return p, torch.full((rows, width), -1, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV), ints([0, 0, 0])

    parents, children, ended, starts = ints(np.zeros(8)), ints(np.zeros(8)), ints(np.zeros(5)), ints(np.zeros(rows + 1))

    def call(p, table, lens, told):
        tq.tq_pages_fork(p, table, lens, parents, children, missing=told[:1])
        tq.tq_pages_free(p, table, lens, ended)
        tq.tq_pages_compact(p, table, n_live=told[1:2])
        lens.add_(starts.diff())
        tq.tq_pages_reserve(p, table, lens, 20, missing=told[2:], starts=starts)

    a, b = state(), state()
    call(*state())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*a)
    for t, u in zip((a[0].k, a[0].v, a[0].k_scale, a[0].bounds), (b[0].k, b[0].v, b[0].k_scale, b[0].bounds)):
        x = torch.from_numpy(rng.integers(-100, 100, t.shape)).to(t.dtype)
        t.copy_(x), u.copy_(x)
    live = 0
    for i in range(12):
        new = rng.integers(0, 21, rows)
        starts.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(new)])))
        parents.copy_(torch.from_numpy(rng.integers(0, rows, 8)))
        children.copy_(torch.from_numpy(rng.integers(0, rows, 8)))
        ended.copy_(torch.from_numpy(rng.integers(0, rows, 5)))
        graph.replay()
        call(*b)
        if i % 3 == 0:
            torch.cuda.synchronize()
        for x, y in zip((*a[1:], a[0].refs, a[0].k, a[0].v, a[0].k_scale, a[0].bounds), (*b[1:], b[0].refs, b[0].k, b[0].v, b[0].k_scale, b[0].bounds)):
            assert torch.equal(x, y), i
        live = max(live, int(a[3][1]))
    assert live > 20
