"""Numbers of the paged cache's calls that the library's 32 bits do not hold, or that are none."""
import numpy as np
import pytest
import torch

from tests import test_gpu_pages as T

pytestmark = pytest.mark.gpu

tq = pytest.importorskip("paper_2504_19874_amd")

DEV, ints = T.DEV, T.ints


def test_numbers_beyond_32_bits_are_refused():
    p = tq.make_pages(4, 2, 64, 16, bounds=True, device=DEV)
    table, lens, starts = ints([[0, 1]]), ints([5]), ints([0, 1])
    q = torch.zeros((1, 4, 64), dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device=DEV)
    pick = torch.zeros((1, 2, 2), dtype=torch.int32, device=DEV)
    for n in (2**31, 2**32, 2**32 + 1, -2**31 - 1, 1.5, "1", None):
        for match, f in [
                ("max_new", lambda: tq.tq_pages_append(p, kv, kv, table, lens, starts, n)),
                ("max_new", lambda: tq.tq_pages_attend(p, q, table, lens, starts, n, 0.1, q.clone())),
                ("window", lambda: tq.tq_pages_attend(p, q, table, lens, starts, 1, 0.1, q.clone(), window=n)),
                ("max_new", lambda: tq.tq_pages_select(p, q, table, lens, starts, n, pick)),
                ("keep_first", lambda: tq.tq_pages_select(p, q, table, lens, starts, 1, pick, keep_first=n)),
                ("keep_last", lambda: tq.tq_pages_select(p, q, table, lens, starts, 1, pick, keep_last=n)),
                ("max_new", lambda: tq.tq_pages_reserve(p, table, lens, n))]:
            with pytest.raises(tq.TurboQuantError, match=match):
                f()


def test_whole_numbers_of_any_type():
    p = tq.make_pages(4, 2, 64, 16, bounds=True, device=DEV)
    table, lens, starts = ints([[0, 1]]), ints([5]), ints([0, 1])
    rng = np.random.default_rng(111)
    kv = torch.from_numpy(rng.standard_normal((5, 2, 64)).astype(np.float32)).to(DEV)
    tq.tq_pages_append(p, kv, kv, table, lens, None, 5)
    q = torch.from_numpy(rng.standard_normal((1, 4, 64)).astype(np.float32)).to(DEV)
    want = torch.empty_like(q)
    tq.tq_pages_attend(p, q, table, lens, starts, 1, 0.25, want, window=3)
    for kind in (np.int64, np.int32, torch.tensor):
        got = torch.empty_like(q)
        tq.tq_pages_attend(p, q, table, lens, starts, kind(1), np.float32(0.25), got, window=kind(3))
        assert torch.equal(got, want)
