"""Choosing pages: bounds that are infinite or no numbers."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as po
from tests import test_gpu_pages as T

pytestmark = pytest.mark.gpu

tq = pytest.importorskip("paper_2504_19874_amd")

DEV, ints = T.DEV, T.ints


@pytest.mark.parametrize("d,page,dtype,heads,group,lens,new,n", [
    (128, 16, "bf16", 2, 4, [900, 17], [2, 1], 9), (64, 16, "f32", 1, 1, [700, 100], [4, 1], 7), (256, 32, "bf16", 3, 2, [900, 31], [2, 2], 10),
    (64, 16, "bf16", 1, 9, [600], [1], 30), (128, 16, "f32", 2, 2, [20000], [1], 200)])
def test_bounds_that_are_not_finite(d, page, dtype, heads, group, lens, new, n):
    """Channels without a bound on one side or both, pages marked by infinite bounds, NaN among them, queries with zeros and NaN."""
    rng = np.random.default_rng([91, d, group])
    b = T.Batch(rng, lens, new, page)
    bounds = np.sort(rng.standard_normal((b.n_pages, heads, 2, d)), 2)
    few = rng.random((b.n_pages, heads, 1, 1))
    bounds[:, :, 0][(rng.random((b.n_pages, heads, d)) < 0.02) & (few[:, :, 0] < 0.5)] = -np.inf
    bounds[:, :, 1][(rng.random((b.n_pages, heads, d)) < 0.02) & (few[:, :, 0] < 0.5)] = np.inf
    one_channel = np.flatnonzero(rng.random(b.n_pages) < 0.3)
    bounds[one_channel, :, 0, 5] = -np.inf  # a score that is finite where the query's value is positive
    for value, share in ((-np.inf, 0.05), (np.inf, 0.05), (np.nan, 0.05)):
        at = rng.random(b.n_pages) < share
        bounds[at, :, int(value > 0), rng.integers(0, d)] = value
    bounds[rng.random(b.n_pages) < 0.05] = -np.inf
    bounds = torch.from_numpy(bounds).to(DEV, torch.bfloat16)
    zero = torch.zeros((b.n_pages, heads, page, d), dtype=torch.int8, device=DEV)
    ones = torch.ones((b.n_pages, heads), device=DEV)
    p = tq.Pages(zero, zero, ones, ones, bounds=bounds)
    q = rng.standard_normal((b.rows, heads * group, d)).astype(np.float32)
    q[rng.random(q.shape) < 0.1] = 0
    for case in ("finite", "positive", "nan"):
        if case == "positive":
            q[..., 5] = np.abs(q[..., 5])
        if case == "nan":
            q[-1, -1, d // 2] = np.nan
        t = torch.from_numpy(q).to(DEV, T.TYPES[dtype])
        chosen = torch.full((b.rows, heads, n), -7, dtype=torch.int32, device=DEV)
        tq.tq_pages_select(p, t, *b.args(), chosen, keep_first=0, keep_last=1)
        want = po.select(*[T.as64(bounds[:, :, i]) for i in (0, 1)], page, t.double().cpu().numpy(), b.table, b.lens, b.starts, n, 0, 1)
        assert np.array_equal(chosen.cpu().numpy(), want), case


@pytest.mark.parametrize("kind,dtype", [("e4m3", "f32"), ("e4m3", "bf16"), ("int8", "f32")])
def test_bounds_hold_what_was_appended_and_nearly_what_is_stored(kind, dtype):
    """Keys appended a few at a time, larger and larger, so that codes are rounded again and again.  Every value lies between its channel's
    bounds.  A stored one may lie beyond them: e4m3 by its first rounding, 2^-4 of its size, and by roundings to subnormal codes, half of
    2^-9 of the scale that each is made with; int8 by half of the scale that each is made with.  A scale that grows at least doubles,
    so the scales up to the last one add up to less than twice that.  The sum of a row's products is within that of the page's score."""
    rng = np.random.default_rng([92, kind == "int8"])
    heads, d, page = 2, 64, 16
    p = tq.make_pages(1, heads, d, page, dtype=T.KINDS[kind], bounds=True, device=DEV)
    x = rng.standard_normal((page, heads, d)) * np.exp2(np.linspace(0, 9, page))[:, None, None] * np.exp(rng.normal(0, 2, (page, heads, d)))
    x = torch.from_numpy(x.astype(np.float32)).to(T.TYPES[dtype])
    table, n, beyond = ints([[0]]), 0, 0
    for new in (1, 1, 2, 1, 3, 1, 1, 4, 2):
        part = x[n:n + new].to(DEV)
        n += new
        tq.tq_pages_append(p, part, part, table, ints([n]), None, new)
        c = T.cache64(p)
        lower, upper, scale = c["lower"][0], c["upper"][0], c["k_scale"][0][:, None]
        given = x[:n].double().numpy().transpose(1, 0, 2)
        stored = (c["k"][0] * scale[:, None])[:, :n]
        assert (given >= lower[:, None]).all() and (given <= upper[:, None]).all()
        excess = 2.0**-4 * np.maximum(np.abs(lower), np.abs(upper)) + 2.0**-9 * scale if kind == "e4m3" else np.broadcast_to(scale, lower.shape)
        assert (stored >= (lower - excess)[:, None]).all() and (stored <= (upper + excess)[:, None]).all()
        q = rng.standard_normal((20, d))
        for h in range(heads):
            score = np.maximum(q * lower[h], q * upper[h]).sum(1)
            sums = 1e-12 * np.abs(q) @ np.maximum(np.abs(lower[h]), np.abs(upper[h]))  # (of the 64-bit sums here)
            assert ((q @ given[h].T).max(1) <= score + sums).all()
            assert ((q @ stored[h].T).max(1) <= score + np.abs(q) @ excess[h] + sums).all()
        beyond += int((stored > upper[:, None]).sum() + (stored < lower[:, None]).sum())
    assert n == page and beyond > 0
