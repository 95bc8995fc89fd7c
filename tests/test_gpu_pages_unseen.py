"""What a row of attention over pages does not see does not reach it: scales of pages behind it, places of the table that are no page."""
import math

import numpy as np
import pytest
import torch

from tests import test_gpu_pages as T

pytestmark = pytest.mark.gpu

tq = pytest.importorskip("paper_2504_19874_amd")

DEV, ints = T.DEV, T.ints
BAD = [0.0, math.nan, math.inf, -1.0]  # what a scale holds that append has not written


def queries(rng, rows, heads, d, dtype):
    return torch.from_numpy(rng.standard_normal((rows, heads, d)).astype(np.float32)).to(DEV, T.TYPES[dtype])


def attended(p, q, *args, **more):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    tq.tq_pages_attend(p, q, *args, 0.1, out, lse=lse, **more)
    return out, lse


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("kind,dtype,d", [("e4m3", "bf16", 128), ("int8", "f32", 64), ("int8", "bf16", 256)])
def test_scales_of_chosen_pages_behind_the_row(kind, dtype, d, bad):
    """A list with places behind the row's position, whose pages nothing was ever appended to: the same bits as without them."""
    rng = np.random.default_rng([81, d])
    heads, page = 2, 16
    b = T.Batch(rng, [100, 40], [3, 1], page, spare=6, wide=0)
    p = T.filled(rng, b, heads, d, kind)
    table, lens, starts, most = b.args()
    free = sorted(set(range(b.n_pages)) - {x for row in b.table for x in row[:-(-100 // page)] if 0 <= x < b.n_pages})[:2]
    table = torch.cat([table, ints([free] * 2)], 1)
    for t in (p.k_scale, p.v_scale):
        t[free] = bad
    width = table.shape[1]
    q = queries(rng, b.rows, 2 * heads, d, dtype)
    pick = ints([[[0, 2, width - 2, 1, width - 1, 6]] * heads] * b.rows)
    plain = torch.where(pick >= width - 2, -1, pick)
    got, want = attended(p, q, table, lens, starts, most, chosen=pick), attended(p, q, table, lens, starts, most, chosen=plain)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not got[0].isnan().any()


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("d,dtype,seqs,new", [(128, "bf16", 1, 3), (64, "f32", 2, 20), (64, "bf16", 24, 70), (128, "bf16", 24, 70), (256, "bf16", 24, 70)])
def test_scales_of_pages_that_the_window_has_left(d, dtype, seqs, new, bad):
    """Pages of 16 before every row's window, given to somebody else since: their scales are anything."""
    rng = np.random.default_rng([82, d, seqs])
    heads, page, window, n = 8, 16, 20, 150
    b = T.Batch(rng, [n] * seqs, [new] * seqs, page)
    p = T.filled(rng, b, heads, d, "int8")
    q = queries(rng, b.rows, heads, d, dtype)
    want = attended(p, q, *b.args(), window=window)
    gone = (n - new - window + 1) // page  # whole pages before the first row's first key
    assert gone > 0
    for row in b.table:
        for t in (p.k_scale, p.v_scale):
            t[row[:gone]] = bad
    got = attended(p, q, *b.args(), window=window)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not got[0].isnan().any()


@pytest.mark.parametrize("d,dtype,seqs,new", [(128, "bf16", 1, 40), (64, "f32", 1, 40), (64, "bf16", 24, 70), (128, "bf16", 24, 70), (256, "bf16", 24, 70)])
def test_a_scale_that_some_rows_see(d, dtype, seqs, new):
    """A scale that is not a number makes the rows that see its page NaN, and no others, also among the rows of one tile."""
    rng = np.random.default_rng([83, d, seqs])
    heads, page, n = 8, 16, 96
    b = T.Batch(rng, [n] * seqs, [new] * seqs, page)
    p = T.filled(rng, b, heads, d, "e4m3")
    q = queries(rng, b.rows, heads, d, dtype)
    want = attended(p, q, *b.args())
    last = [row[n // page - 1] for row in b.table]
    for bad in (math.nan, 0.0):
        p.v_scale[last] = bad
        got = attended(p, q, *b.args())
        sees = (torch.arange(n - new, n, device=DEV) >= n - page).repeat(seqs)
        assert torch.equal(got[0][~sees], want[0][~sees]) and torch.equal(got[1][~sees], want[1][~sees])
        assert got[0][sees].isnan().all() and got[1][sees].isnan().all()


SHAPES = [(128, "bf16", 1, 3), (64, "f32", 2, 20), (256, "bf16", 1, 1), (64, "bf16", 24, 70), (128, "bf16", 24, 70), (256, "bf16", 24, 70)]


@pytest.mark.parametrize("window", [0, 2**31 - 1, 9])
@pytest.mark.parametrize("d,dtype,seqs,new", SHAPES)
def test_the_largest_lengths_over_places_that_are_no_page(d, dtype, seqs, new, window):
    """Lengths up to 2^31 - 1: what is no page is not there, whatever the pool's first tokens are; what is a page is seen whole."""
    rng = np.random.default_rng([84, d, seqs])
    heads, page = 8, 16
    b = T.Batch(rng, [48] * seqs, [new] * seqs, page, spare=2, wide=0)
    p = T.filled(rng, b, heads, d, "e4m3")
    table, _, starts, most = b.args()
    q = queries(rng, b.rows, heads, d, dtype)
    none = torch.full_like(table, -1)
    pick = ints([[[0, 1, 2]] * heads] * b.rows)
    for n in (2**31 - 1, 2**31 - 1000, 0x70000000, 0x70000000 + new - 1):
        lens = torch.full((seqs,), n, dtype=torch.int32, device=DEV)
        for more in ({}, {"chosen": pick}):
            out, lse = attended(p, q, none, lens, starts, most, window=window, **more)
            assert (out == 0).all() and (lse == -math.inf).all(), n
            holes = table.clone()
            holes[:, 1] = -1
            got = attended(p, q, holes, lens, starts, most, window=window, **more)
            want = attended(p, q, holes, ints([1000] * seqs), starts, most, window=0 if window > 9 else window, **more)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), n


@pytest.mark.parametrize("d,dtype,seqs,new", SHAPES)
def test_the_smallest_lengths(d, dtype, seqs, new):
    """Rows whose positions lie below -2^31 see nothing, and choose nothing."""
    rng = np.random.default_rng([85, d, seqs])
    heads, page = 8, 16
    b = T.Batch(rng, [48] * seqs, [new] * seqs, page, spare=2, wide=0)
    p = T.filled(rng, b, heads, d, "e4m3")
    p = tq.Pages(p.k, p.v, p.k_scale, p.v_scale, bounds=torch.zeros((b.n_pages, heads, 2, d), dtype=torch.bfloat16, device=DEV))
    table, _, starts, most = b.args()
    q = queries(rng, b.rows, heads, d, dtype)
    lens = torch.full((seqs,), -2**31, dtype=torch.int32, device=DEV)
    for more in ({}, {"chosen": ints([[[0, 1, 2]] * heads] * b.rows)}):
        out, lse = attended(p, q, table, lens, starts, most, **more)
        assert (out == 0).all() and (lse == -math.inf).all()
    chosen = torch.full((b.rows, heads, 3), 7, dtype=torch.int32, device=DEV)
    tq.tq_pages_select(p, q, table, lens, starts, most, chosen)
    assert (chosen == -1).all()
