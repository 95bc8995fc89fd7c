"""The kernel that attends for prompts, in every form: head sizes, pages, code types, joined ranges, windows, ragged rows, values that are not numbers.
(tests/test_pages_plan.py checks that these cases are given to that kernel, and into how many ranges.)"""
import math

import numpy as np
import pytest
import torch

from tests import test_gpu_pages as T

pytestmark = pytest.mark.gpu

tq = pytest.importorskip("paper_2504_19874_amd")

DEV, ints = T.DEV, T.ints

# d, page, cache, heads, query heads of each, lengths, new rows, window, ranges
CASES = [
    (256, 32, "e4m3", 8, 1, [70 + 13 * i for i in range(26)], [70 - i for i in range(26)], 0, 1),
    (256, 16, "int8", 4, 3, [257] * 48, [26 - i % 3 for i in range(48)], 31, 1),
    (256, 128, "e4m3", 8, 2, [200 + 7 * i for i in range(12)], [100 + 8 * i for i in range(12)], 0, 1),
    (256, 64, "int8", 8, 5, [300, 5, 141, 0] * 6, [27, 5, 14, 0] * 6, 0, 1),
    (256, 64, "e4m3", 4, 1, [6300, 66, 3000, 1, 70, 0, 129, 5], [66, 66, 1, 1, 66, 0, 65, 5], 0, 7),
    (256, 16, "int8", 4, 2, [5300, 33, 2000, 1, 70, 40, 129, 5], [33, 33, 1, 1, 33, 33, 30, 5], 5200, 6),
    (128, 128, "int8", 8, 4, [129, 300, 17, 128] * 4, [65, 20, 17, 64] * 4, 0, 1),
    (128, 128, "e4m3", 4, 16, [129, 300, 140, 257] * 8, [65, 20, 17, 40] * 8, 100, 1),
    (128, 16, "e4m3", 8, 3, [90 + i for i in range(20)], [30 - i % 7 for i in range(20)], 1, 1),
    (128, 64, "int8", 8, 1, [3300, 66, 2100, 64, 70, 5], [66, 66, 66, 64, 1, 5], 3000, 3),
    (64, 64, "e4m3", 4, 1, [4100, 66, 3000, 0] + [80 + i for i in range(12)], [66, 66, 66, 0] + [66 - i for i in range(12)], 2500, 3),
    (64, 128, "int8", 8, 2, [2300, 150, 200], [150, 150, 20], 0, 3),
    (64, 16, "int8", 8, 9, [100, 33, 8, 250] * 6, [8, 8, 8, 8] * 6, 0, 1),
    # rows before the first token, a row more than a tile, one row fewer
    (256, 32, "int8", 8, 1, [3, 129, 127, 128] * 3, [129, 129, 127, 128] * 3, 0, 1),
    (64, 32, "e4m3", 8, 1, [3, 257, 255, 256] * 3, [257, 257, 255, 256] * 3, 0, 1),
    (128, 32, "e4m3", 8, 1, [3, 257, 255, 256] * 3, [257, 257, 255, 256] * 3, 0, 1),
]


@pytest.mark.parametrize("case", CASES)
def test_prompts(case):
    d, page, kind, heads, group, lens, new, window, _ = case
    T.run_attend(12, d, page, kind, "bf16", heads, group, lens, new, window)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_logits_far_apart(d):
    """A frame that moves many times, and weights that leave the type's range."""
    T.run_attend(13, d, 16, "e4m3", "bf16", 8, 1, [200 + 3 * i for i in range(24)], [70] * 24, gain=30.0)
    T.run_attend(14, d, 32, "int8", "bf16", 8, 1, [150 + 3 * i for i in range(24)], [70] * 24, scale=-0.3)


SEQS, NEW, HEADS, PAGE = 24, 70, 8, 16  # of the tests below; d = 256: as many as that kernel is taken for


def prompts(seed, d, n, kind="e4m3"):
    rng = np.random.default_rng([seed, d])
    b = T.Batch(rng, [n] * SEQS, [NEW] * SEQS, PAGE)
    p = T.filled(rng, b, HEADS, d, kind)
    return b, p, torch.from_numpy(rng.standard_normal((b.rows, HEADS, d)).astype(np.float32)).to(DEV, torch.bfloat16)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 40])
def test_values_that_are_not_numbers(d, window):
    """A NaN in one coordinate of one key's values, every place of a tile in turn: that coordinate of the rows that see it, and what other
    rows have keeps its bits."""
    n = 150
    b, p, q = prompts(15, d, n)

    def run():
        out = torch.empty_like(q)
        tq.tq_pages_attend(p, q, *b.args(), 0.1, out, window=window)
        return out.view(SEQS, NEW, HEADS, d).float()

    clean, values = run(), p.v.view(torch.uint8).clone()
    pos = torch.arange(n - NEW, n, device=DEV)
    for turn in range(6):
        at = [(turn * SEQS + s) % 144 for s in range(SEQS)]
        p.v.view(torch.uint8).copy_(values)
        for s in range(SEQS):
            p.v.view(torch.uint8)[b.table[s][at[s] // PAGE], :, at[s] % PAGE, (37 * s + turn) % d] = 0x7f if s % 2 else 0xff
        got = run()
        for s in range(SEQS):
            sees = (pos >= at[s]) & ((pos - at[s] < window) if window else True)
            assert torch.equal(got[s][~sees], clean[s][~sees]), (turn, s)
            assert got[s][sees][..., (37 * s + turn) % d].isnan().all(), (turn, s)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_keys_that_are_not_numbers(d):
    n = 100
    b, p, q = prompts(16, d, n)

    def run():
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
        tq.tq_pages_attend(p, q, *b.args(), 0.1, out, lse=lse)
        return out.view(SEQS, NEW, HEADS, d).float(), lse.view(SEQS, NEW, HEADS)

    clean = run()
    for s in range(SEQS):
        p.k.view(torch.uint8)[b.table[s][(n - 1 - 2 * s) // PAGE], :, (n - 1 - 2 * s) % PAGE, 5 * s % d] = 0x7f
    got = run()
    for s in range(SEQS):
        sees = torch.arange(n - NEW, n, device=DEV) >= n - 1 - 2 * s
        assert torch.equal(got[0][s][~sees], clean[0][s][~sees]) and torch.equal(got[1][s][~sees], clean[1][s][~sees])
        assert got[0][s][sees].isnan().all() and got[1][s][sees].isnan().all() and sees.any()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_rows_of_no_sequence_are_left_alone(d):
    b, p, q = prompts(17, d, 90, "int8")
    table, lens, starts, most = b.args()
    want = torch.empty_like(q)
    tq.tq_pages_attend(p, q, table, lens, starts, most, 0.1, want)
    wide = torch.zeros((b.rows + 5, HEADS, d), dtype=torch.bfloat16, device=DEV)
    wide[2:-3] = q
    out, lse = torch.full_like(wide, 7.0), torch.full(wide.shape[:2], 7.0, device=DEV)
    tq.tq_pages_attend(p, wide, table, lens, starts + 2, most, 0.1, out, lse=lse)
    assert torch.equal(out[2:-3], want) and (lse[2:-3] != 7).all()
    for x in (out, lse):
        assert (x[:2] == 7).all() and (x[-3:] == 7).all()
    # rows outside of the arrays: those that are inside are as ever
    cut = torch.full_like(q, 7.0)
    tq.tq_pages_attend(p, q[:-30], table, lens, starts, most, 0.1, cut[:-30])
    assert torch.equal(cut[:-30], want[:-30]) and (cut[-30:] == 7).all()
    # no more than max_new of a sequence's rows
    few = torch.full_like(q, 7.0)
    tq.tq_pages_attend(p, q, table, lens, starts, 67, 0.1, few)
    few, want = few.view(SEQS, NEW, HEADS, d), want.view(SEQS, NEW, HEADS, d)
    assert torch.equal(few[:, :67], want[:, :67]) and (few[:, 67:] == 7).all()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_views_without_starts(d):
    b, p, q = prompts(18, d, 90)
    table, lens, starts, most = b.args()
    want, lse = torch.empty_like(q), [torch.empty(q.shape[:2], device=DEV) for _ in range(2)]
    tq.tq_pages_attend(p, q, table, lens, starts, most, 0.1, want, lse=lse[0])
    wide = torch.full((b.rows, HEADS + 2, d + 16), math.nan, dtype=torch.bfloat16, device=DEV)
    wide[:, 1:-1, 8:-8] = q
    out = torch.full((HEADS, b.rows, d + 8), 7.0, dtype=torch.bfloat16, device=DEV)
    tq.tq_pages_attend(p, wide[:, 1:-1, 8:-8], table, lens, None, most, 0.1, out.transpose(0, 1)[..., :d], lse=lse[1])
    assert torch.equal(out.transpose(0, 1)[..., :d], want) and (out[..., d:] == 7).all() and torch.equal(*lse)
