"""GPU parity of the paged 8-bit cache (tq_pages_*) against its definition in 64 bits.

Appending is exact: a scale is a power of two, a value over it is exact in fp32 and rounded to its code once, so codes, scales and
bounds are compared for equality.

Attending.  With u = 2^-24: a logit is an fp32 sum of d products, off by at most (d + 8) u of scale sum |q_c k_c| =: reach (8: the
products with scale and the logarithm's factor, the sum with the frame), so weights move by exp(2 (d + 8) u reach) at most; a
weight is rounded to 2^-11 (bf16 output) or 2^-22 (fp32) and its exponential is good to 4 u; sums over n keys are made of
n / 32 products of 32, in up to 2 n / 32 + 64 additions of u each.  All of that is relative to sum_j p_j |v_j|; the output's own
rounding is half a step, eps / 2.  lse: the logits' error, the sums' and 4 u of its own size.

That leaves the weights below fp16's normal range, whose error is absolute: half of 2^-24, with one piece or two.  The kernel's weight of key
j is 2^x with the scale of its value block in x, and its frame puts the largest such weight of a row at 2^7 or above (a frame is taken at
2^7 and kept until a weight passes 2^15).  So in units of p_j v_scale_j every weight is off by 2^-25 / 2^7 = 2^-32 of the largest of
these, and the sum over the keys by 2^-32 max_j(p_j v_scale_j) sum_j |code_j|: `floor`.  It is what is left of a coordinate
where the codes of all weighty keys are zero.
"""
import math

import numpy as np
import pytest
import torch

from oracle import pages_oracle as po

pytestmark = pytest.mark.gpu

tq = pytest.importorskip("paper_2504_19874_amd")

DEV = "cuda"
KINDS = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def as64(codes):
    return (codes.float() if codes.dtype != torch.int8 else codes).double().cpu().numpy()


def to_codes(x, kind):
    t = torch.from_numpy(np.asarray(x, np.float32))
    return t.to(KINDS[kind]).to(DEV) if kind == "e4m3" else t.to(torch.int8).to(DEV)


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def random_codes(rng, shape, kind, stale=True):
    """Any code, NaN among the e4m3 ones where nothing is stored yet."""
    raw = rng.integers(0, 256, shape).astype(np.uint8)
    if kind == "int8":
        raw[raw == 128] = 0
    elif not stale:
        raw[(raw & 0x7f) == 0x7f] = 0
    return torch.from_numpy(raw).to(DEV).view(KINDS[kind])


class Batch:
    """Sequences of given lengths and new rows over scattered pages; what lies behind a length or in no page is garbage."""

    def __init__(self, rng, lens, new, page, spare=3, wide=2):
        self.lens, self.new, self.page = list(lens), list(new), page
        need = [-(-n // page) for n in lens]
        self.n_pages = max(1, sum(need) + spare)
        ids = iter(rng.permutation(self.n_pages).tolist())
        self.table = [[next(ids) for _ in range(k)] for k in need]
        width = max(need) + wide
        for i, row in enumerate(self.table):
            row += [[-1, self.n_pages, 2**30, -2**31][(i + j) % 4] for j in range(width - len(row))]
        self.starts = np.concatenate([[0], np.cumsum(new)]).tolist()
        self.rows, self.max_new = self.starts[-1], max(list(new) + [0])

    def args(self, starts=True):
        return ints(self.table), ints(self.lens), ints(self.starts) if starts else None, self.max_new


def filled(rng, b, heads, d, kind, bounds=False, gain=1.0):
    """A cache of normal keys and values with an outlier channel; slots that hold no token are anything."""
    shape = (b.n_pages, heads, b.page, d)
    k, v = rng.standard_normal(shape) * gain, rng.standard_normal(shape) * np.exp(rng.normal(0, 1, (b.n_pages, heads, 1, 1)))
    k[..., 3] *= 10
    stale = np.ones((b.n_pages, b.page), bool)
    for row, n in zip(b.table, b.lens):
        for i in range(-(-n // b.page)):
            stale[row[i], :min(b.page, n - i * b.page)] = False
    out = []
    for x in (k, v):
        scale = np.array([[po.scale_of(np.abs(y).max(), kind) for y in page] for page in x])
        codes = to_codes(po.round_code(x / scale[..., None, None], kind), kind)
        junk = random_codes(rng, shape, kind)
        mask = torch.from_numpy(stale).to(DEV)[:, None, :, None].expand(shape)
        codes = torch.where(mask, junk.view(torch.uint8), codes.view(torch.uint8)).view(KINDS[kind])
        empty = stale.all(1)
        scale[empty] = np.nan
        out += [codes.contiguous(), torch.from_numpy(scale.astype(np.float32)).to(DEV)]
    return tq.Pages(out[0], out[2], out[1], out[3])


def cache64(p):
    c = {"k": as64(p.k), "v": as64(p.v), "k_scale": as64(p.k_scale), "v_scale": as64(p.v_scale)}
    if p.bounds is not None:
        c["lower"], c["upper"] = as64(p.bounds[:, :, 0]), as64(p.bounds[:, :, 1])
    return c


def check_attend(out, lse, want, n_keys, kind_of_out):
    ref, ref_lse, size, reach, floor = want
    u, d = 2.0**-24, ref.shape[2]
    logit = (d + 8) * u * reach
    sums = (2 * n_keys / 32 + 64) * u
    weight = 2.0**-11 if kind_of_out == torch.bfloat16 else 2.0**-22
    rel = np.expm1(2 * logit) + weight + 4 * u + sums
    tol = rel[..., None] * size + 2.0**-32 * floor + torch.finfo(kind_of_out).eps / 2 * np.abs(ref)
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    bad = np.abs(got - ref) > tol + 1e-30
    assert not bad.any(), f"{bad.sum()} of {bad.size} outside, worst {np.nanmax(np.abs(got - ref) / (tol + 1e-30))}"
    if lse is not None:
        got = lse.double().cpu().numpy()
        assert np.array_equal(np.isneginf(got), np.isneginf(ref_lse)) and np.array_equal(np.isnan(got), np.isnan(ref_lse))
        fin = np.isfinite(ref_lse)
        got, ref_lse = np.where(fin, got, 0), np.where(fin, ref_lse, 0)
        tol = (logit + 4 * u + sums) + 4 * u * np.abs(ref_lse)
        assert (np.abs(got - ref_lse) <= tol)[fin].all()


def run_attend(seed, d, page, kind, dtype, heads, group, lens, new, window=0, scale=None, starts=True, chosen=None, gain=1.0):
    rng = np.random.default_rng([seed, d, page])
    b = Batch(rng, lens, new, page)
    p = filled(rng, b, heads, d, kind, gain=gain)
    q = torch.from_numpy(rng.standard_normal((b.rows, heads * group, d)).astype(np.float32)).to(DEV, TYPES[dtype])
    out = torch.full_like(q, math.nan)
    lse = torch.full(q.shape[:2], math.nan, device=DEV)
    scale = 1 / math.sqrt(d) if scale is None else scale
    pick = None
    if chosen:
        pick = rng.integers(-2, len(b.table[0]) + 2, (b.rows, heads, chosen))
        for r in pick.reshape(-1, chosen):  # places are in the list once
            _, first = np.unique(r, return_index=True)
            keep = np.zeros(chosen, bool)
            keep[first] = True
            r[~keep] = -1
    tq.tq_pages_attend(p, q, *b.args(starts), scale, out, lse=lse, window=window, chosen=None if pick is None else ints(pick))
    torch.cuda.synchronize()
    want = po.attend(cache64(p), page, q.double().cpu().numpy(), b.table, b.lens, b.starts, scale, window, pick)
    check_attend(out, lse, want, max(b.lens), TYPES[dtype])


ATTEND = [
    # d, page, cache, type, heads, query heads of each, lengths, new rows, window
    (128, 64, "e4m3", "bf16", 2, 4, [1, 33, 64, 65, 200], [1, 1, 1, 1, 1], 0),
    (128, 64, "int8", "bf16", 2, 4, [1, 33, 64, 65, 200], [1, 1, 1, 1, 1], 0),
    (128, 16, "e4m3", "f32", 1, 1, [31, 0, 17], [1, 0, 1], 0),
    (64, 16, "int8", "f32", 3, 5, [100, 7, 513], [17, 7, 1], 0),
    (64, 32, "e4m3", "bf16", 1, 16, [95, 300], [3, 40], 0),
    (64, 128, "e4m3", "f32", 2, 17, [130, 1], [2, 1], 0),
    (256, 128, "e4m3", "bf16", 1, 2, [129, 260, 3], [5, 33, 3], 0),
    (256, 32, "int8", "f32", 1, 3, [150], [9], 0),
    (128, 64, "e4m3", "bf16", 1, 8, [300, 70], [70, 70], 0),
    (128, 32, "int8", "bf16", 2, 1, [257, 129], [129, 129], 0),
    (128, 16, "e4m3", "f32", 1, 2, [333, 40], [100, 40], 50),
    (128, 64, "e4m3", "bf16", 2, 4, [500, 20], [1, 1], 100),
    (64, 64, "int8", "bf16", 1, 4, [200, 64], [65, 1], 1),
    (128, 64, "e4m3", "f32", 2, 4, [2100], [2], 0),
    # keys in ranges that a second launch joins
    (64, 16, "int8", "bf16", 2, 4, [1000, 5, 900], [1, 2, 1], 0),
    (64, 32, "e4m3", "f32", 1, 3, [1500, 31], [7, 1], 0),
    (128, 32, "int8", "f32", 2, 1, [1300, 0, 1], [1, 0, 1], 700),
    (256, 16, "e4m3", "bf16", 1, 5, [1200, 800], [4, 1], 0),
    (256, 64, "int8", "f32", 3, 2, [700], [3], 0),
    # rows at positions below zero
    (128, 16, "e4m3", "bf16", 1, 2, [3, 0], [5, 2], 0),
]


@pytest.mark.parametrize("case", ATTEND)
def test_attend(case):
    d, page, kind, dtype, heads, group, lens, new, window = case
    run_attend(1, d, page, kind, dtype, heads, group, lens, new, window)


PROMPTS = [  # more than 64 rows to a head, half the compute units with a workgroup: the kernel for prompts
    (128, 64, "e4m3", 8, 1, [70 + 13 * i for i in range(16)], [70 - i for i in range(16)], 0),
    (128, 16, "int8", 8, 1, [90 + 13 * i for i in range(16)], [65] * 16, 30),
    (64, 16, "e4m3", 4, 3, [257] * 32, [26 - i % 3 for i in range(32)], 0),
    (64, 32, "int8", 16, 2, [33 + i for i in range(8)], [33] * 8, 7),
    (128, 128, "int8", 4, 16, [129] * 2 + [300], [129, 65, 67], 0),
    (128, 64, "e4m3", 8, 1, [4100, 66, 3000, 1], [66, 66, 1, 1], 0),  # keys in ranges
    (64, 64, "e4m3", 8, 1, [4100, 66, 3000, 0], [66, 66, 66, 0], 2500),
    (256, 32, "e4m3", 8, 1, [70 + 13 * i for i in range(16)], [70 - i for i in range(16)], 0),
    (256, 16, "int8", 4, 3, [257] * 32, [26 - i % 3 for i in range(32)], 31),
    (256, 64, "e4m3", 8, 1, [4100, 66, 3000, 1], [66, 66, 1, 1], 0),
]


@pytest.mark.parametrize("case", PROMPTS)
def test_prompts(case):
    d, page, kind, heads, group, lens, new, window = case
    run_attend(8, d, page, kind, "bf16", heads, group, lens, new, window)


@pytest.mark.parametrize("kind,group,new,chosen", [("e4m3", 4, 5, 0), ("int8", 3, 11, 0), ("e4m3", 20, 2, 40)])
def test_more_than_16_rows_of_many_sequences(kind, group, new, chosen):
    """32 rows to a workgroup."""
    n = 40 if chosen else 64
    lens = [7 + 9 * i for i in range(n - 1)] + [600]
    run_attend(9, 128, 16, kind, "bf16", 8, group, lens, [min(new, m) for m in lens], chosen=chosen or None)


@pytest.mark.parametrize("d,dtype,seqs,new", [(128, "bf16", 1, 7), (64, "f32", 1, 20), (128, "bf16", 20, 70), (64, "bf16", 20, 70), (256, "bf16", 20, 70)])
def test_what_a_row_does_not_see_does_not_reach_it(d, dtype, seqs, new):
    """NaN among later tokens' keys and values, in what a window has left behind, and behind the last token: rows that see none of it have
    the same bits as without it.  A NaN key makes a row NaN; a NaN value its coordinate, or the row."""
    rng = np.random.default_rng([41, d, seqs])
    page, heads, window = 16, 8, 40
    b = Batch(rng, [100] * seqs, [new] * seqs, page)
    p = filled(rng, b, heads, d, "e4m3")
    q = torch.from_numpy(rng.standard_normal((b.rows, heads, d)).astype(np.float32)).to(DEV, TYPES[dtype])

    def run():
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
        tq.tq_pages_attend(p, q, *b.args(), 0.1, out, lse=lse, window=window)
        return out.view(seqs, new, heads, d).float(), lse.view(seqs, new, heads)

    clean, clean_lse = run()
    at = {"k": 97, "v": 95, "old": 100 - new - window}  # the last position is 99, the first row's 100 - new
    for s in range(seqs):
        p.k.view(torch.uint8)[b.table[s][at["k"] // page], :, at["k"] % page, 5] = 0x7f
        p.v.view(torch.uint8)[b.table[s][at["v"] // page], :, at["v"] % page, 7] = 0xff
        if at["old"] >= 0:
            p.v.view(torch.uint8)[b.table[s][at["old"] // page], :, at["old"] % page] = 0x7f
    got, got_lse = run()
    pos = torch.arange(100 - new, 100, device=DEV)
    sees_v = (pos >= at["v"]) & (pos - window < at["v"])
    sees_k = (pos >= at["k"]) & (pos - window < at["k"])
    if at["old"] >= 0:
        assert not ((pos >= at["old"]) & (pos - window < at["old"])).any()
    assert torch.equal(got[:, ~(sees_v | sees_k)], clean[:, ~(sees_v | sees_k)]) and torch.equal(got_lse[:, ~(sees_v | sees_k)], clean_lse[:, ~(sees_v | sees_k)])
    assert got[:, sees_k].isnan().all() and got_lse[:, sees_k].isnan().all()
    assert got[:, sees_v][..., 7].isnan().all() and sees_v.any() and sees_k.any()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("window", [0, 40])
def test_prompts_over_values_that_are_not_numbers(d, window):
    """A NaN in one coordinate of one key's values, every place of a tile in turn: that coordinate of the rows that see it, and what other
    rows have keeps its bits."""
    rng = np.random.default_rng([43, d, window])
    page, heads, seqs, new, n = 16, 8, 20, 70, 150
    b = Batch(rng, [n] * seqs, [new] * seqs, page)
    p = filled(rng, b, heads, d, "e4m3")
    q = torch.from_numpy(rng.standard_normal((b.rows, heads, d)).astype(np.float32)).to(DEV, torch.bfloat16)

    def run():
        out = torch.empty_like(q)
        tq.tq_pages_attend(p, q, *b.args(), 0.1, out, window=window)
        return out.view(seqs, new, heads, d).float()

    clean = run()
    at = [(17 * s + 3) % n if s < 4 else n - 1 - 7 * s % 130 for s in range(seqs)]
    for s in range(seqs):
        p.v.view(torch.uint8)[b.table[s][at[s] // page], :, at[s] % page, s % d] = 0x7f if s % 2 else 0xff
    got = run()
    pos = torch.arange(n - new, n, device=DEV)
    for s in range(seqs):
        sees = (pos >= at[s]) & ((pos - at[s] < window) if window else True)
        assert torch.equal(got[s][~sees], clean[s][~sees]), s
        assert got[s][sees][..., s % d].isnan().all(), s
    assert sees.any()


@pytest.mark.parametrize("d,page,kind,dtype,group,lens,new,n", [
    (128, 64, "e4m3", "bf16", 4, [700, 90], [1, 1], 5), (64, 16, "int8", "f32", 3, [300, 33], [4, 2], 9),
    (256, 32, "e4m3", "f32", 20, [200], [2], 1), (128, 16, "int8", "bf16", 16, [999], [3], 40),
    (64, 16, "e4m3", "f32", 2, [1500, 60], [2, 1], 64), (256, 64, "int8", "bf16", 3, [2000], [3], 20)])
def test_attend_over_chosen_pages(d, page, kind, dtype, group, lens, new, n):
    run_attend(2, d, page, kind, dtype, 2, group, lens, new, chosen=n)


def test_attend_with_logits_far_apart():
    """Weights that leave fp32's range; a frame that moves many times."""
    run_attend(3, 128, 16, "e4m3", "f32", 1, 4, [400, 77], [1, 5], gain=30.0)
    run_attend(4, 64, 32, "int8", "bf16", 1, 4, [400, 77], [1, 5], gain=30.0)
    run_attend(5, 64, 32, "int8", "f32", 1, 4, [400, 77], [1, 5], scale=0.0)
    run_attend(6, 64, 32, "int8", "f32", 1, 4, [400, 77], [1, 5], scale=-0.3)


def test_attend_without_starts():
    run_attend(7, 128, 64, "e4m3", "bf16", 2, 4, [100, 65, 2], [2, 2, 2], starts=False)


APPEND = [
    (128, 64, "e4m3", "bf16", 2, [1, 64, 65, 130], [1, 1, 1, 1]),
    (128, 64, "int8", "f32", 2, [1, 64, 65, 130], [1, 1, 1, 1]),
    (64, 16, "e4m3", "f32", 3, [100, 16, 40], [100, 7, 33]),
    (64, 16, "int8", "bf16", 1, [100, 0, 40], [61, 0, 3]),
    (256, 128, "e4m3", "bf16", 1, [300, 128], [290, 128]),
    (256, 32, "int8", "f32", 2, [77], [50]),
    (128, 128, "int8", "bf16", 1, [500, 3], [255, 5]),
]


@pytest.mark.parametrize("case", APPEND)
def test_append(case):
    d, page, kind, dtype, heads, lens, new = case
    rng = np.random.default_rng([11, d, page])
    b = Batch(rng, lens, new, page)
    shape = (b.n_pages, heads, page, d)
    k, v = random_codes(rng, shape, kind, False), random_codes(rng, shape, kind, False)
    scales = [torch.from_numpy(2.0**rng.integers(-9, 2, shape[:2])).to(DEV, torch.float32) for _ in range(2)]
    bounds = torch.from_numpy(np.sort(rng.standard_normal((b.n_pages, heads, 2, d)), 2)).to(DEV, torch.bfloat16)
    p = tq.Pages(k, v, *scales, bounds=bounds)
    x = [torch.from_numpy((rng.standard_normal((b.rows, heads, d)) * np.exp(rng.normal(0, 2, (b.rows, heads, 1)))).astype(np.float32)).to(DEV, TYPES[dtype])
         for _ in range(2)]
    want = cache64(p)
    po.append(want, kind, page, *[t.double().cpu().numpy() for t in x], b.table, b.lens, b.starts)
    tq.tq_pages_append(p, *x, *b.args())
    torch.cuda.synchronize()
    got = cache64(p)
    for name in want:
        assert np.array_equal(got[name], want[name]), name


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_scales_and_codes_on_either_side_of_a_step(kind):
    """A page of one row for every case: amax on, just below and just above what a scale can hold, the ends of the exponents, ties between
    codes, subnormal codes, zeros, and values that are not finite."""
    top = np.float32(po.TOP[kind])
    rows = [[x] for e in (-46, -41, -40, -39, -3, 0, 5, 39, 40, 41, 90) for x in (np.float32(2.0**e) * top, np.nextafter(np.float32(2.0**e) * top, np.float32(0)),
                                                                                     np.nextafter(np.float32(2.0**e) * top, np.float32(np.inf)))]
    rows += [[top, x] for x in np.float32([0.5, 1.5, 2.5, 2.0**-10, 1.5 * 2.0**-9, 2.5 * 2.0**-9, 2.0**-6 * 1.0625, 17, 19, 18, 126.5, 416, 432, 440])]
    rows += [[0.0], [np.inf], [np.inf, 3.0], [-np.inf, 1e-3], [np.nan], [np.nan, 5.0], [np.nan, np.inf, -2.0], [1e-42], [3e38, 1.0]]
    x = np.zeros((len(rows), 1, 64), np.float32)
    for i, r in enumerate(rows):
        x[i, 0, :len(r)] = r
        x[i, 0, 32:32 + len(r)] = np.negative(r)
    n = len(rows)
    p = tq.make_pages(n, 1, 64, 16, dtype=KINDS[kind], bounds=True, device=DEV)
    want = cache64(p)
    table, lens, starts = [[i] for i in range(n)], [1] * n, list(range(n + 1))
    po.append(want, kind, 16, x.astype(np.float64), x.astype(np.float64), table, lens, starts)
    tq.tq_pages_append(p, *[torch.from_numpy(x).to(DEV)] * 2, ints(table), ints(lens), None, 1)
    torch.cuda.synchronize()
    got = cache64(p)
    for name in want:
        assert np.array_equal(got[name], want[name], equal_nan=True), (name, np.argwhere(~((got[name] == want[name]) | np.isnan(want[name])))[:5])


@pytest.mark.parametrize("kind", ["e4m3", "int8"])
def test_a_scale_that_append_has_not_made(kind):
    """It is taken up to a power of two; what was there moves by half a step of its code at most (and u of the product before)."""
    rng = np.random.default_rng(51)
    p = tq.make_pages(2, 1, 64, 16, dtype=KINDS[kind], device=DEV)
    p.k.copy_(random_codes(rng, p.k.shape, kind, False)), p.v.copy_(p.k)
    p.k_scale.fill_(0.3), p.v_scale.fill_(3.0)
    before = cache64(p)
    x = torch.from_numpy(rng.standard_normal((1, 1, 64)).astype(np.float32)).to(DEV)
    tq.tq_pages_append(p, x, x, ints([[1]]), ints([11]), None, 1)
    got = cache64(p)
    assert got["k_scale"][1, 0] == 0.5 and got["v_scale"][1, 0] == 4.0
    for name, to in (("k", 0.5), ("v", 4.0)):
        was = before[name][1, 0, :10] * before[name + "_scale"][1, 0]
        step = to * (1.0 if kind == "int8" else np.maximum(2.0**-9, 2.0**-3 * np.abs(was / to)))
        assert (np.abs(got[name][1, 0, :10] * to - was) <= step / 2 * (1 + 2.0**-20) + 2.0**-23 * np.abs(was)).all()
        assert np.array_equal(got[name][1, 0, 11:], before[name][1, 0, 11:]) and np.array_equal(got[name][0], before[name][0])


SELECT = [
    (128, 64, "bf16", 2, 4, [1, 64, 65, 2000], [1, 1, 1, 1], 5, 1, 1),
    (64, 16, "f32", 1, 3, [700, 100], [4, 1], 7, 0, 0),
    (256, 32, "bf16", 3, 1, [900, 31], [2, 2], 40, 2, 3),
    (64, 16, "bf16", 1, 16, [4000], [1], 64, 1, 2),
    (128, 16, "f32", 2, 2, [333, 20], [1, 3], 5, 2, 3),   # no room for others
    (128, 16, "bf16", 1, 5, [3, 0], [5, 2], 2, 0, 1),     # rows before the first token
    (256, 16, "f32", 1, 2, [20000], [1], 200, 0, 1),
]


@pytest.mark.parametrize("case", SELECT)
def test_select(case):
    d, page, dtype, heads, group, lens, new, n, first, last = case
    rng = np.random.default_rng([21, d, page])
    b = Batch(rng, lens, new, page)
    bounds = torch.from_numpy(np.sort(rng.standard_normal((b.n_pages, heads, 2, d)), 2)).to(DEV, torch.bfloat16)
    longest = b.table[int(np.argmax(lens))]
    if max(lens) > 2 * page:
        bounds[longest[0]] = bounds[longest[2]]  # equal scores
    zero = torch.zeros((b.n_pages, heads, page, d), dtype=torch.int8, device=DEV)
    ones = torch.ones((b.n_pages, heads), device=DEV)
    p = tq.Pages(zero, zero, ones, ones, bounds=bounds)
    q = torch.from_numpy(rng.standard_normal((b.rows, heads * group, d)).astype(np.float32)).to(DEV, TYPES[dtype])
    chosen = torch.full((b.rows, heads, n), -7, dtype=torch.int32, device=DEV)
    tq.tq_pages_select(p, q, *b.args(), chosen, keep_first=first, keep_last=last)
    torch.cuda.synchronize()
    c = cache64(p)
    want = po.select(c["lower"], c["upper"], page, q.double().cpu().numpy(), b.table, b.lens, b.starts, n, first, last)
    assert np.array_equal(chosen.cpu().numpy(), want)


def pool_state(rng, n_pages, rows, width, page, heads=2, d=64, kind="int8", live=None):
    """A pool with some sequences in it; every page's content is its own number."""
    order = rng.permutation(n_pages).tolist()
    table, lens = np.full((rows, width), -1), np.zeros(rows, int)
    refs = np.zeros(n_pages, int)
    for r in range(rows if live is None else live):
        lens[r] = rng.integers(0, width * page + 1)
        for i in range(-(-lens[r] // page)):
            if not order:
                lens[r] = i * page
                break
            table[r, i] = order.pop()
            refs[table[r, i]] = 1
    p = tq.make_pages(n_pages, heads, d, page, dtype=KINDS[kind], bounds=True, device=DEV)
    for t in (p.k, p.v):
        t.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 120, t.shape).astype(np.uint8)))
    for t in (p.k_scale, p.v_scale, p.bounds):
        t.copy_(torch.from_numpy(rng.random(t.shape)).to(t.dtype))
    p.refs.copy_(ints(refs))
    return p, po.Pool(table, lens, refs, page)


def contents(p):
    return [t.clone() if t.dtype != torch.float8_e4m3fn else t.view(torch.uint8).clone() for t in (p.k, p.v, p.k_scale, p.v_scale, p.bounds)]


def moved(before, pairs):
    if pairs:
        src, dst = (torch.tensor(x, device=DEV) for x in zip(*pairs))
        for t in before:
            t[dst] = t[src]
    return before


def same_pool(p, pool, table, lens):
    return np.array_equal(table.cpu().numpy(), pool.table) and np.array_equal(lens.cpu().numpy(), pool.lens) and np.array_equal(p.refs.cpu().numpy(), pool.refs)


@pytest.mark.parametrize("n_pages,rows,width,page", [(50, 6, 5, 16), (3000, 40, 60, 32), (20, 9, 4, 64)])
def test_pool(n_pages, rows, width, page):
    rng = np.random.default_rng([31, n_pages])
    p, pool = pool_state(rng, n_pages, rows, width, page, live=rows // 2)
    table, lens = ints(pool.table), ints(pool.lens)
    missing = torch.full((1,), -1, dtype=torch.int32, device=DEV)
    # fork: into the rows that hold nothing
    parents, children = rng.integers(0, rows // 2, rows - rows // 2), np.arange(rows // 2, rows)
    want = contents(p)
    pairs, short = pool.fork(parents, children)
    tq.tq_pages_fork(p, table, lens, ints(parents), ints(children), missing=missing)
    assert same_pool(p, pool, table, lens) and int(missing) == short
    assert all(torch.equal(a, b) for a, b in zip(contents(p), moved(want, pairs)))
    # grow
    grow = np.where(pool.lens + page + 3 <= width * page, page + 3, 0)
    pool.lens += grow
    lens += ints(grow)
    short = pool.reserve(page + 3)
    tq.tq_pages_reserve(p, table, lens, page + 3, missing=missing)
    assert same_pool(p, pool, table, lens) and int(missing) == short
    # end some, one of them twice, one that is none
    rows_gone = [0, rows - 1]
    pool.free(rows_gone)
    tq.tq_pages_free(p, table, lens, ints(rows_gone + [0, rows, -1]))
    assert same_pool(p, pool, table, lens)
    # make dense
    want = contents(p)
    pairs, live = pool.compact()
    tq.tq_pages_compact(p, table, n_live=missing)
    assert same_pool(p, pool, table, lens) and int(missing) == live
    got = contents(p)
    assert all(torch.equal(a, b) for a, b in zip(got, moved(want, pairs)))
    # and copies of pages
    src, dst = [0, 1, n_pages, 2], [n_pages - 1, n_pages - 2, 4, -1]
    tq.tq_pages_copy(p, ints(src), ints(dst))
    assert all(torch.equal(a, b) for a, b in zip(contents(p), moved(got, list(zip(src, dst))[:2])))


def test_forks_that_are_skipped():
    """Rows that are none, a child twice, a child with tokens, a row into itself, an empty parent that is a child as well."""
    rng = np.random.default_rng(33)
    p, pool = pool_state(rng, 60, 9, 5, 16, live=4)
    pool.lens[:4] = [40, 33, 80, 1]
    pool.table[:], pool.refs[:] = -1, 0
    for r in range(4):
        pool.table[r, :-(-pool.lens[r] // 16)] = np.arange(12 * r, 12 * r + -(-pool.lens[r] // 16))
    pool.refs[pool.table[pool.table >= 0]] = 1
    p.refs.copy_(ints(pool.refs))
    table, lens = ints(pool.table), ints(pool.lens)
    parents = [0, 1, 2, 9, -1, 0, 3, 2, 4, 5, 1, 3]
    children = [4, 4, 5, 6, 6, -2, 3, 1, 6, 7, 9, 4]
    want = contents(p)
    pairs, short = pool.fork(parents, children)
    missing = ints([-1])
    tq.tq_pages_fork(p, table, lens, ints(parents), ints(children), missing=missing)
    assert same_pool(p, pool, table, lens) and int(missing) == short
    assert all(torch.equal(a, b) for a, b in zip(contents(p), moved(want, pairs)))
    assert pool.lens.tolist() == [40, 33, 80, 1, 40, 80, 0, 0, 0]


def test_more_new_tokens_than_there_can_be():
    """max_new is a bound: one of 2^31 - 1 takes no longer."""
    most = 2**31 - 1
    rng = np.random.default_rng(35)
    p, pool = pool_state(rng, 40, 3, 6, 16, heads=1, live=0)
    pool.lens[:] = [90, 0, 33]
    table, lens, missing = ints(pool.table), ints(pool.lens), ints([-1])
    assert pool.reserve(most) == 0
    tq.tq_pages_reserve(p, table, lens, most, missing=missing)
    assert same_pool(p, pool, table, lens) and int(missing) == 0
    x = torch.from_numpy(rng.standard_normal((123, 1, 64)).astype(np.float32)).to(DEV)
    want = cache64(p)
    po.append(want, "int8", 16, *[x.double().cpu().numpy()] * 2, pool.table.tolist(), [90, 0, 33], [0, 90, 90, 123])
    tq.tq_pages_append(p, x, x, table, lens, ints([0, 90, 90, 123]), most)
    got = cache64(p)
    assert all(np.array_equal(got[n], want[n]) for n in want)


def test_many_forks_in_a_pool_that_runs_out():
    rng = np.random.default_rng(34)
    p, pool = pool_state(rng, 2100, 3003, 4, 16, heads=1, live=3)
    pool.lens[:3] = [17, 40, 15]
    pool.table[:], pool.refs[:] = -1, 0
    pool.table[0, :2], pool.table[1, :3], pool.table[2, :1] = [5, 7], [2099, 2000, 1], [1024]
    pool.refs[[5, 7, 2099, 2000, 1, 1024]] = 1
    p.refs.copy_(ints(pool.refs))
    table, lens = ints(pool.table), ints(pool.lens)
    parents, children = rng.integers(0, 3, 3000), 3 + rng.permutation(3000)
    want = contents(p)
    pairs, short = pool.fork(parents, children)
    missing = ints([-1])
    tq.tq_pages_fork(p, table, lens, ints(parents), ints(children), missing=missing)
    assert short > 0 and same_pool(p, pool, table, lens) and int(missing) == short
    assert all(torch.equal(a, b) for a, b in zip(contents(p), moved(want, pairs)))
    gone = rng.permutation(3003)[:2000]
    pool.free(gone)
    tq.tq_pages_free(p, table, lens, ints(gone))
    want = contents(p)
    pairs, live = pool.compact()
    tq.tq_pages_compact(p, table)
    assert same_pool(p, pool, table, lens)
    assert all(torch.equal(a, b) for a, b in zip(contents(p), moved(want, pairs)))
