"""The paged 8-bit cache in 64 bits, written from its definition: sequence by sequence, row by row, on the CPU.

A cache is a dict of float64 arrays of what the codes stand for before their scale: k, v [page][head][token][d], k_scale, v_scale
[page][head], lower, upper [page][head][d].  NaN is NaN."""
import numpy as np

TOP = {"e4m3": 448.0, "int8": 127.0}
LOW, HIGH = -40, 40


def round_code(x, kind):
    """To the nearest code, ties to the even one; beyond the largest the largest; NaN to NaN (int8: 0)."""
    x = np.asarray(x, np.float64)
    if kind == "int8":
        return np.nan_to_num(np.clip(np.rint(x), -127, 127), nan=0.0)
    out = np.array(x)
    fin = np.isfinite(x)
    e = np.frexp(np.where(fin, x, 0.0))[1] - 1  # 2^e <= |x| < 2^(e+1)
    step = np.ldexp(1.0, np.maximum(e, -6) - 3)  # three bits behind the leading one; subnormal steps of 2^-9
    out[fin] = (np.rint(x / step) * step)[fin]
    return np.clip(out, -448.0, 448.0)  # (NaN passes)


def scale_of(amax, kind):
    if not amax > 0:
        return 2.0**LOW
    e = LOW
    while e < HIGH and amax / 2.0**e > TOP[kind]:
        e += 1
    return 2.0**e


def bf16_outward(x, down):
    big = 3.3895313892515355e38
    x = float(min(max(x, -big), big))
    if x == 0:
        return 0.0
    step = np.ldexp(1.0, max(int(np.frexp(x)[1]) - 8, -133))
    return float((np.floor if down else np.ceil)(x / step) * step)


def append(cache, kind, page, rows_k, rows_v, table, lens, starts):
    """rows_k, rows_v [row][head][d] float64; changes the cache in place."""
    for s in range(len(lens)):
        count = starts[s + 1] - starts[s]
        begin = lens[s] - count
        for name, rows in (("k", rows_k), ("v", rows_v)):
            for first in range(0, lens[s], page):
                a, b = max(begin, first, 0), min(lens[s], first + page)
                i = first // page
                if a >= b or i >= len(table[s]) or not 0 <= table[s][i] < len(cache["k"]):
                    continue
                p, had = table[s][i], a - first
                x = rows[starts[s] + a - begin:starts[s] + b - begin]
                for h in range(x.shape[1]):
                    y = x[:, h]
                    fin = np.abs(y[np.isfinite(y)])
                    to = scale_of(fin.max() if fin.size else 0.0, kind)
                    if had:
                        was = cache[name + "_scale"][p, h]
                        to = max(to, was)
                        cache[name][p, h, :had] = round_code(cache[name][p, h, :had] * (was / to), kind)
                    cache[name][p, h, had:had + b - a] = round_code(y / to, kind)
                    cache[name + "_scale"][p, h] = to
                    if name == "k" and "lower" in cache:
                        for j in range(y.shape[1]):
                            v = y[:, j][~np.isnan(y[:, j])]
                            lo, hi = (bf16_outward(v.min(), True), bf16_outward(v.max(), False)) if v.size else (0.0, 0.0)
                            if had:
                                lo, hi = min(lo, cache["lower"][p, h, j]), max(hi, cache["upper"][p, h, j])
                            cache["lower"][p, h, j], cache["upper"][p, h, j] = lo, hi


def seen_keys(cache, page, table_row, pos, window, chosen=None):
    """(page, token of it) of every key that a row at position pos sees."""
    out = []
    for i in (range(len(table_row)) if chosen is None else chosen):
        if not 0 <= i < len(table_row) or not 0 <= table_row[i] < len(cache["k"]):
            continue
        for j in range(page):
            at = i * page + j
            if at <= pos and (not window or at > pos - window):
                out.append((table_row[i], j))
    return out


def attend(cache, page, q, table, lens, starts, scale, window=0, chosen=None):
    """-> out [row][head][d], lse [row][head], and what tolerances are made of: sum_j p_j |v_j| [row][head][d], the largest
    sum_c |q_c k_c| scale [row][head], and max_j(p_j v_scale_j) sum_j |code_j| [row][head][d]."""
    n, heads, d = q.shape
    kv = cache["k"].shape[1]
    out, lse = np.zeros((n, heads, d)), np.full((n, heads), -np.inf)
    size, reach, floor = np.zeros((n, heads, d)), np.zeros((n, heads)), np.zeros((n, heads, d))
    for s in range(len(lens)):
        count = starts[s + 1] - starts[s]
        for row in range(starts[s], starts[s + 1]):
            pos = lens[s] - count + row - starts[s]
            for h in range(kv):
                at = seen_keys(cache, page, table[s], pos, window, None if chosen is None else chosen[row][h])
                if not at:
                    continue
                p, j = np.array(at).T
                k, v = cache["k"][p, h, j] * cache["k_scale"][p, h][:, None], cache["v"][p, h, j] * cache["v_scale"][p, h][:, None]
                for i in range(h * heads // kv, (h + 1) * heads // kv):
                    with np.errstate(invalid="ignore"):
                        x = scale * (k @ q[row, i])
                        m = x.max()
                        w = np.exp(x - m)
                        out[row, i], lse[row, i] = w @ v / w.sum(), m + np.log(w.sum())
                        size[row, i], reach[row, i] = w @ np.abs(v) / w.sum(), abs(scale) * np.max(np.abs(k) @ np.abs(q[row, i]))
                        floor[row, i] = np.max(w * cache["v_scale"][p, h]) / w.sum() * np.abs(cache["v"][p, h, j]).sum(0)
    return out, lse, size, reach, floor


def select(lower, upper, page, q, table, lens, starts, n_chosen, keep_first, keep_last):
    n, heads, _ = q.shape
    kv = lower.shape[1]
    out = np.full((n, kv, n_chosen), -1, np.int32)
    for s in range(len(lens)):
        count = starts[s + 1] - starts[s]
        for row in range(starts[s], starts[s + 1]):
            pos = lens[s] - count + row - starts[s]
            last = pos // page if pos >= 0 else -1
            for h in range(kv):
                rank = []
                for i in range(min(last + 1, len(table[s]))):
                    p = table[s][i]
                    if not 0 <= p < len(lower):
                        continue
                    with np.errstate(invalid="ignore", over="ignore"):
                        x, lo, hi = q[row, h * heads // kv:(h + 1) * heads // kv], lower[p, h], upper[p, h]
                        terms = np.where((x == 0) & ~np.isnan(lo) & ~np.isnan(hi), 0.0, np.maximum(x * lo, x * hi))
                        score = terms.sum(1).astype(np.float32).max()  # (NaN of one head is the page's)
                    kept = i < keep_first or i > last - keep_last
                    rank.append((0, 0.0, i) if kept else (2, 0.0, i) if np.isnan(score) else (1, -score, i))
                best = sorted(r[-1] for r in sorted(rank)[:n_chosen])
                out[row, h, :len(best)] = best
    return out


class Pool:
    """Tables, lengths and counts, one step at a time; `moves` collects (from, to) of the contents."""

    def __init__(self, table, lens, refs, page):
        self.table, self.lens, self.refs, self.page = np.array(table), np.array(lens), np.array(refs), page

    def _take(self):
        free = np.flatnonzero(self.refs <= 0)
        if not free.size:
            return -1
        self.refs[free[0]] = 1
        return int(free[0])

    def reserve(self, max_new, starts=None):
        missing = 0
        for s in range(len(self.lens)):
            new = max_new if starts is None else min(max(starts[s + 1] - starts[s], 0), max_new)
            first = max(0, self.lens[s] - new)
            for i in range(first // self.page, -(-max(self.lens[s], 0) // self.page)):
                if new > 0 and i < self.table.shape[1] and not 0 <= self.table[s, i] < len(self.refs):
                    if i * self.page >= first:  # (else tokens before the new ones were there without a page)
                        self.table[s, i] = self._take()
                    missing += not 0 <= self.table[s, i] < len(self.refs)
        return missing

    def fork(self, parents, children):
        moves, missing = [], 0
        fresh, taken = {}, set()
        skip = []
        for p, c in zip(parents, children):
            skip.append(not (0 <= p < len(self.lens) and 0 <= c < len(self.lens)) or p == c or self.lens[c] > 0 or c in taken)
            if not skip[-1]:
                taken.add(c)
        before = np.maximum(self.lens, 0)
        for n, (p, c) in enumerate(zip(parents, children)):  # pages are given out before any count changes
            if skip[n]:
                continue
            full = before[p] // self.page
            if before[p] % self.page and full < self.table.shape[1] and 0 <= self.table[p, full] < len(self.refs):
                fresh[n] = self._take()
                missing += fresh[n] < 0
                if fresh[n] >= 0:
                    moves.append((int(self.table[p, full]), fresh[n]))
        for n, (p, c) in enumerate(zip(parents, children)):
            if skip[n]:
                continue
            full = min(before[p] // self.page, self.table.shape[1])
            self.table[c] = -1
            self.table[c, :full] = self.table[p, :full]
            for x in self.table[c, :full]:
                if 0 <= x < len(self.refs):
                    self.refs[x] += 1
            if full < self.table.shape[1]:
                self.table[c, full] = fresh.get(n, -1)
            self.lens[c] = before[p]
        return moves, missing

    def free(self, rows):
        for r in rows:
            if 0 <= r < len(self.lens):
                for x in self.table[r]:
                    if 0 <= x < len(self.refs):
                        self.refs[x] -= 1
                self.table[r], self.lens[r] = -1, 0

    def compact(self):
        live = int((self.refs > 0).sum())
        src = [p for p in range(live, len(self.refs)) if self.refs[p] > 0]
        dst = [p for p in range(live) if self.refs[p] <= 0]
        to = dict(zip(src, dst))
        for s, d in to.items():
            self.refs[d], self.refs[s] = self.refs[s], 0
        for i, x in np.ndenumerate(self.table):
            if live <= x < len(self.refs):
                self.table[i] = to.get(int(x), -1)
        return list(to.items()), live
