"""The operators of the 8-bit paged cache: filling it, attending over it, choosing pages of it, and its page pool.

A serving program keeps the keys and values of many sequences in pages of some tokens each, as 8-bit codes with one
power-of-two scale for every page and head.  Every generated token (or every piece of a prompt) appends to the pages and
attends over them; a long context is read in part, by pages whose bounds promise large scores; sequences are forked, ended
and the pool compacted.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TOP = {"e4m3": 448.0, "int8": 127.0}
LOW, HIGH = -40, 40  # exponents of the scales
OUTLIERS, OUTLIER_GAIN = 4, 20.0  # key channels as in the serving configurations


def listed():
    return [
        # One token of 64 conversations goes into the cache; the next piece of four prompts does, into an int8 cache.
        {"name": "append_token", "op": "append", "seqs": 64, "tokens": 4096, "new": 1, "ragged": True, "heads": 8, "d": 128, "page": 64, "cache": "e4m3", "type": "bf16"},
        {"name": "append_prompt", "op": "append", "seqs": 4, "tokens": 8191, "new": 4095, "ragged": True, "heads": 8, "d": 128, "page": 64, "cache": "int8", "type": "bf16"},
        # One generated token early in a conversation and in a long document, a full batch of conversations, a piece of four
        # prompts, and a short draft checked at once by an fp32 model with a sliding window over an int8 cache.
        {"name": "attend_1k", "op": "attend", "seqs": 1, "tokens": 1024, "new": 1, "ragged": False, "heads": 8, "group": 4, "d": 128, "page": 64, "cache": "e4m3", "type": "bf16", "window": 0, "pages": 0},
        {"name": "attend_64k", "op": "attend", "seqs": 1, "tokens": 65536, "new": 1, "ragged": False, "heads": 8, "group": 4, "d": 128, "page": 64, "cache": "e4m3", "type": "bf16", "window": 0, "pages": 0},
        {"name": "attend_batch", "op": "attend", "seqs": 64, "tokens": 8192, "new": 1, "ragged": True, "heads": 8, "group": 4, "d": 128, "page": 64, "cache": "e4m3", "type": "bf16", "window": 0, "pages": 0},
        {"name": "attend_prompt", "op": "attend", "seqs": 4, "tokens": 8192, "new": 2048, "ragged": False, "heads": 8, "group": 4, "d": 128, "page": 64, "cache": "e4m3", "type": "bf16", "window": 0, "pages": 0},
        {"name": "attend_draft", "op": "attend", "seqs": 5, "tokens": 3001, "new": 17, "ragged": True, "heads": 3, "group": 5, "d": 64, "page": 16, "cache": "int8", "type": "f32", "window": 1000, "pages": 0},
        # 64 pages of 64 tokens out of four documents of 131072 tokens.
        {"name": "attend_chosen", "op": "attend", "seqs": 4, "tokens": 131072, "new": 1, "ragged": False, "heads": 8, "group": 4, "d": 128, "page": 64, "cache": "e4m3", "type": "bf16", "window": 0, "pages": 64},
        # Choosing those pages, and choosing for a few queries of fp32 models in medium contexts.
        {"name": "select_128k", "op": "select", "seqs": 4, "tokens": 131072, "new": 1, "ragged": False, "heads": 8, "group": 4, "d": 128, "page": 64, "type": "bf16", "pages": 64},
        {"name": "select_16k", "op": "select", "seqs": 7, "tokens": 16000, "new": 3, "ragged": True, "heads": 4, "group": 8, "d": 64, "page": 32, "type": "f32", "pages": 33},
        # Three more answers started from each of 16 prompts, and a pool made dense after a third of the sequences ended.
        {"name": "fork_48", "op": "fork", "rows": 64, "tokens": 1500, "each": 3, "heads": 8, "d": 128, "page": 64, "cache": "e4m3"},
        {"name": "compact_64", "op": "compact", "rows": 64, "tokens": 1500, "each": 3, "heads": 8, "d": 128, "page": 64, "cache": "e4m3"},
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "select", "fork", "compact"])
    d, page = rng.choice([64, 128, 128, 256]), rng.choice([16, 32, 64, 128])
    c = {"op": op, "heads": rng.choice([1, 2, 4, 5, 8]), "d": d, "page": page}
    if op in ("fork", "compact"):
        return dict(c, rows=rng.randint(8, 64), tokens=_log(rng, 32, 1500), each=rng.randint(1, 4), cache=rng.choice(["e4m3", "int8"]))
    kind = rng.choice(["bf16", "bf16", "f32"])
    if op == "append":
        new = rng.choice([1, 1, _log(rng, 2, 2000)])
        return dict(c, seqs=_log(rng, 1, 64 if new == 1 else 8), tokens=new + _log(rng, 1, 4000), new=new, ragged=rng.random() < 0.7,
                    cache=rng.choice(["e4m3", "int8"]), type=kind)
    group = rng.choice([1, 2, 4, 4, 5, 8, 16])
    if op == "select":
        return dict(c, seqs=_log(rng, 1, 8), tokens=_log(rng, 64, 64000), new=rng.choice([1, 1, 2, 5]), ragged=rng.random() < 0.5, group=group,
                    type=kind, pages=_log(rng, 4, 100))
    way = rng.choice(["token", "token", "prompt", "chosen"])
    c = dict(c, group=group, ragged=rng.random() < 0.6, cache=rng.choice(["e4m3", "int8"]), type=kind, window=0, pages=0)
    if way == "prompt":
        new = _log(rng, 2, 1000)
        return dict(c, seqs=rng.randint(1, 4), tokens=new + _log(rng, 1, 4000), new=new, window=rng.choice([0, 0, 777]))
    if way == "chosen":
        return dict(c, seqs=rng.randint(1, 4), tokens=_log(rng, 1000, 60000), new=rng.choice([1, 2]), pages=_log(rng, 4, 100))
    return dict(c, seqs=_log(rng, 1, 48), tokens=_log(rng, 16, 8000), new=rng.choice([1, 1, 3]), window=rng.choice([0, 0, 500]))


# --- lengths, tables and contents -------------------------------------------------------------------------------------------


def _lengths(c):
    """Tokens of every sequence, the call's own among them, and how many of these are new: by the case alone."""
    r = random.Random("%d %d %d" % (c["seqs"], c["tokens"], c["new"]))
    new = [c["new"] if i == 0 or not c["ragged"] else r.randint(1, c["new"]) for i in range(c["seqs"])]
    lens = [c["tokens"] if i == 0 or not c["ragged"] else max(n, r.randint(c["tokens"] // 8, c["tokens"])) for i, n in enumerate(new)]
    return lens, new


def _pow2(e):
    """2^e as fp32, for whole e."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scale_of(amax, cache):
    """The smallest power of two s with amax / s no larger than the largest code, between 2^LOW and 2^HIGH."""
    m, e = torch.frexp(amax)
    mt, et = math.frexp(TOP[cache])
    return _pow2(torch.where(amax > 0, e - et + (m > mt), LOW).clamp(LOW, HIGH))


def _code(x, cache):
    """Values over their scale as codes: to nearest, ties to even, the largest code beyond it."""
    x = x.clamp(-TOP[cache], TOP[cache])
    return x.to(torch.float8_e4m3fn) if cache == "e4m3" else x.round().to(torch.int8)


def _store(g, n, c, keys):
    """n pages of [heads][page][d] codes with their scales and, of keys, bounds."""
    gain = torch.ones(c["heads"], 1, c["d"], device=DEV)
    if keys:
        gain.view(c["heads"], -1)[:, torch.randperm(c["d"], generator=g, device=DEV)[:OUTLIERS]] = OUTLIER_GAIN
    codes = torch.empty(n, c["heads"], c["page"], c["d"], device=DEV, dtype=torch.float8_e4m3fn if c.get("cache", "e4m3") == "e4m3" else torch.int8)
    scale = torch.empty(n, c["heads"], device=DEV)
    bounds = torch.empty(n, c["heads"], 2, c["d"], device=DEV, dtype=torch.bfloat16) if keys else None
    step = max(1, (1 << 26) // (c["heads"] * c["page"] * c["d"]))
    for i in range(0, n, step):
        x = torch.randn(codes[i:i + step].shape, generator=g, device=DEV) * gain
        s = _scale_of(x.abs().amax((2, 3)), c.get("cache", "e4m3"))
        codes[i:i + step], scale[i:i + step] = _code(x / s[:, :, None, None], c.get("cache", "e4m3")), s
        if keys:
            bounds[i:i + step, :, 0], bounds[i:i + step, :, 1] = x.amin(2), x.amax(2)
    return codes, scale, bounds


def _tables(g, lens, page, spare):
    """Every sequence's pages, scattered over a pool that has some more, as a serving program's pool is after a while."""
    need = [-(-n // page) for n in lens]
    n = sum(need) + spare
    at = torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    table, first = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32, device=DEV), 0
    for i, k in enumerate(need):
        table[i, :k] = at[first:first + k]
        first += k
    return table, n


def _dtype(c):
    return torch.bfloat16 if c["type"] == "bf16" else torch.float32


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = (_prepare_pool if case["op"] in ("fork", "compact") else _prepare_batch)(case, g)
    s["case"] = case
    if own:
        import paper_2504_19874_amd as tq
        s["tq"] = tq
        if case["op"] == "select":  # choosing reads nothing but the bounds; the codes are those of a cache of the same pages
            n, h, _, d = s["bounds"].shape
            s["k"] = s["v"] = torch.zeros(n, h, case["page"], d, dtype=torch.int8, device=DEV)
            s["k_scale"] = s["v_scale"] = torch.ones(n, h, device=DEV)
        s["cache"] = tq.Pages(s["k"], s["v"], s["k_scale"], s["v_scale"], bounds=s["bounds"], refs=s.get("refs"))
    return s


def _prepare_batch(c, g):
    lens, new = _lengths(c)
    rows = sum(new)
    table, n = _tables(g, lens, c["page"], 7)
    s = {"table": table, "lens": _ints(lens), "starts": _ints([sum(new[:i]) for i in range(len(new) + 1)])}
    if c["op"] == "select":
        mean = torch.randn(n, c["heads"], c["d"], generator=g, device=DEV)
        reach = torch.rand(n, c["heads"], c["d"], generator=g, device=DEV) + 1.5
        s["bounds"] = torch.stack([mean - reach, mean + reach], 2).to(torch.bfloat16)
    else:
        s["k"], s["k_scale"], s["bounds"] = _store(g, n, c, True)
        s["v"], s["v_scale"], _ = _store(g, n, c, False)
    if c["op"] == "append":
        s["new_k"] = torch.randn(rows, c["heads"], c["d"], generator=g, device=DEV)
        s["new_k"][:, :, torch.randperm(c["d"], generator=g, device=DEV)[:OUTLIERS]] *= OUTLIER_GAIN
        s["new_k"] = s["new_k"].to(_dtype(c))
        s["new_v"] = torch.randn(rows, c["heads"], c["d"], generator=g, device=DEV).to(_dtype(c))
        return s
    s["q"] = torch.randn(rows, c["heads"] * c["group"], c["d"], generator=g, device=DEV).to(_dtype(c))
    if c["op"] == "select":
        s["chosen"] = torch.empty(rows, c["heads"], c["pages"], dtype=torch.int32, device=DEV)
        return s
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty(rows, c["heads"] * c["group"], device=DEV)
    s["chosen"] = None
    if c["pages"]:
        # of every query: its last page, and others in any number up to the whole list
        last = torch.cat([torch.arange(a - b, a) for a, b in zip(lens, new)]).to(DEV) // c["page"]
        r = torch.rand(rows, c["heads"], int(table.shape[1]), generator=g, device=DEV)
        r = torch.where(torch.arange(r.shape[2], device=DEV) < last[:, None, None], r, -1.0).scatter(2, last[:, None, None].expand(rows, c["heads"], 1), 2.0)
        top, at = r.topk(min(c["pages"], r.shape[2]), 2)
        at = torch.where(top >= 0, at, 1 << 30).sort(2).values
        s["chosen"] = torch.full((rows, c["heads"], c["pages"]), -1, dtype=torch.int32, device=DEV)
        s["chosen"][:, :, :at.shape[2]] = torch.where(at < (1 << 30), at, -1)
    return s


def _prepare_pool(c, g):
    """A pool a third empty; the first quarter of the rows (fork) or two thirds (compact) hold sequences."""
    r = random.Random("%d %d" % (c["rows"], c["tokens"]))
    live = c["rows"] // (1 + c["each"]) if c["op"] == "fork" else c["rows"]
    lens = [c["tokens"] if i == 0 else r.randint(max(1, c["tokens"] // 8), c["tokens"]) for i in range(live)]
    table, n = _tables(g, lens, c["page"], sum(lens) // c["page"] // 2 + c["rows"])
    full = torch.full((c["rows"], table.shape[1]), -1, dtype=torch.int32, device=DEV)
    full[:live] = table
    refs = torch.zeros(n, dtype=torch.int32, device=DEV)
    refs[full[full >= 0].long()] = 1
    lens = _ints(lens + [0] * (c["rows"] - live))
    whole = torch.cat([full.reshape(-1), lens, refs])  # what a pass changes, and starts from
    now = whole.clone()
    a, b = full.numel(), full.numel() + c["rows"]
    s = {"whole": whole, "now": now, "table": now[:a].view(full.shape), "lens": now[a:b], "refs": now[b:]}
    s["k"], s["k_scale"], s["bounds"] = _store(g, n, c, True)
    s["v"], s["v_scale"], _ = _store(g, n, c, False)
    if c["op"] == "fork":
        s["parents"] = torch.arange(live, device=DEV, dtype=torch.int32).repeat_interleave(c["each"])[:c["rows"] - live]
        s["children"] = torch.arange(live, live + s["parents"].numel(), device=DEV, dtype=torch.int32)
    else:
        s["ended"] = torch.randperm(c["rows"], generator=g, device=DEV)[:-(-c["rows"] // 3)].to(torch.int32)
    return s


# --- one pass ---------------------------------------------------------------------------------------------------------------


def run(s):
    c = s["case"]
    return {"append": _append, "attend": _attend, "select": _select, "fork": _fork, "compact": _compact}[c["op"]](s, c)


def _append(s, c):
    if own:
        s["tq"].tq_pages_append(s["cache"], s["new_k"], s["new_v"], s["table"], s["lens"], s["starts"], c["new"])
    else:
        page = c["page"]
        seq, at = _rows(s)
        slot = s["table"][seq, at // page].long()
        count = s["starts"].diff()
        begin = s["lens"] - count  # tokens that were there
        # the pages that get a row, and how many of their own tokens were there before
        index = (begin // page)[:, None] + torch.arange(-(-c["new"] // page) + 1, device=DEV)
        touched = (index * page < s["lens"][:, None]) & (count[:, None] > 0)
        had = (begin[:, None] - index * page).clamp(min=0)[touched]
        ids = s["table"].gather(1, index.clamp(max=s["table"].shape[1] - 1).long())[touched].long()
        for x, codes, scale in ((s["new_k"], s["k"], s["k_scale"]), (s["new_v"], s["v"], s["v_scale"])):
            x = x.float()
            amax = torch.zeros_like(scale).index_reduce_(0, slot, x.abs().amax(2), "amax")
            before = torch.where(had[:, None] > 0, scale[ids], 2.0**LOW)
            after = torch.maximum(before, _scale_of(amax[ids], c["cache"]))
            again = _code(codes[ids].float() * (before / after)[:, :, None, None], c["cache"])
            keep = torch.arange(page, device=DEV) < had[:, None]
            codes.view(torch.uint8)[ids] = torch.where(keep[:, None, :, None], again.view(torch.uint8), codes.view(torch.uint8)[ids])
            scale[ids] = after
            head = torch.arange(c["heads"], device=DEV)
            codes.view(torch.uint8)[slot[:, None], head, (at % page)[:, None]] = _code(x / scale[slot][:, :, None], c["cache"]).view(torch.uint8)
        x = s["new_k"].float().clamp(-_BF16, _BF16)
        lo = torch.full(s["bounds"][:, :, 0].shape, math.inf, device=DEV).index_reduce_(0, slot, x, "amin")[ids]
        hi = torch.full(s["bounds"][:, :, 0].shape, -math.inf, device=DEV).index_reduce_(0, slot, x, "amax")[ids]
        was = s["bounds"][ids].float()
        old = had[:, None, None] > 0
        lo, hi = torch.where(old, torch.minimum(lo, was[:, :, 0]), lo), torch.where(old, torch.maximum(hi, was[:, :, 1]), hi)
        s["bounds"][ids] = torch.stack([_outward(lo, True), _outward(hi, False)], 2).to(torch.bfloat16)
    return {"k": s["k"], "v": s["v"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "bounds": s["bounds"]}


_BF16 = 3.3895313892515355e38  # the largest bf16


def _outward(x, down):
    """fp32 to the next value of bf16 below (above)."""
    bits = x.contiguous().view(torch.int32)
    cut = bits & -65536
    away = ((bits & 65535) != 0) & ((bits < 0) if down else (bits >= 0))
    return (cut + away.to(torch.int32) * 65536).view(torch.float32)


def _rows(s):
    """Sequence and position of every query or new row."""
    count = s["starts"].diff()
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=DEV), count.long())
    at = torch.arange(seq.numel(), device=DEV) - s["starts"][seq] + (s["lens"] - count)[seq]
    return seq, at


def _attend(s, c):
    scale = 1 / math.sqrt(c["d"])
    if own:
        s["tq"].tq_pages_attend(s["cache"], s["q"], s["table"], s["lens"], s["starts"], c["new"], scale, s["out"], lse=s["lse"], window=c["window"], chosen=s["chosen"])
        return {"out": s["out"], "lse": s["lse"]}
    h, g, d, page = c["heads"], c["group"], c["d"], c["page"]
    seq, at = _rows(s)
    q = s["q"].float().view(-1, h, g, d)
    if s["chosen"] is not None:  # one block of [group] rows per query and head, with its own keys
        pages = s["table"][seq[:, None, None], s["chosen"].clamp(min=0).long()].long()
        head = torch.arange(h, device=DEV)[None, :, None]
        k = (s["k"][pages, head].float() * s["k_scale"][pages, head][..., None, None]).flatten(2, 3)
        v = (s["v"][pages, head].float() * s["v_scale"][pages, head][..., None, None]).flatten(2, 3)
        where = (s["chosen"][..., None].long() * page + torch.arange(page, device=DEV)).flatten(2)
        seen = ((where >= 0) & (where <= at[:, None, None]))[:, :, None]
    else:  # one block of [new * group] rows per sequence and head
        count, longest, width = s["starts"].diff(), c["new"], -(-c["tokens"] // page)
        pages = s["table"][:, :width].clamp(min=0).long()
        k = (s["k"][pages].float() * s["k_scale"][pages][..., None, None]).transpose(1, 2).flatten(2, 3)
        v = (s["v"][pages].float() * s["v_scale"][pages][..., None, None]).transpose(1, 2).flatten(2, 3)
        take = (s["starts"][:-1, None] + torch.arange(longest, device=DEV)).clamp(max=q.shape[0] - 1).long()
        q = q[take].permute(0, 2, 1, 3, 4).flatten(2, 3)
        mine = ((s["lens"] - count)[:, None] + torch.arange(longest, device=DEV))[:, None, :, None]
        where = torch.arange(k.shape[2], device=DEV)
        seen = (where <= mine) & (where < s["lens"][:, None, None, None])
        if c["window"]:
            seen &= where > mine - c["window"]
        seen = seen.repeat_interleave(g, 2)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).masked_fill_(~seen, -math.inf)
    m = x.amax(3, keepdim=True)
    m = torch.where(m > -math.inf, m, 0.0)
    p = x.sub_(m).exp_()
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    lse = (total.log() + m)[..., 0]
    if s["chosen"] is None:
        inside = (torch.arange(longest, device=DEV) < count[:, None])
        o = o.view(count.numel(), h, longest, g, d).transpose(1, 2)[inside]
        lse = lse.view(count.numel(), h, longest, g).transpose(1, 2)[inside]
    return {"out": o.reshape(s["q"].shape).to(s["q"].dtype), "lse": lse.reshape(s["lse"].shape)}


KEEP_FIRST, KEEP_LAST = 1, 2  # pages that are chosen whatever their bounds


def _select(s, c):
    if own:
        s["tq"].tq_pages_select(s["cache"], s["q"], s["table"], s["lens"], s["starts"], c["new"], s["chosen"], keep_first=KEEP_FIRST, keep_last=KEEP_LAST)
        return {"chosen": s["chosen"]}
    seq, at = _rows(s)
    width = -(-c["tokens"] // c["page"])
    pages = s["table"][:, :width].clamp(min=0).long()
    lo, hi = (s["bounds"][pages][:, :, :, i].permute(0, 2, 3, 1).double()[seq] for i in (0, 1))  # [row][head][d][page]
    q = s["q"].double().view(-1, c["heads"], c["group"], c["d"])
    score = (torch.matmul(q.clamp(min=0), hi) + torch.matmul(q.clamp(max=0), lo)).float().amax(2)  # 64 bits: whole numbers hang on it
    last, j = (at // c["page"])[:, None, None], torch.arange(width, device=DEV)
    score = torch.where((j < KEEP_FIRST) | (j > last - KEEP_LAST), math.inf, score)
    score = torch.where(j <= last, score, -math.inf)
    order = score.sort(dim=2, descending=True, stable=True)
    k = min(c["pages"], width)
    best = torch.where(order.values[:, :, :k] > -math.inf, order.indices[:, :, :k], 1 << 30).sort(2).values
    chosen = torch.full((q.shape[0], c["heads"], c["pages"]), -1, dtype=torch.int32, device=DEV)
    chosen[:, :, :k] = torch.where(best < (1 << 30), best, -1)
    return {"chosen": chosen}


def _pool(s):
    return {n: s[n] for n in ("table", "lens", "refs", "k", "v", "k_scale", "v_scale", "bounds")}


def _move(s, dst, src):
    for x in (s["k"].view(torch.uint8), s["v"].view(torch.uint8), s["k_scale"], s["v_scale"], s["bounds"]):
        x[dst] = x[src]


def _fork(s, c):
    s["now"].copy_(s["whole"])
    if own:
        s["tq"].tq_pages_fork(s["cache"], s["table"], s["lens"], s["parents"], s["children"])
        return _pool(s)
    p, kids = s["parents"].long(), s["children"].long()
    j, n = torch.arange(s["table"].shape[1], device=DEV), s["lens"][p]
    row = torch.where(j < (n // c["page"])[:, None], s["table"][p], -1)
    part = (n % c["page"] > 0).nonzero()[:, 0]
    new, at = (s["refs"] == 0).nonzero()[:part.numel(), 0], (n // c["page"])[part].long()
    shared = row[row >= 0].long()
    s["refs"].index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    s["refs"][new] = 1
    row[part, at] = new.to(torch.int32)
    _move(s, new, s["table"][p[part], at].long())
    s["table"][kids], s["lens"][kids] = row, n
    return _pool(s)


def _compact(s, c):
    s["now"].copy_(s["whole"])
    if own:
        s["tq"].tq_pages_free(s["cache"], s["table"], s["lens"], s["ended"])
        s["tq"].tq_pages_compact(s["cache"], s["table"])
        return _pool(s)
    rows = s["ended"].long()
    gone = s["table"][rows]
    gone = gone[gone >= 0].long()
    s["refs"].index_add_(0, gone, -torch.ones_like(gone, dtype=torch.int32))
    s["table"][rows], s["lens"][rows] = -1, 0
    live = s["refs"] > 0
    n = int(live.sum())
    src, dst = live[n:].nonzero()[:, 0] + n, (~live[:n]).nonzero()[:, 0]
    _move(s, dst, src)
    to = torch.arange(live.numel(), device=DEV, dtype=torch.int32)
    to[src] = dst.to(torch.int32)
    s["refs"][dst] = s["refs"][src]
    s["refs"][src] = 0
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], -1))
    return _pool(s)


# --- what a pass cannot do without ------------------------------------------------------------------------------------------


def _seen(n, new, window):
    """Query-key pairs of one sequence and head, and the keys that some query sees."""
    last = range(n - new, n)
    pairs = sum(min(p + 1, window) if window else p + 1 for p in last)
    return pairs, (n - max(0, n - new + 1 - window) if window else n)


def _page_bytes(c):
    return c["heads"] * (2 * c["page"] * c["d"] + 8 + 4 * c["d"])


def work(case):
    c = case
    if c["op"] in ("fork", "compact"):
        r = random.Random("%d %d" % (c["rows"], c["tokens"]))
        live = c["rows"] // (1 + c["each"]) if c["op"] == "fork" else c["rows"]
        lens = [c["tokens"] if i == 0 else r.randint(max(1, c["tokens"] // 8), c["tokens"]) for i in range(live)]
        need = [-(-n // c["page"]) for n in lens]
        pool = sum(need) + sum(lens) // c["page"] // 2 + c["rows"]
        if c["op"] == "fork":
            parents = [i for i in range(live) for _ in range(c["each"])][:c["rows"] - live]
            return {"bytes": 2 * _page_bytes(c) * sum(lens[p] % c["page"] > 0 for p in parents) + 4 * (pool + 2 * sum(need[p] for p in parents)), "flops": 0}
        share = 1 - -(-c["rows"] // 3) / c["rows"]
        stay = sum(need) * share  # on average: which sequences end hangs on the seed
        return {"bytes": 2 * _page_bytes(c) * stay * (1 - stay / pool) + 8 * (pool + sum(need)), "flops": 0}
    lens, new = _lengths(c)
    e, rows = (2 if c["type"] == "bf16" else 4), sum(new)
    h, d, page = c["heads"], c["d"], c["page"]
    if c["op"] == "append":
        touched = sum((n - 1) // page - (n - k) // page + 1 for n, k in zip(lens, new))
        return {"bytes": rows * h * 2 * d * (e + 1) + touched * h * (8 + 4 * d), "flops": 0}
    heads = h * c["group"]
    if c["op"] == "select":
        pages = sum(-(-n // page) for n in lens)
        pairs = sum(-(-n // page) * k for n, k in zip(lens, new)) * heads
        return {"bytes": pages * h * 4 * d + rows * heads * d * e + rows * h * 4 * c["pages"], "flops": pairs * 2 * d}
    if c["pages"]:
        keys = pairs = sum(min(c["pages"] * page, n) * k for n, k in zip(lens, new))
    else:
        seen = [_seen(n, k, c["window"]) for n, k in zip(lens, new)]
        pairs, keys = sum(p for p, _ in seen), sum(k for _, k in seen)
    return {"bytes": keys * h * (2 * d + 8 / page) + rows * heads * (2 * d * e + 4), "flops": pairs * heads * 4 * d}


# --- the definition, in 64 bits ---------------------------------------------------------------------------------------------


def exact(case, seed):
    """Appending and attending, sequence by sequence; the other operators return whole numbers and copies."""
    if case["op"] not in ("append", "attend"):
        return None
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return (_exact_append if case["op"] == "append" else _exact_attend)(s, case)


def _round64(x, cache):
    if cache == "int8":
        return x.round().clamp(-127, 127)
    e = torch.frexp(x.abs())[1]  # |x| in [2^(e-1), 2^e): four significant bits, none below 2^-9
    step = torch.exp2((e - 4).clamp(min=-9).double())
    return ((x / step).round() * step).clamp(-448, 448)


def _exact_append(s, c):
    lens, new = _lengths(c)
    page, top = c["page"], TOP[c["cache"]]
    got = {"k": s["k"].double(), "v": s["v"].double(), "k_scale": s["k_scale"].double(), "v_scale": s["v_scale"].double(), "bounds": s["bounds"].double()}
    table = s["table"].tolist()
    row = 0
    for i, (n, count) in enumerate(zip(lens, new)):
        for first in range((n - count) // page, (n - 1) // page + 1):
            a, b = max(n - count, first * page), min(n, (first + 1) * page)
            p, had = table[i][first], a - first * page
            for name in "kv":
                x = s["new_" + name][row:row + b - a].double().transpose(0, 1)  # [head][row][d]
                amax, was = x.abs().amax((1, 2)), got[name + "_scale"][p]
                e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 2.0**LOW) / top))
                e = torch.where(torch.exp2(e) * top < amax, e + 1, e)  # the logarithm's own rounding
                e = torch.where(torch.exp2(e - 1) * top >= amax, e - 1, e)
                to = torch.exp2(torch.where(amax > 0, e, LOW).clamp(LOW, HIGH))
                if had:
                    to = torch.maximum(to, was)
                    got[name][p][:, :had] = _round64(got[name][p][:, :had] * (was / to)[:, None, None], c["cache"])
                got[name][p][:, had:had + b - a] = _round64(x / to[:, None, None], c["cache"])
                got[name + "_scale"][p] = to
            x = s["new_k"][row:row + b - a].double()
            lo, hi = x.amin(0), x.amax(0)
            if had:
                lo, hi = torch.minimum(lo, got["bounds"][p, :, 0]), torch.maximum(hi, got["bounds"][p, :, 1])
            for side, y in ((0, lo), (1, hi)):
                step = torch.exp2((torch.frexp(y)[1] - 8).clamp(min=-133).double())
                got["bounds"][p, :, side] = (torch.floor(y / step) if side == 0 else torch.ceil(y / step)) * step
            row += b - a
    return got


def _exact_attend(s, c):
    lens, new = _lengths(c)
    if sum(a * b for a, b in zip(lens, new)) * c["heads"] * c["group"] * c["d"] > 2e12:
        return None
    h, g, d, page = c["heads"], c["group"], c["d"], c["page"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device=DEV)
    row = 0
    for i, (n, count) in enumerate(zip(lens, new)):
        for head in range(h):
            mine = slice(head * g, (head + 1) * g)
            for a in ([row] if s["chosen"] is None else range(row, row + count)):
                b = row + count if s["chosen"] is None else a + 1
                order = torch.arange(-(-n // page), device=DEV) if s["chosen"] is None else s["chosen"][a, head][s["chosen"][a, head] >= 0].long()
                ids = s["table"][i][order].long()
                k = (s["k"][ids, head].double() * s["k_scale"][ids, head].double()[:, None, None]).reshape(-1, d)
                v = (s["v"][ids, head].double() * s["v_scale"][ids, head].double()[:, None, None]).reshape(-1, d)
                where = (order[:, None] * page + torch.arange(page, device=DEV)).reshape(-1)
                at = torch.arange(n - count + a - row, n - count + b - row, device=DEV).repeat_interleave(g)[:, None]
                x = (s["q"][a:b, mine].double().reshape(-1, d) @ k.T.contiguous()) / math.sqrt(d)
                x = torch.where((where <= at) & (where > at - (c["window"] or n + 1)), x, -math.inf)
                lse[a:b, mine] = torch.logsumexp(x, 1).view(-1, g)
                out[a:b, mine] = (torch.softmax(x, 1) @ v).view(-1, g, d)
        row += count
    return {"out": out, "lse": lse}
