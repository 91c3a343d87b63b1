"""What the speed of the cached-sequence operators is measured on: keys and values appended to a cache in pages, attention
over it, and the pages' bookkeeping, at the sizes they are used at.

A case is a plain dict; `prepare` makes what a serving program holds before the call (inputs, pools, page tables, output
buffers, workspace), `run` is one pass: through the binding where `own` is true, else in elementary torch operations in 32
bits.  `exact` computes the same from the definitions in 64 bits.  Fields of a case:

  op          "append" | "attend" | "reserve" | "fork" | "compact"
  dtype       "float32" | "float16" | "bfloat16": of everything that holds vectors
  B           sequences: one per worker of each group, or per request
  heads, kv   query heads, heads of the cache;  dim  floats per head
  page        tokens per page
  short, long sequence b's length lies between the two (the first has `long`), new tokens included
  new         new tokens per sequence; 0: the whole sequence is new (a prompt)
  window, sinks   of attend; 0: no limit
  pairs, axes, split, norm   of append: rotated pairs, position axes, halves instead of neighbours, with norms
  planes, pages   of the page operators: pools (two per layer) and pages in each
  children    of fork: new sequences per old one; 0: every other sequence ends, the others go on
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
EPS = 1e-6
BASE = 10000.0
SCRATCH = 1 << 27                                             # bytes of workspace that a program keeps for all its calls


def listed():
    def append(name, **f):
        return dict({"name": name, "op": "append", "axes": 1, "split": True, "norm": True, "page": 16}, **f)

    def attend(name, **f):
        return dict({"name": name, "op": "attend", "window": 0, "sinks": 0, "page": 16}, **f)

    def pages(name, op, **f):
        return dict({"name": name, "op": op, "dtype": "bfloat16", "kv": 8, "dim": 128, "page": 16, "children": 0}, **f)

    return [
        # Appending: the next token of one group's 24 workers (12 heads of 64, the text workload's 768 floats); ragged prompts
        # of a batch; patches of a video with three axes of positions and a head size that is no power of two.
        append("append_token", dtype="float32", B=24, heads=12, kv=12, dim=64, pairs=32, short=90, long=129, new=1),
        append("append_prompts", dtype="bfloat16", B=8, heads=32, kv=8, dim=128, pairs=64, short=901, long=3900, new=0),
        append("append_patches", dtype="float16", B=4, heads=16, kv=16, dim=80, pairs=40, axes=3, split=False, norm=False,
               short=2311, long=2601, new=0),
        # Attention for single tokens: one group's workers on short sequences, three requests with very long ones, and the
        # workers of eight groups with a window and four first tokens that stay visible.
        attend("attend_token_short", dtype="float32", B=24, heads=12, kv=12, dim=64, short=90, long=129, new=1),
        attend("attend_token_long", dtype="bfloat16", B=3, heads=32, kv=8, dim=128, short=61003, long=131072, new=1),
        attend("attend_token_window", dtype="float16", B=192, heads=16, kv=2, dim=128, short=200, long=9001, new=1, window=1024,
               sinks=4),
        # Attention for prompts: the coded text sequences of eight groups (128 tokens each), two long prompts, and one with a
        # window.
        attend("attend_text", dtype="float32", B=192, heads=12, kv=12, dim=64, short=128, long=128, new=0),
        attend("attend_prompts", dtype="bfloat16", B=2, heads=32, kv=8, dim=128, short=4099, long=7001, new=0),
        attend("attend_prompt_window", dtype="float16", B=1, heads=24, kv=8, dim=64, page=64, short=12001, long=12001, new=0,
               window=2048, sinks=4),
        # Pages: room for one more token of every worker's sequence; one prompt's cache forked to the 24 workers of a group, eight
        # groups at once (eight layers, two planes each); and the pages that ended sequences left free closed up.
        pages("pages_reserve", "reserve", B=192, short=33, long=2100, planes=0, pages=32768),
        pages("pages_fork", "fork", B=8, short=120, long=1001, planes=16, pages=4096, children=24),
        pages("pages_compact", "compact", B=96, short=33, long=600, planes=16, pages=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one token to long prompts, one sequence to many, odd sizes, each type."""
    op = rng.choice(["append", "append", "attend", "attend", "attend", "reserve", "fork", "compact"])
    c = {"op": op, "dtype": rng.choice(["float32", "float16", "bfloat16", "bfloat16"]), "page": rng.choice([8, 16, 16, 32, 64, 128])}
    c["kv"] = kv = rng.choice([1, 2, 4, 8, 8, 12])
    c["dim"] = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128, 160, 256])
    if op in ("append", "attend"):
        c["heads"] = heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
        token = rng.random() < 0.5
        c["new"] = rng.choice([1, 1, 1, 2, 5]) if token else rng.choice([0, 0, 0, _log_int(rng, 16, 2000)])
        c["B"] = B = _log_int(rng, 1, 256) if token else _log_int(rng, 1, 24)
        # at most 300 MB of vectors in a pass of append; at most 150 GFLOP and 1 GB of cache in one of attend
        size = {"float32": 4, "float16": 2, "bfloat16": 2}[c["dtype"]] * c["dim"]
        if op == "append":
            most = int(3e8) // (2 * size * (heads + 2 * kv) * B)
            c["long"] = max(c["new"], _log_int(rng, 6, 100000) if c["new"] else max(2, min(most, _log_int(rng, 6, 20000))))
        else:
            most = int(5e8) // (size * kv * B)
            if token:
                c["long"] = max(c["new"], min(most, _log_int(rng, 6, 131072)))
            else:
                most = min(most, int(math.sqrt(7.5e10 / (c["dim"] * heads * B))))
                c["long"] = max(c["new"], 2, min(most, _log_int(rng, 6, 9000)))
        if op == "append":
            # the pools hold the whole sequences: a bound for what is prepared, not for what a pass costs
            c["long"] = max(c["new"], 2, min(c["long"], int(2e9) // (2 * size * kv * B)))
        c["short"] = max(1, c["new"], int(c["long"] * rng.choice([0.3, 0.9, 1.0])))
        if op == "append":
            c["axes"] = rng.choice([1, 1, 2, 3])
            c["pairs"] = rng.choice([c["dim"] // 2, c["dim"] // 2, c["dim"] // 4])
            c["split"], c["norm"] = rng.random() < 0.5, rng.random() < 0.7
        else:
            c["window"] = rng.choice([0, 0, _log_int(rng, 16, 4096)])
            c["sinks"] = rng.choice([0, 1, 4, 64]) if c["window"] else 0
        return c
    c["B"] = B = _log_int(rng, 1, 256)
    c["long"] = _log_int(rng, 8, 4000)
    c["short"] = max(1, int(c["long"] * rng.choice([0.3, 0.9])))
    c["children"] = rng.choice([0, 1, 4, 24]) if op == "fork" else 0
    held = B * -(-c["long"] // c["page"]) + B * (c["children"] + 1)
    c["pages"] = held + _log_int(rng, 1, 4000)
    plane = c["pages"] * kv * c["page"] * c["dim"] * {"float32": 4, "float16": 2, "bfloat16": 2}[c["dtype"]]
    c["planes"] = 0 if op == "reserve" else max(2, min(64, int(1.8e9 / plane)) // 2 * 2)
    while op != "reserve" and c["planes"] * plane > 1.8e9:                     # two planes are too much already: shorter sequences
        c["long"], c["short"] = c["long"] // 2 + 1, max(1, c["short"] // 2)
        held = B * -(-c["long"] // c["page"]) + B * (c["children"] + 1)
        c["pages"] = held + 7
        plane = c["pages"] * kv * c["page"] * c["dim"] * {"float32": 4, "float16": 2, "bfloat16": 2}[c["dtype"]]
    return c


# ---- what a case fixes whatever the seed --------------------------------------------------------------------------------
def _lengths(case):
    """int64 [B]: spread over short..long, the first the longest."""
    b = np.arange(case["B"])
    return case["long"] - np.floor((case["long"] - case["short"] + 1) * ((b * 0.6180339887498949) % 1.0)).astype(np.int64)


def _new(case):
    lens = _lengths(case)
    return lens if case["new"] == 0 else np.minimum(lens, case["new"])


def _visible(case, p):
    """How many keys a query at place p sees (an array of places)."""
    if case["window"] == 0:
        return p + 1
    near = np.minimum(p + 1, case["window"])
    return near + np.minimum(case["sinks"], p + 1 - near)


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.as_tensor(np.asarray(values), dtype=torch.int32, device=DEVICE)


def _axis_of_pair(case):
    """Pairs in turn for time, height and width, as sections of the head."""
    return np.minimum(np.arange(case["pairs"]) * case["axes"] // case["pairs"], case["axes"] - 1).astype(np.int32)


def _frequencies(case):
    return BASE ** (-np.arange(case["pairs"], dtype=np.float64) / case["pairs"])


def _table(g, lens, page, pages, columns):
    """int32 [B, columns]: every sequence's pages, at places drawn from all of them; -1 behind its last one."""
    count = -(-lens // page)
    order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
    first = np.concatenate([[0], np.cumsum(count)])
    at = torch.as_tensor(first[:-1, None] + np.arange(columns)[None, :], device=DEVICE)
    used = torch.as_tensor(np.arange(columns)[None, :] < count[:, None], device=DEVICE)
    return torch.where(used, order[at.clamp(max=pages - 1)], torch.full_like(at, -1, dtype=torch.int32)).contiguous()


def prepare(case, seed):
    g = _generator(seed)
    op, t, B, page = case["op"], TYPES[case["dtype"]], case["B"], case["page"]
    lens = _lengths(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE).to(t)

    s = {"op": op, "page": page, "B": B}
    if op in ("append", "attend"):
        heads, kv, dim = case["heads"], case["kv"], case["dim"]
        n = _new(case)
        T = int(n.sum())
        columns = -(-int(lens.max()) // page) + 1
        P = int((-(-lens // page)).sum()) + 3
        s["table"] = _table(g, lens, page, P, columns)
        s["lens"], s["starts"] = _ints(lens), _ints(np.concatenate([[0], np.cumsum(n)]))
        s["out"] = torch.empty((T, heads, dim), dtype=t, device=DEVICE)
        s["status"] = torch.empty((B,), dtype=torch.int32, device=DEVICE)
        if op == "append":
            s["k_pool"] = torch.zeros((P, kv, page, dim), dtype=t, device=DEVICE)
            s["v_pool"] = torch.zeros((P, kv, page, dim), dtype=t, device=DEVICE)
            # one projection's output holds all three
            rows = normal(T, heads + 2 * kv, dim)
            s["q"], s["k"], s["v"] = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
            s["q_weight"] = (1.0 + 0.1 * normal(dim)).to(t) if case["norm"] else None
            s["k_weight"] = (1.0 + 0.1 * normal(dim)).to(t) if case["norm"] else None
            s["split"], s["freq"], s["axis"], s["positions"] = case["split"], _frequencies(case), None, None
            if case["axes"] > 1:
                s["axis"] = _axis_of_pair(case)
                s["positions"] = torch.randint(0, 700, (T, case["axes"]), generator=g, device=DEVICE).to(torch.int32)
            s["axis_index"] = torch.as_tensor(_axis_of_pair(case), device=DEVICE).long()
            s["freq_device"] = torch.as_tensor(s["freq"], device=DEVICE)
            return s
        s["q"] = normal(T, heads, dim)
        s["k_pool"], s["v_pool"] = normal(P, kv, page, dim), normal(P, kv, page, dim)
        s["window"], s["sinks"] = case["window"], case["sinks"]
        s["max_rows"], s["max_len"] = int(n.max()), int(lens.max())
        s["workspace"] = torch.empty((SCRATCH,), dtype=torch.uint8, device=DEVICE)
        return s

    # the page operators: what a program holds is one buffer of table, lens and refs, and the pools
    P, columns = case["pages"], -(-int(lens.max()) // page) + 2
    table = _table(g, lens, page, P, columns)
    if op == "compact":                                       # every third sequence has ended and given its pages back
        lens = np.where(np.arange(B) % 3 == 1, 0, lens)
        table = torch.where(_ints(lens)[:, None] > 0, table, torch.full_like(table, -1))
    refs = torch.zeros((P,), dtype=torch.int32, device=DEVICE)
    refs[table[table >= 0].long()] = 1
    s["kept"] = torch.cat([table.flatten(), _ints(lens), refs])
    state = torch.empty_like(s["kept"])
    s["state"] = state
    s["table"], s["lens"], s["refs"] = state[:B * columns].view(B, columns), state[B * columns:B * columns + B], state[B * columns + B:]
    if op == "reserve":
        s["add"] = torch.randint(1, 3, (B,), generator=g, device=DEVICE).to(torch.int32)
        s["status"] = torch.empty((B,), dtype=torch.int32, device=DEVICE)
    else:
        s["pools"] = torch.empty((case["planes"], P, case["kv"], page, case["dim"]), dtype=t, device=DEVICE)
        for plane in s["pools"]:
            plane.normal_(generator=g)
    if op == "fork":
        children = case["children"]
        parents = np.repeat(np.arange(B), children) if children else np.where(np.arange(B) % 2 == 1, -1, np.arange(B))
        n = len(parents)
        s["parents"] = _ints(parents)
        s["table_out"] = torch.empty((n, columns), dtype=torch.int32, device=DEVICE)
        s["lens_out"] = torch.empty((n,), dtype=torch.int32, device=DEVICE)
        s["refs_out"] = torch.empty((P,), dtype=torch.int32, device=DEVICE)
        s["status"] = torch.empty((n,), dtype=torch.int32, device=DEVICE)
    if op == "compact":
        s["moved"] = torch.empty((P,), dtype=torch.int32, device=DEVICE)
        s["live"] = torch.empty((1,), dtype=torch.int32, device=DEVICE)
    s["workspace"] = torch.empty((SCRATCH,), dtype=torch.uint8, device=DEVICE)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------
def _places(s):
    """Of every new token: its sequence, its index there, and its place."""
    T = s["q"].shape[0]
    t = torch.arange(T, device=DEVICE)
    starts, lens = s["starts"].long(), s["lens"].long()
    b = torch.searchsorted(starts, t, right=True) - 1
    i = t - starts[b]
    return b, i, lens[b] - (starts[b + 1] - starts[b]) + i


def _plain_append(s):
    b, _, place = _places(s)
    position = place[:, None] if s["positions"] is None else s["positions"].long()
    angle = position.double()[:, s["axis_index"]] * s["freq_device"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    R = cos.shape[2]

    def turned(x, weight):
        y = x.float()
        if weight is not None:
            y = y * torch.rsqrt((y * y).mean(2, keepdim=True) + EPS) * weight.float()
        if s["split"]:
            a, c = y[..., :R], y[..., R:2 * R]
            z = torch.cat([a * cos - c * sin, a * sin + c * cos, y[..., 2 * R:]], dim=2)
        else:
            a, c = y[..., 0:2 * R:2], y[..., 1:2 * R:2]
            z = torch.cat([torch.stack([a * cos - c * sin, a * sin + c * cos], dim=3).flatten(2), y[..., 2 * R:]], dim=2)
        return z.to(x.dtype)

    page = s["table"].long()[b, place // s["page"]]
    slot = place % s["page"]
    s["k_pool"][page, :, slot] = turned(s["k"], s["k_weight"])
    s["v_pool"][page, :, slot] = s["v"]
    s["out"].copy_(turned(s["q"], s["q_weight"]))
    s["status"].zero_()
    return s["out"], s["k_pool"], s["v_pool"], s["status"]


def _plain_attend(s):
    q, B, kv, dim = s["q"], s["B"], s["k_pool"].shape[1], s["q"].shape[2]
    group = q.shape[1] // kv
    R, columns = s["max_rows"], -(-s["max_len"] // s["page"])
    table = s["table"][:, :columns].long().clamp(min=0)
    k = s["k_pool"][table].float().transpose(1, 2).reshape(B, kv, -1, dim)                 # [B, kv, keys, dim]
    v = s["v_pool"][table].float().transpose(1, 2).reshape(B, kv, -1, dim)
    starts, lens = s["starts"].long(), s["lens"].long()
    n = starts[1:] - starts[:-1]
    i = torch.arange(R, device=DEVICE)
    rows = q[(starts[:-1, None] + i).clamp(max=q.shape[0] - 1)].float()                     # [B, R, heads, dim]
    rows = rows.view(B, R, kv, group, dim).permute(0, 2, 1, 3, 4).reshape(B, kv, R * group, dim)
    score = torch.matmul(rows, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(dim))
    place = (lens - n)[:, None, None] + i[None, :, None]                                    # [B, R, 1]
    key = torch.arange(k.shape[2], device=DEVICE)
    hidden = key > place
    if s["window"]:
        hidden |= (key <= place - s["window"]) & (key >= s["sinks"])
    score = score.view(B, kv, R, group, -1).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    top = score.amax(4, keepdim=True)
    weight = score.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = weight.sum(4, keepdim=True)
    out = torch.matmul(weight.view(B, kv, R * group, -1), v).view(B, kv, R, group, dim) / torch.where(total == 0, 1.0, total)
    b, at, _ = _places(s)
    s["out"].copy_(out.permute(0, 2, 1, 3, 4).reshape(B, R, -1, dim)[b, at])
    s["status"].zero_()
    return s["out"], s["status"]


def _free_pages(refs):
    """Free pages in ascending order (behind them the others), and how many there are."""
    return torch.sort((refs != 0).to(torch.int8), stable=True).indices.to(torch.int32), (refs == 0).sum()


def _plain_reserve(s):
    table, lens, refs, add = s["table"], s["lens"].long(), s["refs"], s["add"].long()
    old, new = (lens + s["page"] - 1) // s["page"], (lens + add + s["page"] - 1) // s["page"]
    last = refs[table.gather(1, (old - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0).long()]
    shared = (lens % s["page"] != 0) & (add > 0) & (last > 1)
    want = torch.where(shared, 0, new - old)
    upto = want.cumsum(0)
    free, count = _free_pages(refs)
    short = (upto > count) & (want > 0)
    ok = ~(shared | short)
    column = torch.arange(table.shape[1], device=DEVICE)
    fresh = (column >= old[:, None]) & (column < new[:, None]) & ok[:, None]
    rank = ((upto - want)[:, None] + column - old[:, None]).clamp(0, refs.shape[0] - 1)
    taken = torch.arange(refs.shape[0], device=DEVICE) < torch.where(ok, upto, 0).max()
    refs[free.long()] = torch.where(taken, 1, refs[free.long()])
    table.copy_(torch.where(fresh, free[rank], table))
    s["lens"].copy_(torch.where(ok, lens + add, lens))
    s["status"].copy_(torch.where(shared, 4, torch.where(short, 3, 0)))
    return s["table"], s["lens"], s["refs"], s["status"]


def _plain_fork(s):
    table, lens, refs, page, parents = s["table"], s["lens"].long(), s["refs"], s["page"], s["parents"].long()
    P, n, columns = refs.shape[0], parents.shape[0], table.shape[1]
    column = torch.arange(columns, device=DEVICE)
    parent = parents.clamp(min=0)
    length = torch.where(parents >= 0, lens[parent], 0)
    full, partial = length // page, length % page != 0
    whole = column < full[:, None]
    rows = table[parent]

    def holders(rows, used):
        return torch.zeros((P + 1,), dtype=torch.int32, device=DEVICE).index_add_(
            0, torch.where(used, rows, P).flatten().long(), torch.ones((rows.numel(),), dtype=torch.int32, device=DEVICE))[:P]

    left = refs - holders(table, column < (-(-lens // page))[:, None]) + holders(rows, whole)
    source = torch.where(partial, rows.gather(1, full.clamp(max=columns - 1)[:, None])[:, 0].long(), P)
    index = torch.arange(n, device=DEVICE)
    first = torch.full((P + 1,), n, device=DEVICE).scatter_reduce_(0, source, index, "amin")
    left = torch.cat([left, left.new_ones(1)])
    keeps = partial & (left[source] == 0) & (first[source] == index)
    left[torch.where(keeps, source, P)] = 1
    left = left[:P]
    copies = partial & ~keeps
    upto = copies.to(torch.int64).cumsum(0)
    free, count = _free_pages(left)
    target = free[(upto - 1).clamp(0, P - 1)].long()
    taken = torch.arange(P, device=DEVICE) < upto[-1]
    left[free.long()] = torch.where(taken, 1, left[free.long()])
    last = torch.where(copies, target, source).to(torch.int32)
    rows = torch.where(whole, rows, torch.where((column == full[:, None]) & partial[:, None], last[:, None], -1))
    # a row that copies nothing repeats the first copy, or, where there is none, copies page 0 onto itself
    one = copies.to(torch.int8).argmax(0, keepdim=True)
    to = torch.where(copies, target, torch.where(copies[one], target[one], 0))
    from_ = torch.where(copies, source, torch.where(copies[one], source[one], 0))
    s["pools"][:, to] = s["pools"][:, from_]
    s["table_out"].copy_(rows)
    s["lens_out"].copy_(length)
    s["refs_out"].copy_(left)
    s["status"].copy_(torch.where(copies & (upto > count), 3, 0))
    return s["table_out"], s["lens_out"], s["refs_out"], s["status"], s["pools"]


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    P = refs.shape[0]
    alive = refs != 0
    live = alive.sum()
    index = torch.arange(P, device=DEVICE)
    # the k-th live page behind the line goes to the k-th free place before it
    high, low = alive & (index >= live), ~alive & (index < live)
    from_ = torch.sort((~high).to(torch.int8), stable=True).indices
    to = torch.sort((~low).to(torch.int8), stable=True).indices
    moves = high.sum()
    real = index < moves
    moved = torch.where(alive, index, -1)
    moved[from_] = torch.where(real, to, moved[from_])
    # never more than half of all pages move; a pair that is none repeats the first, or copies page 0 onto itself
    half = P // 2
    a, b = (torch.where(real, x, torch.where(moves > 0, x[:1], 0))[:half] for x in (from_, to))
    s["pools"][:, b] = s["pools"][:, a]
    refs.copy_(torch.zeros_like(refs).scatter_add_(0, moved.clamp(min=0), torch.where(alive, refs, 0)))
    table.copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()], -1))
    s["moved"].copy_(moved)
    s["live"].copy_(live)
    return s["table"], s["refs"], s["moved"], s["live"], s["pools"]


def run(s):
    op = s["op"]
    if "kept" in s:                                           # the sequences as they stood before the step
        s["state"].copy_(s["kept"])
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "reserve": _plain_reserve, "fork": _plain_fork,
                "compact": _plain_compact}[op](s)
    from paper_2109_09868_amd import binding
    if op == "append":
        binding.approxifer_append(s["q"], s["k"], s["v"], s["k_pool"], s["v_pool"], s["table"], s["lens"], s["starts"], s["freq"],
                                  q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, positions=s["positions"],
                                  axis=s["axis"], interleaved=not s["split"], q_out=s["out"], status=s["status"])
        return s["out"], s["k_pool"], s["v_pool"], s["status"]
    if op == "attend":
        return binding.approxifer_attend(s["q"], s["k_pool"], s["v_pool"], s["table"], s["lens"], s["starts"], s["max_rows"],
                                         s["max_len"], window=s["window"], sinks=s["sinks"], out=s["out"], status=s["status"],
                                         workspace=s["workspace"])
    if op == "reserve":
        binding.approxifer_cache_reserve(s["table"], s["lens"], s["refs"], s["add"], s["page"], status=s["status"])
        return s["table"], s["lens"], s["refs"], s["status"]
    if op == "fork":
        binding.approxifer_cache_fork(s["pools"], s["table"], s["lens"], s["refs"], s["parents"], table_out=s["table_out"],
                                      lens_out=s["lens_out"], refs_out=s["refs_out"], status=s["status"],
                                      workspace=s["workspace"])
        return s["table_out"], s["lens_out"], s["refs_out"], s["status"], s["pools"]
    binding.approxifer_cache_compact(s["pools"], s["table"], s["lens"], s["refs"], moved=s["moved"], live=s["live"],
                                     workspace=s["workspace"])
    return s["table"], s["refs"], s["moved"], s["live"], s["pools"]


def work(case):
    B, page, lens = case["B"], case["page"], _lengths(case)
    size = 4 if case["dtype"] == "float32" else 2
    if case["op"] in ("append", "attend"):
        heads, kv, dim, n = case["heads"], case["kv"], case["dim"], _new(case)
        T = float(n.sum())
        if case["op"] == "append":
            values = T * (heads + 2 * kv) * dim
            return {"bytes": 2.0 * size * values + 4.0 * T * (case["axes"] if case["axes"] > 1 else 0),
                    "flops": T * (heads + kv) * (dim * (4 if case["norm"] else 0) + 6.0 * case["pairs"])}
        pairs = keys = 0.0
        for length, new in zip(lens, n):
            first = int(length - new)
            pairs += float(_visible(case, np.arange(first, int(length))).sum())
            seen = int(length)
            if case["window"]:                                # the sinks, and what the first of its windows begins with
                lo = max(0, first - case["window"] + 1)
                seen = min(case["sinks"], lo) + int(length) - lo
            keys += seen
        return {"bytes": size * dim * (2.0 * T * heads + 2.0 * keys * kv), "flops": 4.0 * dim * heads * pairs}
    columns, P = -(-int(lens.max()) // page) + 2, case["pages"]
    page_bytes = case["planes"] * case["kv"] * page * case["dim"] * size
    if case["op"] == "reserve":
        return {"bytes": 4.0 * (B + B + B + P), "flops": float(P)}
    if case["op"] == "fork":
        children = case["children"]
        copies = int((lens % page != 0).sum()) * max(0, children - 1)
        n = B * children if children else B
        return {"bytes": 4.0 * (B * columns + n * columns + 2 * P) + 2.0 * copies * page_bytes, "flops": float(P)}
    held = int((-(-np.where(np.arange(B) % 3 == 1, 0, lens) // page)).sum())
    # pages lie anywhere: of the live ones the share behind the line moves
    return {"bytes": 4.0 * (2 * B * columns + 3 * P) + 2.0 * held * (P - held) / P * page_bytes, "flops": float(P)}


# ---- the same results in 64 bits, from the definitions ------------------------------------------------------------------
def _exact_append(s, case):
    starts, lens, table = (s[x].cpu().numpy() for x in ("starts", "lens", "table"))
    n = np.diff(starts)
    place = np.concatenate([np.arange(l - m, l) for l, m in zip(lens, n)])
    page = np.concatenate([row[np.arange(l - m, l) // case["page"]] for row, l, m in zip(table, lens, n)])
    page, slot = (torch.as_tensor(x, device=DEVICE).long() for x in (page, place % case["page"]))
    R, axis = case["pairs"], np.minimum(np.arange(case["pairs"]) * case["axes"] // case["pairs"], case["axes"] - 1)
    position = s["positions"].cpu().numpy() if s["positions"] is not None else place[:, None]
    angle = position[:, axis].astype(np.float64) * np.exp(-np.arange(R) / R * math.log(BASE))
    turn = torch.polar(torch.ones((), dtype=torch.float64), torch.as_tensor(angle))
    turn = turn.to(DEVICE)[:, None]

    def rotated(x, weight):
        y = x.double()
        if weight is not None:
            y = y / (y.square().sum(2, keepdim=True) / case["dim"] + EPS).sqrt() * weight.double()
        pair = y[..., :2 * R].unflatten(2, (2, R)).transpose(2, 3) if case["split"] else y[..., :2 * R].unflatten(2, (R, 2))
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        y[..., :2 * R] = (z.transpose(2, 3) if case["split"] else z).flatten(2)
        return y

    pools = [p.double() for p in (s["k_pool"], s["v_pool"])]
    pools[0][page, :, slot] = rotated(s["k"].clone(), s["k_weight"])
    pools[1][page, :, slot] = s["v"].double()
    return rotated(s["q"].clone(), s["q_weight"]), pools[0], pools[1], s["status"].zero_()


def _exact_attend(s, case):
    starts, lens, table = (s[x].cpu().numpy() for x in ("starts", "lens", "table"))
    heads, kv, dim, page = case["heads"], case["kv"], case["dim"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for b in range(case["B"]):
        length, r0, r1 = int(lens[b]), int(starts[b]), int(starts[b + 1])
        used = torch.as_tensor(table[b, :-(-length // page)], device=DEVICE).long()
        k, v = (s[x][used].double().transpose(0, 1).reshape(kv, -1, dim)[:, :length] for x in ("k_pool", "v_pool"))
        for c0 in range(r0, r1, 2048):
            c1 = min(r1, c0 + 2048)
            p = torch.arange(length - (r1 - c0), length - (r1 - c1), device=DEVICE)
            far = p[:, None] - torch.arange(length, device=DEVICE)                         # how far back a key lies
            seen = far >= 0
            if case["window"]:
                seen &= (far < case["window"]) | (torch.arange(length, device=DEVICE) < case["sinks"])
            for h in range(heads):
                w = torch.mm(s["q"][c0:c1, h].double(), k[h * kv // heads].t().contiguous()) / math.sqrt(dim)
                w = torch.softmax(w.masked_fill_(~seen, -math.inf), dim=1)
                out[c0:c1, h] = torch.mm(w, v[h * kv // heads])
    return out, s["status"].zero_()


def _exact_pages(s, case):
    """Tables in plain Python; the pools as they have to stand afterwards."""
    s["state"].copy_(s["kept"])
    table, lens, refs = (s[x].cpu().numpy().copy() for x in ("table", "lens", "refs"))
    page, P, n = case["page"], case["pages"], case["B"]
    if case["op"] == "reserve":
        free, status = list(np.flatnonzero(refs == 0)), np.zeros(n, np.int32)
        for b, add in enumerate(s["add"].cpu().numpy()):
            old, new = -(-lens[b] // page), -(-(lens[b] + add) // page)
            if new - old > len(free):
                raise ValueError("the cases leave room for every sequence")
            table[b, old:new], free = free[:new - old], free[new - old:]
            refs[table[b, old:new]] = 1
            lens[b] += add
        return _ints(table), _ints(lens), _ints(refs), _ints(status)
    pools = s["pools"]
    if case["op"] == "fork":
        parents = s["parents"].cpu().numpy()
        rows = np.full((len(parents), table.shape[1]), -1, np.int32)
        length = np.array([lens[p] if p >= 0 else 0 for p in parents], np.int32)
        for b in range(n):
            refs[table[b, :-(-lens[b] // page)]] -= 1
        for i, p in enumerate(parents):
            rows[i, :length[i] // page] = table[p, :length[i] // page]
            refs[rows[i, :length[i] // page]] += 1
        wants = [(i, int(table[p, length[i] // page])) for i, p in enumerate(parents) if p >= 0 and length[i] % page]
        again = []
        for i, source in wants:                               # in order: the first to want a page that nobody holds has it
            if refs[source] == 0:
                rows[i, length[i] // page], refs[source] = source, 1
            else:
                again.append((i, source))
        free = np.flatnonzero(refs == 0)
        for (i, source), target in zip(again, free):
            rows[i, length[i] // page], refs[target] = target, 1
            pools[:, target] = pools[:, source]
        return _ints(rows), _ints(length), _ints(refs), _ints(np.zeros(len(parents))), pools.double()
    alive = np.flatnonzero(refs)
    live = len(alive)
    moved = np.full(P, -1, np.int32)
    moved[alive] = alive
    for a, b in zip(alive[alive >= live], np.flatnonzero(refs[:live] == 0)):
        moved[a] = b
        pools[:, b] = pools[:, a]
    after = np.zeros_like(refs)
    after[moved[alive]] = refs[alive]
    return _ints(np.where(table >= 0, moved[table], -1)), _ints(after), _ints(moved), _ints([live]), pools.double()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(s, case)
    if case["op"] != "attend":
        return _exact_pages(s, case)
    if work(case)["flops"] > 1.5e12:
        return None
    return _exact_attend(s, case)
