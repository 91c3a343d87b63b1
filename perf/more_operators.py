"""What the speed of three more cached-sequence operators is measured on: attention of sequences that share a prefix, attention that
adds up the weights which every cached token is given, and eviction of the tokens that were given least.

A case is a plain dict; `prepare` makes what a serving program holds before the call (inputs, pools, page tables, output
buffers, workspace), `run` is one pass: through the binding where `own` is true, else in elementary torch operations in 32
bits.  `exact` computes the same from the definitions in 64 bits.  Fields of a case:

  op          "shared" | "mass" | "evict"
  dtype       "float32" | "float16" | "bfloat16": of everything that holds vectors
  B           sequences: one per worker of each group, or per request
  heads, kv   query heads, heads of the cache;  dim  floats per head
  page        tokens per page
  short, long sequence b's length lies between the two (the first has `long`), new tokens included; of "shared": of what is its own
  new         new tokens per sequence; 0: the whole sequence is new (a prompt), of "shared": all that is its own
  clusters, prefix, prefix_short   of shared: how many prefixes there are, and how long (the first is `prefix` tokens)
  planes, budget, first, recent    of evict: pools (two per layer), tokens that a sequence keeps, the ones that always stay
  common      of evict: tokens of a prompt that all sequences begin with and whose full pages they share
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
SIZES = {"float32": 4, "float16": 2, "bfloat16": 2}


def listed():
    def shared(name, **f):
        return dict({"name": name, "op": "shared", "page": 16, "clusters": 1, "prefix_short": f["prefix"]}, **f)

    def mass(name, **f):
        return dict({"name": name, "op": "mass", "page": 16}, **f)

    def evict(name, **f):
        return dict({"name": name, "op": "evict", "page": 16, "common": 0}, **f)

    return [
        # A prompt that all workers share, and the next token of each: one group's 24 workers behind a prompt of 500 tokens (12
        # heads of 64, the text workload's 768 floats); the workers of eight groups behind a long one; and requests that came in with
        # sixteen prompts of different lengths.
        shared("shared_token_group", dtype="float32", B=24, heads=12, kv=12, dim=64, prefix=500, short=1, long=144, new=1),
        shared("shared_token_long", dtype="bfloat16", B=192, heads=32, kv=8, dim=128, prefix=8003, short=33, long=512, new=1),
        shared("shared_token_prompts", dtype="float16", B=200, heads=16, kv=2, dim=128, clusters=16, prefix_short=300, prefix=4099,
               short=1, long=301, new=1),
        # The queries' own texts (128 tokens each) read at once behind the prompt.
        shared("shared_text", dtype="bfloat16", B=96, heads=12, kv=12, dim=64, prefix=2011, short=128, long=128, new=0),
        # Weights added up: the next token of one group's workers, and of long sequences; prompts, whose tokens are all new; and
        # short ragged texts with a head size that is no power of two.
        mass("mass_token_group", dtype="float32", B=24, heads=12, kv=12, dim=64, short=90, long=129, new=1),
        mass("mass_token_long", dtype="bfloat16", B=16, heads=32, kv=8, dim=128, short=4001, long=32768, new=1),
        mass("mass_prompts", dtype="bfloat16", B=2, heads=32, kv=8, dim=128, short=2100, long=4001, new=0),
        mass("mass_texts", dtype="float16", B=48, heads=16, kv=16, dim=80, short=33, long=129, new=0),
        # Eviction: one group's workers that have grown a little beyond what they may keep (two layers); long sequences cut to half
        # (three layers); and workers that hold the pages of a common prompt together, which takes pages of their own.
        evict("evict_group", dtype="float32", B=24, kv=12, dim=64, short=129, long=160, planes=4, budget=128, first=4, recent=32),
        evict("evict_long", dtype="bfloat16", B=32, kv=8, dim=128, short=3001, long=4500, planes=6, budget=2048, first=4, recent=256),
        evict("evict_forked", dtype="float16", B=48, kv=4, dim=128, short=700, long=1001, planes=8, budget=600, first=4, recent=64,
              common=500),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one token to prompts, one sequence to many, odd sizes, each type."""
    op = rng.choice(["shared", "shared", "mass", "mass", "evict"])
    c = {"op": op, "dtype": rng.choice(["float32", "float16", "bfloat16", "bfloat16"]), "page": rng.choice([8, 16, 16, 32, 64, 128])}
    c["kv"] = kv = rng.choice([1, 2, 4, 8, 8, 12])
    c["dim"] = dim = rng.choice([32, 64, 64, 72, 80, 96, 128, 128, 128, 160, 256])
    token = 2 * SIZES[c["dtype"]] * kv * dim                  # bytes of keys and values of a token
    if op == "evict":
        # at most 1.5 GB of pools
        c["B"] = B = _log_int(rng, 1, 64)
        c["long"] = _log_int(rng, 24, 5000)
        c["short"] = max(8, int(c["long"] * rng.choice([0.3, 0.7, 1.0])))
        most = int(1.5e9 / token / B)
        while c["long"] + c["page"] > most:
            c["long"], c["short"] = c["long"] // 2 + 4, max(8, c["short"] // 2)
        c["planes"] = 2 * max(1, min(4, int(most / (c["long"] + c["page"]))))
        c["budget"] = max(4, int(c["long"] * rng.choice([0.25, 0.5, 0.9])))
        c["first"], c["recent"] = rng.choice([0, 1, 4]), rng.choice([0, c["budget"] // 8, c["budget"] // 3])
        c["first"] = min(c["first"], c["budget"] - c["recent"])
        c["common"] = rng.choice([0, 0, c["short"] // 2])
        return c
    c["heads"] = heads = kv * rng.choice([1, 1, 2, 3, 4, 8])
    single = rng.random() < 0.6
    c["new"] = rng.choice([1, 1, 1, 2, 5]) if single else 0
    c["B"] = B = _log_int(rng, 1, 256) if single else _log_int(rng, 1, 48)
    # at most 100 GFLOP and 1 GB of cache in a pass
    flops = 1e11 / (4.0 * dim * heads * B)                    # pairs of a sequence
    keys = int(1e9 / token)
    if op == "mass":
        most = keys // B
        most = min(most, int(flops / c["new"])) if single else min(most, int(math.sqrt(2.0 * flops)))
        c["long"] = max(c["new"], 2, min(most, _log_int(rng, 6, 32768) if single else _log_int(rng, 6, 4000)))
    else:
        c["clusters"] = min(B, rng.choice([1, 1, 2, 7, 16]))
        longest = keys // B // 2
        c["long"] = max(c["new"], 2, min(longest, _log_int(rng, 4, 1000) if single else _log_int(rng, 4, 400)))
        rows = c["new"] if single else c["long"]
        most = max(1, min(keys // 2 // c["clusters"], int(flops / rows) - c["long"]))
        c["prefix"] = max(1, min(most, _log_int(rng, 16, 16384)))
        c["prefix_short"] = max(1, int(c["prefix"] * rng.choice([0.1, 0.7, 1.0])))
    c["short"] = max(1, c["new"], int(c["long"] * rng.choice([0.3, 0.9, 1.0])))
    return c


# ---- what a case fixes whatever the seed --------------------------------------------------------------------------------
def _spread(short, long, n):
    """int64 [n]: spread over short..long, the first the longest."""
    i = np.arange(n)
    return long - np.floor((long - short + 1) * ((i * 0.6180339887498949) % 1.0)).astype(np.int64)


def _clusters(case):
    """The first sequence of every cluster and the end, and how long its prefix is."""
    n = case["clusters"]
    return (np.arange(n + 1) * case["B"]) // n, _spread(case["prefix_short"], case["prefix"], n)


def _prefixes(case):
    """Of every sequence: the tokens that it has in common with its cluster's others."""
    if case["op"] != "shared":
        return np.full(case["B"], case.get("common", 0), dtype=np.int64)
    groups, prefix = _clusters(case)
    return np.repeat(prefix, np.diff(groups))


def _lengths(case):
    lens = _spread(case["short"], case["long"], case["B"])
    return lens + _prefixes(case) if case["op"] == "shared" else lens


def _new(case):
    fresh = _spread(case["short"], case["long"], case["B"])
    return fresh if case["new"] == 0 else np.minimum(fresh, case["new"])


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _ints(values):
    return torch.as_tensor(np.asarray(values), dtype=torch.int32, device=DEVICE)


def _table(g, lens, common, cluster, page, spare):
    """int32 [B, columns] and the number of pages: every sequence's pages at places drawn from all of them (the full pages of the
    `common` first tokens of a cluster are its first sequence's), -1 behind its last one; and whose copy of a page that is only
    partly common each sequence has to begin with: (copies, originals, slots), as lists."""
    B = len(lens)
    count = -(-lens // page)
    columns = int(count.max()) + 1
    table = np.full((B, columns), -1, dtype=np.int64)
    first, copies, used = {}, [], 0
    for b in range(B):
        full = 0
        if cluster[b] in first:
            leader = first[cluster[b]]
            full = int(common[b]) // page
            table[b, :full] = table[leader, :full]
            if common[b] % page:
                copies.append((b, leader, full, int(common[b] % page)))
        else:
            first[cluster[b]] = b
        table[b, full:count[b]] = np.arange(used, used + count[b] - full)
        used += int(count[b] - full)
    P = used + 3
    order = torch.randperm(P, generator=g, device=DEVICE)
    at = torch.as_tensor(table, device=DEVICE)
    table = torch.where(at >= 0, order[at.clamp(min=0)], -1)
    return table.to(torch.int32).contiguous(), P, copies


def _equalise(pools, table, copies):
    """The slots of partly common pages that every sequence has a copy of.  pools [.., P, kv, page, dim]."""
    for slots in sorted({c[3] for c in copies}):
        these = [c for c in copies if c[3] == slots]
        to, from_ = (torch.stack([table[c[i], c[2]] for c in these]).long() for i in (0, 1))
        pools[..., to, :, :slots, :] = pools[..., from_, :, :slots, :]


def prepare(case, seed):
    g = _generator(seed)
    op, t, B, page, kv, dim = case["op"], TYPES[case["dtype"]], case["B"], case["page"], case["kv"], case["dim"]
    lens, common = _lengths(case), _prefixes(case)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE).to(t)

    groups = _clusters(case)[0] if op == "shared" else np.array([0, B])
    cluster = np.repeat(np.arange(len(groups) - 1), np.diff(groups)) if op == "shared" or case.get("common") else np.arange(B)
    table, P, copies = _table(g, lens, common, cluster, page, 3)
    s = {"op": op, "page": page, "B": B, "table": table, "status": torch.empty((B,), dtype=torch.int32, device=DEVICE)}
    if op in ("shared", "mass"):
        heads, n = case["heads"], _new(case)
        T = int(n.sum())
        s["lens"], s["starts"] = _ints(lens), _ints(np.concatenate([[0], np.cumsum(n)]))
        s["q"] = normal(T, heads, dim)
        pools = normal(2, P, kv, page, dim)
        _equalise(pools, table, copies)
        s["k_pool"], s["v_pool"] = pools[0], pools[1]
        s["out"] = torch.empty((T, heads, dim), dtype=t, device=DEVICE)
        s["max_rows"], s["max_len"] = int(n.max()), int(lens.max())
        if op == "shared":
            s["clusters"], s["prefix"] = [int(x) for x in groups], [int(x) for x in _clusters(case)[1]]
            s["groups"], s["shared"] = _ints(groups), _ints(_clusters(case)[1])
            s["max_shared"] = case["prefix"]
        else:
            # what the tokens before these have given; nothing yet to the new ones
            kept = torch.rand((B, table.shape[1] * page), generator=g, device=DEVICE) * 4.0
            place = torch.arange(kept.shape[1], device=DEVICE)
            s["before"] = torch.where(place < _ints(lens - n)[:, None], kept, 0.0)
            s["mass"] = torch.empty_like(s["before"])
        if own:
            from paper_2109_09868_amd import binding
            if op == "shared":
                need = binding.approxifer_attend_shared_workspace_bytes(T, B, case["clusters"], heads, kv, dim, t, s["max_rows"],
                                                                        s["max_len"], s["max_shared"])
            else:
                need = binding.approxifer_attend_mass_workspace_bytes(T, B, heads, kv, dim, t, s["max_rows"], s["max_len"])
            s["workspace"] = torch.empty((max(need, 16),), dtype=torch.uint8, device=DEVICE)
        return s

    s["pools"] = torch.empty((case["planes"], P, kv, page, dim), dtype=t, device=DEVICE)
    for plane in s["pools"]:
        plane.normal_(generator=g)
    _equalise(s["pools"], table, copies)
    if case["common"]:                                        # room for what the sequences no longer share
        extra = B * (case["common"] // page + 1)
        s["pools"] = torch.cat([s["pools"], torch.zeros_like(s["pools"][:, :1]).expand(-1, extra, -1, -1, -1)], dim=1)
        P += extra
    refs = torch.zeros((P,), dtype=torch.int32, device=DEVICE)
    refs.index_add_(0, table[table >= 0].long(), torch.ones_like(table[table >= 0]))
    # what attention gives: most to few, and nothing at all to some
    mass = torch.exp(2.0 * torch.randn((B, table.shape[1] * page), generator=g, device=DEVICE))
    mass *= torch.rand(mass.shape, generator=g, device=DEVICE) > 0.05
    mass *= torch.arange(mass.shape[1], device=DEVICE) < _ints(lens)[:, None]
    s["before"], s["mass"] = mass, torch.empty_like(mass)
    s["kept_state"] = torch.cat([table.flatten(), _ints(lens), refs])
    s["state"] = state = torch.empty_like(s["kept_state"])
    cells = table.numel()
    s["table"], s["lens"], s["refs"] = state[:cells].view(table.shape), state[cells:cells + B], state[cells + B:]
    s["budget"], s["first"], s["recent"] = case["budget"], case["first"], case["recent"]
    s["kept"] = torch.empty((B, case["budget"]), dtype=torch.int32, device=DEVICE)
    if own:
        from paper_2109_09868_amd import binding
        need = binding.approxifer_cache_evict_workspace_bytes(B, case["budget"], P, page)
        s["workspace"] = torch.empty((need,), dtype=torch.uint8, device=DEVICE)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------
def _gathered(pool, table):
    """[B, kv, keys, dim] in 32 bits: what the tables' pages hold."""
    x = pool[table.long().clamp(min=0)].float().transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[4])


def _padded_rows(s):
    """The rows [B, kv, most * group, dim] in 32 bits, places [B, most], where each row stands in them, and its sequence."""
    q, B, kv = s["q"], s["B"], s["k_pool"].shape[1]
    T, heads, dim = q.shape
    R = s["max_rows"]
    starts, lens = s["starts"].long(), s["lens"].long()
    n = starts[1:] - starts[:-1]
    i = torch.arange(R, device=DEVICE)
    rows = q[(starts[:-1, None] + i).clamp(max=T - 1)].float()
    rows = rows.view(B, R, kv, heads // kv, dim).permute(0, 2, 1, 3, 4).reshape(B, kv, -1, dim)
    t = torch.arange(T, device=DEVICE)
    b = torch.searchsorted(starts, t, right=True) - 1
    return rows, (lens - n)[:, None] + i, i < n[:, None], b, t - starts[b]


def _plain_mass(s):
    kv = s["k_pool"].shape[1]
    T, heads, dim = s["q"].shape
    R, B, columns = s["max_rows"], s["B"], -(-s["max_len"] // s["page"])
    k, v = (_gathered(s[x], s["table"][:, :columns]) for x in ("k_pool", "v_pool"))
    rows, place, real, b, at = _padded_rows(s)
    score = torch.matmul(rows, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(dim)).view(B, kv, R, heads // kv, -1)
    key = torch.arange(k.shape[2], device=DEVICE)
    score.masked_fill_((key > place[:, :, None])[:, None, :, None, :], -math.inf)
    weight = score.sub_(score.amax(4, keepdim=True)).exp_()
    weight.div_(weight.sum(4, keepdim=True))
    out = torch.matmul(weight.view(B, kv, R * (heads // kv), -1), v).view(B, kv, R, heads // kv, dim)
    s["out"].copy_(out.permute(0, 2, 1, 3, 4).reshape(B, R, heads, dim)[b, at])
    weight.masked_fill_(~real[:, None, :, None, None], 0.0)
    s["mass"][:, :key.shape[0]] += weight.sum((1, 2, 3))
    s["status"].zero_()
    return s["out"], s["mass"], s["status"]


def _plain_shared(s):
    kv = s["k_pool"].shape[1]
    T, heads, dim = s["q"].shape
    R, B, page, group = s["max_rows"], s["B"], s["page"], heads // kv
    rows, place, real, b, at = _padded_rows(s)
    scale = 1.0 / math.sqrt(dim)
    # what every sequence has of its own: its pages from the one on that holds its first own token
    sizes = [y - x for x, y in zip(s["clusters"], s["clusters"][1:])]
    prefix = s["shared"].long().repeat_interleave(torch.as_tensor(sizes, device=DEVICE), output_size=B)
    low = prefix // page
    columns = min(s["table"].shape[1], (s["max_len"] - min(s["prefix"])) // page + 2)
    column = low[:, None] + torch.arange(columns, device=DEVICE)
    mine = s["table"].gather(1, column.clamp(max=s["table"].shape[1] - 1))
    k, v = _gathered(s["k_pool"], mine), _gathered(s["v_pool"], mine)
    key = (low * page)[:, None] + torch.arange(columns * page, device=DEVICE)                   # [B, keys]
    score = torch.matmul(rows, k.transpose(2, 3).contiguous()).mul_(scale).view(B, kv, R, group, -1)
    hidden = (key[:, None] > place[:, :, None]) | (key < prefix[:, None])[:, None]
    score.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    top = score.amax(4, keepdim=True)
    rows = rows.view(B, kv, R, group, dim)
    for c, (x, y) in enumerate(zip(s["clusters"], s["clusters"][1:])):
        used = s["table"][x:x + 1, :-(-s["prefix"][c] // page)]
        pk, pv = (_gathered(s[p], used)[0, :, :s["prefix"][c]] for p in ("k_pool", "v_pool"))
        these = rows[x:y].permute(1, 0, 2, 3, 4).reshape(kv, -1, dim)
        far = torch.matmul(these, pk.transpose(1, 2).contiguous()).mul_(scale).view(kv, y - x, R, group, -1).transpose(0, 1)
        most = torch.maximum(far.amax(4, keepdim=True), top[x:y])
        far = (far - most).exp_()
        near = (score[x:y] - most).exp_()
        total = far.sum(4, keepdim=True) + near.sum(4, keepdim=True)
        out = torch.matmul(near.view(y - x, kv, R * group, -1), v[x:y]).view(y - x, kv, R, group, dim)
        out += torch.matmul(far.transpose(0, 1).reshape(kv, (y - x) * R * group, -1), pv).view(kv, y - x, R, group, dim).transpose(0, 1)
        rows[x:y] = out.div_(total)
    s["out"].copy_(rows.permute(0, 2, 1, 3, 4).reshape(B, R, heads, dim)[b, at])
    s["status"].zero_()
    return s["out"], s["status"]


def _plain_evict(s):
    table, lens, refs, mass, page, budget = s["table"], s["lens"].long(), s["refs"], s["mass"], s["page"], s["budget"]
    B, columns = table.shape
    L, P = mass.shape[1], refs.shape[0]
    place = torch.arange(L, device=DEVICE)
    there = place < lens[:, None]
    fixed = there & ((place < s["first"]) | (place >= lens[:, None] - s["recent"]))
    # in the order in which they stay: the fixed ones, then by mass, the earlier first
    rank = torch.where(fixed, math.inf, torch.where(there, mass, -math.inf))
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices
    stays = torch.zeros_like(there).scatter_(1, order[:, :budget], True) & there
    new = stays.sum(1)
    kept = torch.sort((~stays).to(torch.int8), dim=1, stable=True).indices[:, :budget]
    slot = torch.arange(budget, device=DEVICE)
    real = slot < new[:, None]
    cut = lens > budget
    # pages that change: from the one with the first place that moves on, or that holds the end
    first_move = torch.where(real & (kept != slot), slot, budget).amin(1)
    low = torch.minimum(first_move // page, torch.where(new % page != 0, new // page, columns))
    column = torch.arange(columns, device=DEVICE)
    before, after = (lens + page - 1) // page, (new + page - 1) // page
    changes = cut[:, None] & (column >= low[:, None]) & (column < after[:, None])
    held = table.clamp(min=0).long()
    wants = changes & (refs[held] > 1)
    upto = wants.flatten().to(torch.int64).cumsum(0).view(B, columns)
    free = torch.sort((refs != 0).to(torch.int8), stable=True).indices
    fresh = torch.where(wants, free[(upto - 1).clamp(0, P - 1)], held)
    drops = cut[:, None] & (column >= after[:, None]) & (column < before[:, None])
    gone = torch.where(wants | drops, held, P).flatten()
    count = torch.cat([refs, refs.new_zeros(1)])
    count.index_add_(0, gone, -torch.ones_like(gone, dtype=torch.int32))
    count.index_add_(0, torch.where(wants, fresh, P).flatten(), torch.ones_like(gone, dtype=torch.int32))
    # every kept token of the changed pages, at once; one that does not move is written where it stands
    source = held.gather(1, kept // page)
    target = fresh.gather(1, (slot // page).clamp(max=columns - 1).expand(B, -1))
    moves = cut[:, None] & real & (slot >= low[:, None] * page)
    b, i = torch.nonzero(moves, as_tuple=True)
    pools = s["pools"]
    for plane in pools:
        plane[target[b, i], :, i % page] = plane[source[b, i], :, kept[b, i] % page]
    moved = torch.where(real, mass.gather(1, kept), 0.0)
    mass.copy_(torch.where(cut[:, None], torch.cat([moved, mass.new_zeros(B, max(0, L - budget))], dim=1)[:, :L], mass))
    refs.copy_(count[:P])
    table.copy_(torch.where(drops, -1, torch.where(wants, fresh.to(torch.int32), table)))
    s["lens"].copy_(torch.where(cut, new, lens))
    s["kept"].copy_(torch.where(real, kept, -1))
    s["status"].zero_()
    return s["table"], s["lens"], refs, mass, s["kept"], s["status"], pools


def run(s):
    op = s["op"]
    if "before" in s:                                         # the sequences as they stood before the step
        s["mass"].copy_(s["before"])
    if "kept_state" in s:
        s["state"].copy_(s["kept_state"])
    if not own:
        return {"shared": _plain_shared, "mass": _plain_mass, "evict": _plain_evict}[op](s)
    from paper_2109_09868_amd import binding
    if op == "shared":
        return binding.approxifer_attend_shared(s["q"], s["k_pool"], s["v_pool"], s["table"], s["lens"], s["starts"], s["groups"],
                                                s["shared"], s["max_rows"], s["max_len"], s["max_shared"], out=s["out"],
                                                status=s["status"], workspace=s["workspace"])
    if op == "mass":
        binding.approxifer_attend_mass(s["q"], s["k_pool"], s["v_pool"], s["table"], s["lens"], s["starts"], s["mass"], s["max_rows"],
                                       s["max_len"], out=s["out"], status=s["status"], workspace=s["workspace"])
        return s["out"], s["mass"], s["status"]
    binding.approxifer_cache_evict(s["pools"], s["table"], s["lens"], s["refs"], s["mass"], s["budget"], first=s["first"],
                                   recent=s["recent"], kept=s["kept"], status=s["status"], workspace=s["workspace"])
    return s["table"], s["lens"], s["refs"], s["mass"], s["kept"], s["status"], s["pools"]


def work(case):
    B, page, lens, size = case["B"], case["page"], _lengths(case), SIZES[case["dtype"]]
    kv, dim = case["kv"], case["dim"]
    if case["op"] == "evict":
        kept = float(np.where(lens > case["budget"], case["budget"] - case["first"], 0).sum())
        return {"bytes": 2.0 * kept * case["planes"] * kv * dim * size + 4.0 * (float(lens.sum()) + 3.0 * kept), "flops": float(lens.sum())}
    n = _new(case)
    T = float(n.sum())
    pairs = float((n * (lens - n) + n * (n + 1) / 2.0).sum())
    rows = 2.0 * T * case["heads"] * dim
    if case["op"] == "shared":
        keys = float(_clusters(case)[1].sum() + (lens - _prefixes(case)).sum())
        return {"bytes": size * (rows + 2.0 * keys * kv * dim), "flops": 4.0 * dim * case["heads"] * pairs}
    keys = float(lens.sum())
    # scores of prompts are formed twice: a token's weight needs its row's total
    return {"bytes": size * (rows + 2.0 * keys * kv * dim) + 8.0 * keys,
            "flops": (6.0 if case["new"] == 0 else 4.0) * dim * case["heads"] * pairs}


# ---- the same results in 64 bits, from the definitions ------------------------------------------------------------------
def _exact_attend(s, case):
    """One sequence after the other, all of its keys at once, head by head."""
    starts, lens, table = (s[x].cpu().numpy() for x in ("starts", "lens", "table"))
    heads, kv, dim, page = case["heads"], case["kv"], case["dim"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    mass = s["before"].double() if case["op"] == "mass" else None
    for b in range(case["B"]):
        length, r0, r1 = int(lens[b]), int(starts[b]), int(starts[b + 1])
        used = torch.as_tensor(table[b, :-(-length // page)], device=DEVICE).long()
        k, v = (s[x][used].double().transpose(0, 1).reshape(kv, -1, dim)[:, :length] for x in ("k_pool", "v_pool"))
        last = torch.arange(length - (r1 - r0), length, device=DEVICE)[:, None]
        seen = torch.arange(length, device=DEVICE) <= last
        for h in range(heads):
            w = torch.mm(s["q"][r0:r1, h].double(), k[h * kv // heads].t().contiguous()) / math.sqrt(dim)
            w = torch.softmax(w.masked_fill_(~seen, -math.inf), dim=1)
            out[r0:r1, h] = torch.mm(w, v[h * kv // heads])
            if mass is not None:
                mass[b, :length] += w.sum(0)
    return (out, s["status"].zero_()) if mass is None else (out, mass, s["status"].zero_())


def _exact_evict(s, case):
    """Tables in plain Python; the pools as they have to stand afterwards."""
    s["state"].copy_(s["kept_state"])
    table, lens, refs, mass = (s[x].cpu().numpy().copy() for x in ("table", "lens", "refs", "before"))
    page, budget, first, recent, pools = case["page"], case["budget"], case["first"], case["recent"], s["pools"]
    mass, kept = mass.astype(np.float64), np.full((case["B"], budget), -1, np.int32)
    held, moves, taken = refs.copy(), [], 0
    free = np.flatnonzero(refs == 0)
    for b, length in enumerate(int(x) for x in lens):
        if length <= budget:
            kept[b, :length] = np.arange(length)
            continue
        inner = np.arange(first, length - recent)
        best = inner[np.lexsort((inner, -mass[b, inner]))][:budget - first - recent]
        stays = np.sort(np.concatenate([np.arange(first), best, np.arange(length - recent, length)])).astype(np.int64)
        kept[b] = stays
        shifted = np.flatnonzero(stays != np.arange(budget))
        begin = int(shifted[0]) // page if len(shifted) else budget // page
        sources = table[b, stays // page].copy()
        for j in range(begin, -(-budget // page)):
            page_at = table[b, j]
            if held[page_at] > 1:
                refs[page_at] -= 1
                table[b, j] = free[taken]
                refs[free[taken]] = 1
                taken += 1
        for j in range(-(-budget // page), -(-length // page)):
            refs[table[b, j]] -= 1
            table[b, j] = -1
        i = np.arange(begin * page, budget)
        moves.append((table[b, i // page], i % page, sources[i], stays[i] % page))
        mass[b, :budget], mass[b, budget:] = mass[b, stays], 0.0
        lens[b] = budget
    if moves:
        to, at, from_, was = (torch.as_tensor(np.concatenate(x).astype(np.int64), device=DEVICE) for x in zip(*moves))
        for plane in pools:
            plane[to, :, at] = plane[from_, :, was].clone()
    return (_ints(table), _ints(lens), _ints(refs), torch.as_tensor(mass, device=DEVICE), _ints(kept), s["status"].zero_(), pools.double())


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "evict":
        return _exact_evict(s, case)
    if work(case)["flops"] > 1.5e12:
        return None
    return _exact_attend(s, case)
