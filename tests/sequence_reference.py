"""The cached-sequence operators in 64 bits, row by row from their definitions, and the inputs their tests share."""
import math

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U32 = 2.0 ** -24                                              # half a step of float32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def cache(seed, dtype, lens, new, kv, dim, page, spare=3, columns=None, normal=True):
    """A cache on the CPU: pools whose slots behind every sequence are NaN, and the descriptor's tensors."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    count = [-(-l // page) for l in lens]
    M = max(max(count, default=0), 1) if columns is None else columns
    P = sum(count) + spare
    order = torch.randperm(P, generator=g)
    table = torch.full((B, M), -7, dtype=torch.int32)
    k_pool = torch.full((P, kv, page, dim), math.nan, dtype=dtype)
    v_pool = torch.full((P, kv, page, dim), math.nan, dtype=dtype)
    at = 0
    for b in range(B):
        for j in range(count[b]):
            p = int(order[at])
            at += 1
            table[b, j] = p
            if normal:
                used = min(page, lens[b] - j * page)
                k_pool[p, :, :used] = torch.randn((kv, used, dim), generator=g).to(dtype)
                v_pool[p, :, :used] = torch.randn((kv, used, dim), generator=g).to(dtype)
    starts = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
    return {"table": table, "lens": torch.tensor(lens, dtype=torch.int32), "starts": starts, "k_pool": k_pool, "v_pool": v_pool,
            "page": page, "T": int(sum(new)), "order": order[at:]}


def on(device, c, *names):
    return [c[n].to(device) for n in (names or ("k_pool", "v_pool", "table", "lens", "starts"))]


def held(c, pool, b):
    """float64 [kv, lens[b], dim] of sequence b."""
    length = int(c["lens"][b])
    pages = c["table"][b, :-(-length // c["page"])].long()
    x = c[pool][pages].double().transpose(0, 1)
    return x.reshape(x.shape[0], -1, x.shape[3])[:, :length]


def visible(place, length, window, sinks):
    j = torch.arange(length)
    seen = j <= place
    if window:
        seen &= (j > place - window) | (j < sinks)
    return seen


def attend(c, q, window=0, sinks=0, scale=None):
    """(out float64 [T, Hq, Dh], bound float64 [T, Hq, Dh]): softmax over what each row sees, and how far a float32
    computation may be off.  With u = 2^-24 and all sums in float32, in any order: a score is off by (Dh + 8) u scale sum
    |q k| at most; a weight by twice that for the worst score of its row, and by half a step of the type that it is rounded
    to before the product (16-bit types; half of the smallest step where it is subnormal); the two sums over n keys by (n +
    64) u each; the result by half a step of its type."""
    T, Hq, Dh = q.shape
    dtype = q.dtype
    scale = Dh ** -0.5 if scale is None else scale
    out, bound = torch.zeros((T, Hq, Dh), dtype=torch.float64), torch.zeros((T, Hq, Dh), dtype=torch.float64)
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    for b in range(len(c["lens"])):
        k, v = held(c, "k_pool", b), held(c, "v_pool", b)
        length, t0, t1 = int(c["lens"][b]), int(c["starts"][b]), int(c["starts"][b + 1])
        for t in range(t0, t1):
            place = length - (t1 - t)
            if place < 0:
                continue
            seen = visible(place, length, window, sinks)
            n = int(seen.sum())
            for h in range(Hq):
                kk, vv = k[h * k.shape[0] // Hq][seen], v[h * k.shape[0] // Hq][seen]
                x = q[t, h].double()
                s = kk @ x * scale
                w = torch.softmax(s, 0)
                out[t, h] = w @ vv
                off = 2.0 * (Dh + 8) * U32 * abs(scale) * float((kk.abs() @ x.abs()).max())
                off += 2.0 * (n + 64) * U32 + (half_step(dtype) if dtype != torch.float32 else 0.0)
                bound[t, h] = off * (w @ vv.abs()) + tiny * vv.abs().sum(0) + half_step(dtype) * out[t, h].abs()
    return out, bound


def append(c, q, k, v, freq, q_weight=None, k_weight=None, eps=1e-6, positions=None, axis=None, interleaved=False):
    """(q_out, its bound, k_pool, its bound, v_pool): float64; pools where nothing is written keep their values, bound 0.  A
    norm's sum, root and two products are off by (Dh + 16) u at most, cosine and sine of an angle reduced in float64 by 8 u, the
    rotation's products and sum by 4 u: all relative to the pair's larger values; the result by half a step of its type."""
    T, Hq, Dh = q.shape
    R, page = len(freq), c["page"]
    place = torch.zeros((T,), dtype=torch.long)
    row = torch.zeros((T,), dtype=torch.long)
    for b in range(len(c["lens"])):
        t0, t1 = int(c["starts"][b]), int(c["starts"][b + 1])
        place[t0:t1] = int(c["lens"][b]) - (t1 - t0) + torch.arange(t1 - t0)
        row[t0:t1] = b
    position = place[:, None] if positions is None else positions.long().reshape(T, -1)
    turn = position.double()[:, torch.tensor(np.zeros(R, np.int64) if axis is None else axis, dtype=torch.long)] * torch.tensor(freq)

    def turned(x, weight):
        y = x.double().clone()
        if weight is not None:
            y = y / (y.square().mean(2, keepdim=True) + eps).sqrt() * weight.double()
        z, size = y.clone(), y.abs()
        for i in range(R):
            m, n = (2 * i, 2 * i + 1) if interleaved else (i, i + R)
            cos, sin = turn[:, None, i].cos(), turn[:, None, i].sin()
            z[..., m], z[..., n] = y[..., m] * cos - y[..., n] * sin, y[..., m] * sin + y[..., n] * cos
            size[..., m] = size[..., n] = y[..., m].abs() + y[..., n].abs()
        return z, (Dh + 28) * U32 * size + half_step(x.dtype) * z.abs()

    kz, kb = turned(k, k_weight)
    pools = [c["k_pool"].double(), torch.zeros(c["k_pool"].shape, dtype=torch.float64), c["v_pool"].double()]
    for t in range(T):
        if place[t] < 0:
            continue
        p, s = int(c["table"][row[t], place[t] // page]), int(place[t] % page)
        pools[0][p, :, s], pools[1][p, :, s], pools[2][p, :, s] = kz[t], kb[t], v[t].double()
    return (*turned(q, q_weight), *pools)


# ---- pages, in plain Python ---------------------------------------------------------------------------------------------
def reserve(table, lens, refs, add, page):
    """(table, lens, refs, status): lists in, lists out."""
    M, P = len(table[0]), len(refs)
    table, lens, refs, status = [list(r) for r in table], list(lens), list(refs), [0] * len(lens)
    free = [p for p in range(P) if refs[p] == 0]
    upto, have = 0, len(free)
    for b, a in enumerate(add):
        l = lens[b]
        if l < 0 or a < 0 or l + a > M * page:
            status[b] = 1
            continue
        old, new = -(-l // page), -(-(l + a) // page)
        if l % page and a:
            last = table[b][old - 1]
            if not 0 <= last < P:
                status[b] = 2
                continue
            if refs[last] > 1:
                status[b] = 4
                continue
        upto += new - old
        if new > old and upto > have:
            status[b] = 3
            continue
        for j in range(old, new):
            table[b][j] = free.pop(0)
            refs[table[b][j]] = 1
        lens[b] = l + a
    return table, lens, refs, status


def fork(table, lens, refs, parents, keep, page):
    """(table, lens, refs, status, [(source, target), ..])."""
    B, M, P = len(table), len(table[0]) if table else 0, len(refs)
    refs = list(refs)
    for b in range(B):
        if 0 <= lens[b] <= M * page:
            for p in table[b][:-(-lens[b] // page)]:
                if 0 <= p < P:
                    refs[p] -= 1
    out, length, status, wants = [], [], [], []
    for i, r in enumerate(parents):
        l, st = 0, 0
        if not -1 <= r < B or (keep is not None and keep[i] < 0) or (r >= 0 and not 0 <= lens[r] <= M * page):
            st = 1
        elif r >= 0:
            l = lens[r] if keep is None else min(lens[r], keep[i])
            if any(not 0 <= p < P for p in table[r][:-(-l // page)]):
                l, st = 0, 2
        row = [-1] * M
        for j in range(l // page):
            row[j] = table[r][j]
            refs[row[j]] += 1
        if l % page:
            wants.append((i, table[r][l // page]))
        out.append(row)
        length.append(l)
        status.append(st)
    copies = []
    taken = {}
    for i, p in wants:
        if refs[p] == 0 and p not in taken:
            taken[p] = i
    for p in taken:
        refs[p] = 1
    free = [p for p in range(P) if refs[p] == 0]
    for i, p in wants:
        last = length[i] // page
        if taken.get(p) == i:
            out[i][last] = p
        elif free:
            q = free.pop(0)
            out[i][last] = q
            refs[q] = 1
            copies.append((p, q))
        else:
            for x in out[i][:last]:
                refs[x] -= 1
            out[i], length[i], status[i] = [-1] * M, 0, 3
    return out, length, refs, status, copies


def compact(table, lens, refs, page):
    """(table, refs, moved, live, [(source, target), ..])."""
    P = len(refs)
    alive = [p for p in range(P) if refs[p]]
    live = len(alive)
    moved = [p if refs[p] else -1 for p in range(P)]
    moves = list(zip([p for p in alive if p >= live], [p for p in range(live) if not refs[p]]))
    after = list(refs)
    for a, b in moves:
        moved[a], after[b], after[a] = b, refs[a], 0
    table = [list(r) for r in table]
    for b, row in enumerate(table):
        if 0 <= lens[b] <= len(row) * page:
            for j in range(-(-lens[b] // page)):
                if 0 <= row[j] < P and moved[row[j]] >= 0:
                    row[j] = moved[row[j]]
    return table, after, moved, live, moves
