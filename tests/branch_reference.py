"""Plain forms, in 64 bits and token by token, of the operators for generation that branches over the paged cache.  CPU tensors."""
import math

import torch


def token(pool, layer, page, place):
    """(K, V), each [H_kv, D], of one cached token; pool [layers, pages, 2, H, P, D], values kept as [H, D, P]."""
    _, _, _, H, P, D = pool.shape
    return pool[layer, page, 0, :, place, :], pool[layer, page, 1].reshape(H, D, P)[:, :, place]


def put(pool, layer, page, place, k, v):
    _, _, _, H, P, D = pool.shape
    pool[layer, page, 0, :, place, :] = k
    pool[layer, page, 1].view(H, D, P)[:, :, place] = v


def place_of(pool, table_row, t):
    """(page, place) of token t, or None."""
    P, n_pages = pool.shape[4], pool.shape[1]
    if t < 0 or t // P >= len(table_row):
        return None
    page = int(table_row[t // P])
    return (page, t % P) if 0 <= page < n_pages else None


def append(pool, layer, k, v, cu, lens, table):
    H, D = pool.shape[3], pool.shape[5]
    for b in range(len(lens)):
        for i in range(int(cu[b + 1]) - int(cu[b])):
            at = place_of(pool, table[b], max(int(lens[b]), 0) + i)
            if at is not None:
                r = int(cu[b]) + i
                put(pool, layer, *at, k[r].view(H, D), v[r].view(H, D))


def sees(seen, r, i, j):
    if seen is None:
        return j <= i
    row = seen[r].view(-1).tolist()
    return j // 64 < len(row) and (row[j // 64] >> (j % 64)) & 1 == 1


def attention(pool, layer, q, cu, lens, table, seen, scale):
    """(out, weighted sizes, largest |scale q k| row sums, tokens): out [rows, Hq * D] float64; sizes: sum_t p_t |v_t|; spread: largest scale * sum_d |q_d k_d|
    of a token that the row sees; count: tokens seen.  Rows behind cu[-1] are NaN."""
    H, D = pool.shape[3], pool.shape[5]
    rows, Hq = q.shape[0], q.shape[1] // D
    g = Hq // H
    out = torch.full((rows, Hq, D), math.nan, dtype=torch.float64)
    size, spread, count = torch.zeros(rows, Hq, D, dtype=torch.float64), torch.zeros(rows, Hq, dtype=torch.float64), torch.zeros(rows)
    for b in range(len(lens)):
        n, L = int(cu[b + 1]) - int(cu[b]), max(int(lens[b]), 0)
        at = [place_of(pool, table[b], t) for t in range(min(L + n, table.shape[1] * pool.shape[4]))] if n else []
        there = [t for t, p in enumerate(at) if p is not None]
        if there:
            page, place = (torch.tensor([at[t][x] for t in there]) for x in (0, 1))
            k = pool[layer, page, 0, :, place, :].double()
            v = pool[layer, :, 1].reshape(-1, H, D, pool.shape[4])[page, :, :, place].double()
        for i in range(n):
            r = int(cu[b]) + i
            mine = [x for x, t in enumerate(there) if t < L or sees(seen, r, i, t - L)]
            count[r] = len(mine)
            if not mine:
                out[r] = 0.0
                continue
            for h in range(Hq):
                qk = q[r, h * D:(h + 1) * D].double() * k[mine, h // g]
                p = torch.softmax(scale * qk.sum(1), 0)
                out[r, h] = p @ v[mine, h // g]
                size[r, h] = p @ v[mine, h // g].abs()
                spread[r, h] = abs(scale) * qk.abs().sum(1).max()
    return out.view(rows, -1), size.view(rows, -1), spread.repeat_interleave(D, 1), count


def compact(pool, start, cu, keep, table, to_table):
    """Every token is read before any is written."""
    moves = []
    for b in range(len(start)):
        for i in range(int(cu[b + 1]) - int(cu[b])):
            src, dst = place_of(pool, table[b], int(start[b]) + int(keep[int(cu[b]) + i])), place_of(pool, to_table[b], int(start[b]) + i)
            if src is not None and dst is not None:
                moves.append((src, dst))
    for layer in range(pool.shape[0]):
        held = [tuple(x.clone() for x in token(pool, layer, *src)) for src, _ in moves]
        for (_, dst), (k, v) in zip(moves, held):
            put(pool, layer, *dst, k, v)


def held(row):
    n = 0
    while n < len(row) and row[n] >= 0:
        n += 1
    return n


def fork(pool, parents, lens, table, refs, stride):
    """(new_lens, new_table, lacking) as lists; pool and refs (a list) change."""
    P, n_pages = pool.shape[4], pool.shape[1]
    new_lens, new_table, lacking, waiting = [], [], [], []
    kids = {p: [i for i, x in enumerate(parents) if x == p] for p in range(len(table))}
    for p, row in enumerate(table):
        n = held(row)
        whole = min(max(lens[p], 0), n * P) // P
        for j in range(n):
            if row[j] < n_pages:
                refs[row[j]] += len(kids[p]) - 1 if j < whole else 0 if kids[p] else -1
    for i, p in enumerate(parents):
        if not 0 <= p < len(table):
            new_lens.append(0), new_table.append([-1] * stride), lacking.append(0)
            continue
        n = held(table[p])
        length = min(max(lens[p], 0), n * P)
        keeps = n if kids[p][0] == i else length // P
        new_lens.append(length), new_table.append(list(table[p][:keeps]) + [-1] * (stride - keeps)), lacking.append(0)
        if kids[p][0] != i and length % P:
            waiting.append((i, table[p][length // P], length))
    for i, source, length in waiting:
        free = [x for x in range(n_pages) if refs[x] == 0]
        if not free:
            new_lens[i], lacking[i] = length - length % P, 1
            continue
        refs[free[0]] = 1
        new_table[i][length // P] = free[0]
        for layer in range(pool.shape[0]):
            for t in range(length % P):
                put(pool, layer, free[0], t, *(x.clone() for x in token(pool, layer, source, t)))
    return new_lens, new_table, lacking


def reserve(lens, room, table, refs, P):
    """lacking, a list; table (lists) and refs change."""
    lacking = []
    for row, length in zip(table, lens):
        n, need = held(row), -(-(max(length, 0) + room) // P)
        wants = max(need - n, 0)
        for j in range(n, min(need, len(row))):
            free = [x for x in range(len(refs)) if refs[x] == 0]
            if free:
                refs[free[0]], row[j] = 1, free[0]
                wants -= 1
        lacking.append(wants)
    return lacking


def beam(logits, scores, k, done, end_token):
    """(rows, tokens, scores): lists of n lists of k."""
    n, beams = scores.shape
    rows, tokens, best = [], [], []
    for q in range(n):
        found = []
        for a in range(beams):
            base, l = float(scores[q, a]), logits[q * beams + a].double()
            if done is not None and bool(done[q, a]):
                found.append((base, a, 0, end_token))
                continue
            lse = float(torch.logsumexp(l, 0)) if bool(torch.isfinite(l).any()) else math.nan
            order = torch.sort(torch.where(torch.isnan(l), -math.inf, l), descending=True, stable=True).indices[:k].tolist()
            found += [(base + (float(l[t]) - lse), a, i, t) for i, t in enumerate(order)]
        found = sorted((f for f in found if math.isfinite(f[0])), key=lambda f: (-f[0], f[1], f[2]))[:k]
        rows.append([q * beams + f[1] for f in found] + [-1] * (k - len(found)))
        tokens.append([f[3] for f in found] + [-1] * (k - len(found)))
        best.append([f[0] for f in found] + [-math.inf] * (k - len(found)))
    return rows, tokens, best
