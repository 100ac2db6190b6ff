"""Performance cases of the operators for generation that branches over the paged K/V cache: beams, samples of one prompt, trees of drafted tokens.

  append     focus_kv_append: rows of keys and values into the pages of their sequences.
  tree       focus_tree_attention: attention of every sequence's drafted tokens over its cached tokens and over the drafted ones that its mask shows.
  compact    focus_kv_compact: the tokens of a sequence that stay (the accepted path of a tree, what an eviction leaves) move together, in every layer.
  fork       focus_kv_fork, then focus_kv_reserve: new rows share or copy the pages of the rows they continue, pages that nobody holds any more are free,
             and every row gets room for its next token.
  beam       focus_beam_select: the best continuations of every request's beams.

The pool is [layers, pages, 2, heads, page size, head width]; a page holds K as [heads, tokens, width], then V transposed, [heads, width, tokens].  Token t of a
sequence is token t % size of page table[t / size].

run() computes the operators in plain torch operations where `own` is false and calls the library where it is true.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # One request's eight drafted tokens a layer: latency.
        _append("append_request", 1, 8, 8, 4001, 4001, 8, 128, 64, "bf16"),
        # Prompts, an odd number of rows, written in one go; the head layout of the 8B configuration.
        _append("append_prompt", 3, 5461, 5463, 0, 200, 8, 128, 64, "bf16"),
        # One request, a tree of 24 drafted tokens over a cache of 4001: latency.
        _tree("tree_request", 1, 24, 24, 4001, 4001, False, 32, 8, 128, 64, "bf16", "tree"),
        # A batch of 256 requests with the lengths of the batch-256 configuration, eight drafted tokens each.
        _tree("tree_step", 256, 8, 8, 512, 4096, False, 32, 8, 128, 64, "bf16", "tree"),
        # A ragged batch: no cached token to 32768, no drafted one to 61, small pages, narrow heads.
        _tree("tree_ragged", 9, 0, 61, 0, 32768, True, 16, 4, 64, 16, "bf16", "tree"),
        # Single tokens (no tree) of an fp32 model, 33 sequences.
        _tree("single_f32", 33, 1, 1, 32, 2048, False, 4, 4, 64, 16, "f32", "chain"),
        # The accepted paths of 256 requests' trees of eight.
        dict(name="compact_accept", kind="compact", layers=4, n=256, start_lo=0, start_hi=200, span=8, keep=0.4, heads=8, dim=128, page=64, dtype="bf16"),
        # A third of some 8000 cached tokens of eight sequences stays and moves into pages of its own.
        dict(name="compact_evict", kind="compact", layers=4, n=8, start_lo=0, start_hi=5, span=8001, keep=0.34, heads=8, dim=128, page=64, dtype="bf16"),
        # Four beams of one request.
        dict(name="fork_request", kind="fork", layers=4, n=1, beams=4, prompt_lo=1000, prompt_hi=1000, grown=77, spare=2.0, heads=8, dim=128, page=64, dtype="bf16"),
        # Four beams of 64 requests that share their prompts' pages.
        dict(name="fork_step", kind="fork", layers=4, n=64, beams=4, prompt_lo=512, prompt_hi=4096, grown=150, spare=2.0, heads=8, dim=128, page=64, dtype="bf16"),
        # One request's four beams, the vocabulary of the 8B configuration.
        dict(name="beam_request", kind="beam", n=1, beams=4, vocab=151936, k=8, dtype="f32", pad=0, done=0.0),
        # 64 requests of eight beams, some of them finished, logits in bf16 of odd row length.
        dict(name="beam_step", kind="beam", n=64, beams=8, vocab=151935, k=16, dtype="bf16", pad=2, done=0.1),
    ]


def _append(name, n, rows_lo, rows_hi, len_lo, len_hi, heads, dim, page, dtype):
    return dict(name=name, kind="append", n=n, rows_lo=rows_lo, rows_hi=rows_hi, len_lo=len_lo, len_hi=len_hi, log=False, heads=heads, dim=dim, page=page, dtype=dtype)


def _tree(name, n, rows_lo, rows_hi, len_lo, len_hi, log, q_heads, heads, dim, page, dtype, mask):
    return dict(name=name, kind="tree", n=n, rows_lo=rows_lo, rows_hi=rows_hi, len_lo=len_lo, len_hi=len_hi, log=log, q_heads=q_heads, heads=heads, dim=dim, page=page,
                dtype=dtype, mask=mask)


def _log_int(rng, lo, hi):
    return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["append", "tree", "tree", "tree", "compact", "fork", "beam"])
        heads, dim, page, dtype = rng.choice([1, 2, 4, 8]), rng.choice([64, 128]), rng.choice([16, 32, 64, 64, 128]), rng.choice(["bf16", "bf16", "f32"])
        shape = dict(heads=heads, dim=dim, page=page, dtype=dtype)
        n = _log_int(rng, 1, 256)
        if kind == "append":
            hi = _log_int(rng, 1, 6000)
            c = _append("", n, rng.randint(0, hi), hi, 0, _log_int(rng, 1, 2048), **shape)
        elif kind == "tree":
            hi, far = rng.randint(1, 64), _log_int(rng, 1, 32768)
            c = _tree("", n, rng.randint(0, hi), hi, rng.choice([0, far // 3, far]), far, rng.random() < 0.3, heads * rng.choice([1, 2, 4, 5, 8]), **shape,
                      mask=rng.choice(["tree", "tree", "chain"]))
        elif kind == "compact":
            c = dict(kind=kind, layers=rng.randint(1, 4), n=n, start_lo=0, start_hi=_log_int(rng, 1, 300), span=_log_int(rng, 1, 8192), keep=rng.uniform(0.1, 0.9), **shape)
        elif kind == "fork":
            far = _log_int(rng, 1, 4096)
            c = dict(kind=kind, layers=rng.randint(1, 4), n=_log_int(rng, 1, 64), beams=rng.randint(1, 8), prompt_lo=rng.randint(1, far), prompt_hi=far,
                     grown=rng.randint(0, 300), spare=rng.choice([2.0, 2.0, 0.3]), **shape)
        else:
            beams = rng.randint(1, 12)
            vocab = _log_int(rng, 100, 160000)
            c = dict(kind=kind, n=_log_int(rng, 1, 64), beams=beams, vocab=vocab, k=rng.randint(1, min(32, 2 * beams)), dtype=rng.choice(["f32", "bf16"]),
                     pad=rng.choice([0, 0, 1, 8]), done=rng.choice([0.0, 0.1, 0.5]))
        c.pop("name", None)
        if _cost(c) <= most and _pool_bytes(c) <= 5e9:
            return c


def _spread(n, lo, hi, log):
    """n whole numbers spread evenly from lo to hi (over their logarithm)."""
    if n == 1:
        return [hi]
    if log:
        return [int(round(math.exp(math.log(lo + 1) + (math.log(hi + 1) - math.log(lo + 1)) * i / (n - 1)))) - 1 for i in range(n)]
    return [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _rows(c):
    return sum(_spread(c["n"], c["rows_lo"], c["rows_hi"], False))


def _cached(c):
    return sum(_spread(c["n"], c["len_lo"], c["len_hi"], c["log"]))


def _token_bytes(c):
    """Of a cached token in one layer, keys and values."""
    return 2 * c["heads"] * c["dim"] * (4 if c["dtype"] == "f32" else 2)


def _held(c):
    """Pages that a fork case's rows begin with: those of the prompts, and the beams' own."""
    prompts = _spread(c["n"], c["prompt_lo"], c["prompt_hi"], False)
    own_pages = [(p + c["grown"]) // c["page"] + 1 - p // c["page"] for p in prompts]
    return sum(p // c["page"] for p in prompts) + c["beams"] * sum(own_pages)


def _fork_pages(c):
    """Pages of a fork case's pool; with few spare ones it runs out of them."""
    return _held(c) + int(c["spare"] * c["n"] * c["beams"])


def _pool_bytes(c):
    if c["kind"] == "beam":
        return 0
    if c["kind"] == "fork":
        pages = _fork_pages(c)
    elif c["kind"] == "compact":
        pages = c["n"] * 2 * (-(-(c["start_hi"] + c["span"]) // c["page"]) + 1)
    else:
        pages = c["n"] * (-(-(c["len_hi"] + c["rows_hi"]) // c["page"]) + 1)
    return pages * c["page"] * _token_bytes(c) * c.get("layers", 1)


def _cost(c):
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / (1.2e15 if c["dtype"] == "bf16" else 1e14))


def work(case):
    """Each input read once, each output written once."""
    c = case
    es = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "append":
        return {"bytes": 2 * _rows(c) * _token_bytes(c) + 8 * c["n"], "flops": 0}
    if c["kind"] == "tree":
        rows, cached = _rows(c), _cached(c)
        most = [(a + b) * b for a, b in zip(_spread(c["n"], c["len_lo"], c["len_hi"], c["log"]), _spread(c["n"], c["rows_lo"], c["rows_hi"], False))]
        flops = 4 * c["q_heads"] * c["dim"] * (sum(most) if c["n"] == 1 else rows * cached // c["n"])      # lengths and rows are paired at random
        return {"bytes": (cached + rows) * _token_bytes(c) + 2 * rows * c["q_heads"] * c["dim"] * es + 8 * rows + 4 * cached // c["page"], "flops": flops}
    if c["kind"] == "compact":
        return {"bytes": int(2 * c["n"] * max(1, c["span"] * c["keep"]) * _token_bytes(c) * c["layers"]), "flops": 0}
    if c["kind"] == "fork":
        n_rows = c["n"] * c["beams"]
        distinct = c["beams"] * (1 - (1 - 1 / c["beams"]) ** c["beams"])        # beams that some new row continues, on average
        copied = c["n"] * (c["beams"] - distinct) * c["page"] / 2
        pages = sum(p + c["grown"] for p in _spread(c["n"], c["prompt_lo"], c["prompt_hi"], False)) * c["beams"] // c["page"]
        return {"bytes": int(2 * copied * _token_bytes(c) * c["layers"]) + 8 * pages + 8 * _held(c) + 16 * n_rows, "flops": 0}
    n = c["n"] * c["beams"] * c["vocab"]
    return {"bytes": int(n * es * (1 - c["done"])) + 4 * c["n"] * (c["beams"] + 3 * c["k"]), "flops": 4 * n}


# ---------------------------------------------------------------------------------------------
# inputs

def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, generator=gen, device=gen.device) * std


def _pool(gen, c, layers, pages):
    pool = torch.empty(layers, pages, 2, c["heads"], c["page"], c["dim"], dtype=DTYPES[c["dtype"]], device="cuda")
    step = max(1, (1 << 26) // pool[0, 0].numel())
    for l in range(layers):
        for p in range(0, pages, step):
            pool[l, p:p + step].copy_(_normal(gen, *pool[l, p:p + step].shape))
    return pool


def _shuffled(gen, values):
    """A tensor of whole numbers in an order that the generator picks."""
    v = torch.tensor(values, dtype=torch.int64, device=gen.device)
    return v[torch.randperm(len(values), generator=gen, device=gen.device)]


def _starts(counts):
    """[0, c0, c0 + c1, ...] as int32."""
    return torch.nn.functional.pad(torch.cumsum(counts, 0), (1, 0)).to(torch.int32)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=dict(c))
    if c["kind"] == "beam":
        rows = c["n"] * c["beams"]
        wide = torch.empty(rows, c["vocab"] + c["pad"], dtype=DTYPES[c["dtype"]], device="cuda")
        for r in range(0, rows, 64):
            wide[r:r + 64].copy_(_normal(gen, *wide[r:r + 64].shape, std=2.5))
        s["logits"] = wide[:, :c["vocab"]]
        s["scores"] = -_normal(gen, c["n"], c["beams"]).abs() * 2 - 5
        s["done"] = torch.rand(c["n"], c["beams"], generator=gen, device="cuda") < c["done"] if c["done"] else None
        return s
    if c["kind"] in ("append", "tree"):
        n, size = c["n"], c["page"]
        lens = _shuffled(gen, _spread(n, c["len_lo"], c["len_hi"], c["log"]))
        counts = _shuffled(gen, _spread(n, c["rows_lo"], c["rows_hi"], False))
        rows, stride = int(counts.sum()), -(-(c["len_hi"] + c["rows_hi"]) // size) + 1
        s["pool"] = _pool(gen, c, 1, n * stride)
        s["table"] = torch.randperm(n * stride, generator=gen, device="cuda").to(torch.int32).view(n, stride)
        s["lens"], s["cu"] = lens.to(torch.int32), _starts(counts)
        if c["kind"] == "append":
            # keys and values are columns of a fused projection's rows
            s["kv"] = _normal(gen, rows, 2 * c["heads"] * c["dim"]).to(DTYPES[c["dtype"]])
            return s
        s["q"] = _normal(gen, rows, c["q_heads"] * c["dim"]).to(DTYPES[c["dtype"]])
        s["max_rows"], s["max_len"], s["seen"] = c["rows_hi"], c["len_hi"] + c["rows_hi"], None
        if c["mask"] == "tree":
            # every drafted token's parent is one of the few before it, or the cache; it sees its ancestors and itself
            of = torch.repeat_interleave(torch.arange(n, device="cuda"), counts, output_size=rows)
            i = torch.arange(rows, device="cuda") - s["cu"][of].long()
            back = torch.randint(1, 7, (rows,), generator=gen, device="cuda")
            parent = i - back
            seen = torch.bitwise_left_shift(torch.ones_like(i), i)
            for j in range(c["rows_hi"]):       # row j of every sequence takes its parent's ancestors
                now = (i == j) & (parent >= 0)
                up = seen[(torch.arange(rows, device="cuda") - back).clamp(min=0)]
                seen = torch.where(now, seen | up, seen)
            s["seen"] = seen
        return s
    if c["kind"] == "compact":
        n, size = c["n"], c["page"]
        start = _shuffled(gen, _spread(n, c["start_lo"], c["start_hi"], False))
        stride = -(-(c["start_hi"] + c["span"]) // size) + 1
        pages = torch.randperm(2 * n * stride, generator=gen, device="cuda").to(torch.int32).view(2, n, stride)
        s["pool"], s["table"], s["to"], s["start"] = _pool(gen, c, c["layers"], 2 * n * stride), pages[0].contiguous(), pages[1].contiguous(), start.to(torch.int32)
        stays = torch.rand(n, c["span"], generator=gen, device="cuda") < c["keep"]
        stays[:, 0] = True
        s["keep"], s["cu"] = torch.nonzero(stays)[:, 1].to(torch.int32), _starts(stays.sum(1))
        return s
    # a fork: the beams of a request hold its prompt's pages together, and what they have grown by each for itself
    n, beams, size = c["n"], c["beams"], c["page"]
    prompts = _spread(n, c["prompt_lo"], c["prompt_hi"], False)
    pages = _fork_pages(c)
    order = torch.randperm(pages, generator=gen, device="cuda").tolist()
    stride = (c["prompt_hi"] + c["grown"]) // size + 2
    table, refs, lens, at = [], [0] * pages, [], 0
    for p in prompts:
        shared, own_pages = order[at:at + p // size], (p + c["grown"]) // size + 1 - p // size
        at += len(shared)
        for _ in range(beams):
            row = shared + order[at:at + own_pages]
            at += own_pages
            lens.append(p + c["grown"])
            for page in row:
                refs[page] += 1
            table.append(row + [-1] * (stride - len(row)))
    s["pool"] = _pool(gen, c, c["layers"], pages)
    s["table"], s["refs"], s["lens"] = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (table, refs, lens))
    picks = torch.randint(0, beams, (n, beams), generator=gen, device="cuda")
    s["parents"] = (picks + beams * torch.arange(n, device="cuda").unsqueeze(1)).view(-1).to(torch.int32)
    return s


# ---------------------------------------------------------------------------------------------
# the plain forms

def _places(c, table, seq, token):
    """(page, place inside it) of tokens of sequences."""
    return table[seq, token // c["page"]].long(), token % c["page"]


def _v_of(pool):
    """The values, transposed as they are kept: [layers, pages, heads, width, tokens]."""
    return pool[:, :, 1].view(*pool.shape[:2], pool.shape[3], pool.shape[5], pool.shape[4])


def _plain_append(s):
    c, pool = s["case"], s["pool"]
    r = torch.arange(len(s["kv"]), device=pool.device)
    seq = torch.searchsorted(s["cu"].long(), r, right=True) - 1
    page, place = _places(c, s["table"], seq, (s["lens"][seq] + r - s["cu"][seq]).long())
    k, v = s["kv"].view(-1, 2, c["heads"], c["dim"]).unbind(1)
    pool[0, page, 0, :, place] = k
    _v_of(pool)[0, page, :, :, place] = v
    return pool


def _plain_tree(s):
    c, lens = s["case"], s["lens"].long()
    n, H, D, g, R = c["n"], c["heads"], c["dim"], c["q_heads"] // c["heads"], s["max_rows"]
    rows = len(s["q"])
    r = torch.arange(rows, device=lens.device)
    seq = torch.searchsorted(s["cu"].long(), r, right=True) - 1
    i = r - s["cu"][seq]
    pages = s["table"][:, :-(-s["max_len"] // c["page"])].long()
    k = s["pool"][0, pages, 0].float().transpose(1, 2).reshape(n, H, -1, D)
    v = _v_of(s["pool"])[0, pages].float().permute(0, 2, 1, 4, 3).reshape(n, H, -1, D)
    q = torch.zeros(n, R, H, g, D, device=lens.device)
    q[seq, i] = s["q"].float().view(rows, H, g, D)
    score = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(n, H, R * g, D) / math.sqrt(D), k.transpose(2, 3)).view(n, H, R, g, -1)
    t = torch.arange(score.shape[-1], device=lens.device)
    j = t.unsqueeze(0) - lens.unsqueeze(1)                                           # [n, tokens]: which drafted token, below 0: a cached one
    if s["seen"] is None:
        sees = j.unsqueeze(1) <= torch.arange(R, device=lens.device).view(1, R, 1)
    else:
        seen = torch.zeros(n, R, dtype=torch.int64, device=lens.device)
        seen[seq, i] = s["seen"]
        bit = (seen.unsqueeze(2) >> j.clamp(0, 63).unsqueeze(1)) & 1
        sees = (j < 0).unsqueeze(1) | ((bit == 1) & (j < 64).unsqueeze(1))
    score = score.masked_fill(~sees.view(n, 1, R, 1, -1), -math.inf)
    top = score.amax(dim=-1, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(dim=-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    out = torch.matmul(p.view(n, H, R * g, -1), v).view(n, H, R, g, D).permute(0, 2, 1, 3, 4)
    return out[seq, i].reshape(rows, -1).to(s["q"].dtype)


def _plain_compact(s):
    c, pool = s["case"], s["pool"]
    e = torch.arange(len(s["keep"]), device=pool.device)
    seq = torch.searchsorted(s["cu"].long(), e, right=True) - 1
    start = s["start"][seq].long()
    page, place = _places(c, s["table"], seq, start + s["keep"])
    to_page, to_place = _places(c, s["to"], seq, start + e - s["cu"][seq])
    v = _v_of(pool)
    k_rows, v_rows = pool[:, page, 0, :, place], v[:, page, :, :, place]
    pool[:, to_page, 0, :, to_place] = k_rows
    v[:, to_page, :, :, to_place] = v_rows
    return pool


def _free_pages(refs):
    """The free pages, lowest first, then numbers that are no page."""
    page = torch.arange(len(refs), device=refs.device)
    return torch.sort(torch.where(refs == 0, page, len(refs))).values


def _held_pages(table):
    return (torch.cumsum(table < 0, 1) == 0).sum(1)


def _plain_fork(s, refs):
    c, pool, table, P = s["case"], s["pool"], s["table"].long(), s["case"]["page"]
    lens, parents = s["lens"].long(), s["parents"].long()
    at = torch.arange(table.shape[1], device=table.device)
    held = _held_pages(table)
    whole = torch.minimum(lens // P, held)
    begun = (lens % P > 0) & (whole < held)
    children = torch.zeros_like(lens).index_add_(0, parents, torch.ones_like(parents))
    first = ~torch.tril(parents.unsqueeze(1) == parents, -1).any(1)
    change = torch.where(at < whole.unsqueeze(1), children.unsqueeze(1) - 1, torch.where(children.unsqueeze(1) > 0, 0, -1))
    holds = at < held.unsqueeze(1)
    refs.index_add_(0, torch.where(holds, table, 0).view(-1), torch.where(holds, change, 0).view(-1).to(torch.int32))
    keeps = (at < whole[parents].unsqueeze(1)) | (first.unsqueeze(1) & holds[parents])
    new_table = torch.where(keeps, table[parents], -1)
    wants = ~first & begun[parents]
    page = torch.nn.functional.pad(_free_pages(refs), (0, 1), value=len(refs))[(torch.cumsum(wants, 0) - 1).clamp(0, len(refs))]
    gets = wants & (page < len(refs))
    new_lens = torch.where(wants & ~gets, whole[parents] * P, lens[parents])
    i = torch.nonzero(gets).view(-1)
    new_table[i, whole[parents[i]]] = page[i]
    refs[page[i]] = 1
    source, there = table[parents[i], whole[parents[i]]], torch.arange(P, device=table.device) < (lens[parents[i]] % P).unsqueeze(1)
    v = _v_of(pool)
    pool[:, page[i], 0] = torch.where(there.view(-1, 1, P, 1), pool[:, source, 0], pool[:, page[i], 0])
    v[:, page[i]] = torch.where(there.view(-1, 1, 1, P), v[:, source], v[:, page[i]])
    return new_lens.to(torch.int32), new_table.to(torch.int32), (wants & ~gets).to(torch.int32)


def _plain_reserve(c, lens, room, table, refs):
    held = _held_pages(table)
    need = (lens + room + c["page"] - 1) // c["page"]
    at = torch.arange(table.shape[1], device=table.device)
    wants = (at >= held.unsqueeze(1)) & (at < need.unsqueeze(1))
    page = torch.nn.functional.pad(_free_pages(refs), (0, 1), value=len(refs))[(torch.cumsum(wants.view(-1), 0) - 1).clamp(0, len(refs))].view(wants.shape)
    gets = wants & (page < len(refs))
    table.copy_(torch.where(gets, page, table))
    refs[page[gets]] = 1
    return ((need - held).clamp(min=0) - gets.sum(1)).to(torch.int32)


def _plain_beam(s):
    c = s["case"]
    n, beams, k = c["n"], c["beams"], c["k"]
    l = s["logits"].float()
    top, token = torch.sort(l, dim=1, descending=True, stable=True)
    some = min(k, c["vocab"])
    top, token = top[:, :some].double(), token[:, :some]
    most = top[:, :1]
    lse = most + torch.log(torch.exp(l.double() - most).sum(1, keepdim=True))
    score = s["scores"].double().view(-1, 1) + (top - lse)
    if s["done"] is not None:
        done = s["done"].view(-1, 1)
        alone = torch.arange(some, device=l.device) == 0
        score = torch.where(done, torch.where(alone, s["scores"].double().view(-1, 1), -math.inf), score)
        token = torch.where(done, 0, token)
    score = torch.nn.functional.pad(score.view(n, beams * some), (0, k), value=-math.inf)
    best, at = torch.sort(torch.where(torch.isfinite(score), score, -math.inf), dim=1, descending=True, stable=True)
    best, at = best[:, :k], at[:, :k].clamp(max=beams * some - 1)
    row = at // some + beams * torch.arange(n, device=l.device).unsqueeze(1)
    picked = best > -math.inf
    return torch.where(picked, row, -1).to(torch.int32), torch.where(picked, torch.gather(token.reshape(n, -1), 1, at), -1).to(torch.int32), best.float()


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2601_23278_amd as pk
    if c["kind"] == "append":
        if not own:
            return _plain_append(s)
        width = c["heads"] * c["dim"]
        pk.focus_kv_append(s["pool"], 0, s["kv"][:, :width], s["kv"][:, width:], s["cu"], s["lens"], s["table"])
        return s["pool"]
    if c["kind"] == "tree":
        if not own:
            return _plain_tree(s)
        return pk.focus_tree_attention(s["pool"], 0, s["q"], s["cu"], s["lens"], s["table"], seen=s["seen"], max_rows=s["max_rows"], max_len=s["max_len"])
    if c["kind"] == "compact":
        if not own:
            return _plain_compact(s)
        pk.focus_kv_compact(s["pool"], s["start"], s["cu"], s["keep"], s["table"], s["to"])
        return s["pool"]
    if c["kind"] == "fork":
        refs = s["refs"].clone()
        if not own:
            lens, table, lacking = _plain_fork(s, refs)
            return lens, table, lacking, _plain_reserve(c, lens, 1, table, refs), refs, s["pool"]
        lens, table, lacking = pk.focus_kv_fork(s["pool"], s["parents"], s["lens"], s["table"], refs)
        return lens, table, lacking, pk.focus_kv_reserve(lens, 1, table, refs, c["page"]), refs, s["pool"]
    if not own:
        return _plain_beam(s)
    return pk.focus_beam_select(s["logits"], s["scores"], c["k"], done=s["done"], end_token=0)


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits, apart from the plain forms

def exact(case, seed):
    c = case
    if c["kind"] in ("append", "compact", "fork"):       # nothing is computed: bits move
        return None
    s = prepare(case, seed)
    if c["kind"] == "tree":
        H, D, g, P = c["heads"], c["dim"], c["q_heads"] // c["heads"], c["page"]
        out, cu, lens = torch.zeros(len(s["q"]), c["q_heads"], D, dtype=torch.float64, device="cuda"), s["cu"].tolist(), s["lens"].tolist()
        for b in range(c["n"]):
            count = cu[b + 1] - cu[b]
            total = lens[b] + count
            if count == 0:
                continue
            pages = s["table"][b, :-(-total // P)].tolist()
            both = s["pool"][0, pages].double()
            k = torch.cat(list(both[:, 0]), dim=1)[:, :total]                                             # [heads, tokens, width]
            vt = torch.cat([page.reshape(H, D, P) for page in both[:, 1]], dim=2)[:, :, :total]            # [heads, width, tokens]
            sees = torch.ones(count, total, dtype=torch.bool, device="cuda")
            for a in range(count):
                word = int(s["seen"][cu[b] + a]) if s["seen"] is not None else (1 << (a + 1)) - 1
                sees[a, lens[b]:] = torch.tensor([(word >> x) & 1 == 1 for x in range(count)], device="cuda")
            for h in range(c["q_heads"]):
                w = (s["q"][cu[b]:cu[b + 1], h * D:(h + 1) * D].double() @ k[h // g].t().contiguous()) * D ** -0.5
                w = torch.softmax(torch.where(sees, w, -math.inf), dim=1)
                out[cu[b]:cu[b + 1], h] = w @ vt[h // g].t().contiguous()
        return out.view(len(s["q"]), -1)
    n, beams, V, k = c["n"], c["beams"], c["vocab"], c["k"]
    rows, tokens, scores = ([[] for _ in range(n)] for _ in range(3))
    for b in range(n):
        found = []
        for a in range(beams):
            base = float(s["scores"][b, a])
            if s["done"] is not None and bool(s["done"][b, a]):
                found.append((-base, a, 0, 0))
                continue
            l = s["logits"][b * beams + a].double()
            total = torch.logsumexp(l, 0).item()
            edge = torch.topk(l, min(k, V)).values[-1]
            near = torch.nonzero(l >= edge).view(-1).tolist()
            best = sorted(((-l[t].item(), t) for t in near))[:k]
            found += [(-(base + (-x - total)), a, i, t) for i, (x, t) in enumerate(best)]
        found = sorted(found)[:k]
        for x, a, _, t in found:
            rows[b].append(b * beams + a)
            tokens[b].append(t)
            scores[b].append(-x)
        for v, none in ((rows, -1), (tokens, -1), (scores, -math.inf)):
            v[b] += [none] * (k - len(found))
    return (torch.tensor(rows, dtype=torch.int32, device="cuda"), torch.tensor(tokens, dtype=torch.int32, device="cuda"),
            torch.tensor(scores, dtype=torch.float64, device="cuda"))
