"""Branching generation on the GPU: forms of the kernels that only larger calls or mixed inputs reach, each named by a check on the host that this call takes it."""
import ctypes as C
import math

import pytest
import torch

import branch_reference as ref
from test_gpu_branch import DEV, i32, make_pool, starts, tree_masks

pytestmark = pytest.mark.gpu


def _pk():
    import paper_2601_23278_amd as pk
    return pk


def ragged_table(gen, pages, spare=3):
    """A table whose rows hold as many pages as the list says, in random order, and the pool's pages."""
    stride, total = max(max(pages), 1), sum(pages) + spare
    order = torch.randperm(total, generator=gen).tolist()
    return i32([[order.pop() for _ in range(n)] + [-1] * (stride - n) for n in pages]), total


def ragged_tree(gen, dtype, Hq, H, P, D, lens, counts):
    """Sequences that hold the pages they need, in a pool that is NaN wherever no sequence has a token."""
    table, n_pages = ragged_table(gen, [-(-(a + b) // P) for a, b in zip(lens, counts)])
    pool = make_pool(gen, 1, n_pages, H, P, D, dtype, math.nan)
    everything = starts([a + b for a, b in zip(lens, counts)])
    x = torch.randn(int(everything[-1]), 2 * H * D, generator=gen).to(dtype)
    for b in range(len(lens)):
        for t in range(lens[b] + counts[b]):
            r = int(everything[b]) + t
            ref.put(pool, 0, int(table[b, t // P]), t % P, x[r, :H * D].view(H, D), x[r, H * D:].view(H, D))
    q = torch.randn(sum(counts), Hq * D, generator=gen).to(dtype)
    return pool, q, starts(counts), i32(lens), table


def bytes_of(pool, n, rows, max_rows, max_len, stride, heads):
    """(bytes of the workspace, bytes of the starts of the sequences' work alone)."""
    pk = _pk()
    kv, n_bytes = pk.binding._kv_of(pool), C.c_size_t()
    assert pk.binding._lib.focus_tree_attention_bytes(C.byref(kv), n, rows, max_rows, max_len, stride, heads, C.byref(n_bytes)) == 0
    return n_bytes.value, ((n + 1) * 8 + 255) // 256 * 256


def held_against(got, want, size, spread, count, D):
    """Every infinity and NaN where the 64-bit form has it, and finite values within its bound.  A score is a sum of D products (off by D 2^-24 of the sum of their sizes), its
    distance from the maximum is rounded once more, and the exponential is off by 2^-22 and by what 2^-23 of its argument (at most twice the spread) makes; weights are off by
    twice that, as their sum is too.  Sums over n tokens add n 2^-24.  bf16: weights are rounded (2^-8), and so is the result."""
    weight = 2 * ((2 * D + 8) * 2.0 ** -24 * spread + 2.0 ** -22 + 2 * 2.0 ** -23 * spread) + (count.unsqueeze(1) + 16) * 2.0 ** -24
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    bound = (weight + (half if got.dtype == torch.bfloat16 else 0.0)) * 1.01 * size + half * want.abs() + 1e-30
    got = got.double()
    for kind in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(kind(got), kind(want)), (kind, torch.nonzero(kind(got) != kind(want))[:6].tolist())
    fine = torch.isfinite(want)
    assert bool(((got - want).abs()[fine] <= bound[fine]).all()), float(((got - want).abs() - bound)[fine].max())


# -- attention of more sequences than a workgroup sums up for itself, their units cut ------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,hint", [(257, 0), (300, 1), (700, 1)])
def test_tree_attention_of_many_sequences_whose_units_are_cut(dtype, n, hint):
    """A few long caches among many short ones, rows missing at the ends and in runs: with the whole workspace, one byte less (the starts alone fit), the starts alone, and none."""
    pk, gen = _pk(), torch.Generator().manual_seed(n)
    Hq, H, P, D = 2, 1, 16, 64
    lens = torch.randint(0, 60, (n,), generator=gen).tolist()
    counts = torch.randint(0, 4, (n,), generator=gen).tolist()
    counts[0] = counts[-1] = 0
    counts[n // 2:n // 2 + 30] = [0] * 30
    for b, far in ((1, 1500), (n // 2 - 1, 1111), (n // 2 + 30, 1700), (n - 2, 1300)):
        lens[b], counts[b] = far, 3
    pool, q, cu, lens, table = ragged_tree(gen, dtype, Hq, H, P, D, lens, counts)
    seen = tree_masks(gen, counts, 1, "tree")
    want = ref.attention(pool, 0, q, cu, lens, table, seen, D ** -0.5)
    max_rows, max_len = (3, 1703) if hint else (0, 0)
    full, first = bytes_of(pool, n, q.shape[0], max_rows, max_len, table.shape[1], Hq)
    assert full > first                                    # else the units are whole and this tests something else
    args = [pool.to(DEV), 0, q.to(DEV), cu.to(DEV), lens.to(DEV), table.to(DEV)]
    for room in (full, full - 1, first, 0):
        ws = torch.full((full,), 255, dtype=torch.uint8, device=DEV)[:room]
        got = [pk.focus_tree_attention(*args, seen=seen.to(DEV), max_rows=max_rows, max_len=max_len, workspace=ws).cpu() for _ in range(2)]
        assert torch.equal(got[0], got[1])
        held_against(got[0], *want, D)


# -- values that are no numbers, each kind where the 64-bit form has it --------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("P,D,far", [(64, 128, 40), (16, 64, 40), (64, 64, 900), (16, 128, 900)])
@pytest.mark.parametrize("room", [None, 0])
def test_tree_attention_tells_infinities_and_nan_apart(dtype, P, D, far, room):
    """V alone holds them: +inf, -inf and NaN in columns of their own, +inf and -inf together in one, in drafted tokens that some rows see and in a cached one; with long caches
    and a workspace the units are cut."""
    pk, gen = _pk(), torch.Generator().manual_seed(P + D)
    counts, lens, Hq, H = [20, 3, 9], [far, 0, far + 33], 4, 2
    pool, q, cu, lens, table = ragged_tree(gen, dtype, Hq, H, P, D, lens, counts)
    inf, nan = math.inf, math.nan
    bad = [(0, far + 2, {3: inf}), (0, far + 7, {35: -inf}), (0, far + 11, {6: nan, 63: -inf}), (0, far + 4, {20: inf}), (0, far + 13, {20: -inf}), (1, 0, {0: -inf}), (1, 2, {0: inf, 33: nan}),
           (2, 5, {50: -inf, 51: inf, 52: nan}), (2, far + 33 + 8, {50: inf, 7: -inf})]
    for b, t, columns in bad:
        page, place = ref.place_of(pool, table[b], t)
        for d, x in columns.items():
            pool[0, page, 1].view(H, D, P)[:, d, place] = x
    kw = {} if room is None else dict(workspace=torch.empty(0, dtype=torch.uint8, device=DEV))
    args = [pool.to(DEV), 0, q.to(DEV), cu.to(DEV), lens.to(DEV), table.to(DEV)]
    for kind in ("tree", "all", "none", None):
        seen = None if kind is None else tree_masks(gen, counts, 1, kind)
        want = ref.attention(pool, 0, q, cu, lens, table, seen, D ** -0.5)
        got = pk.focus_tree_attention(*args, seen=None if seen is None else seen.to(DEV), max_rows=20, max_len=far + 42, **kw).cpu()
        held_against(got, *want, D)
        if kind in ("all", None):
            assert all(bool(f(want[0]).any()) for f in (torch.isnan, torch.isposinf, torch.isneginf))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("far", [5, 900])
def test_tree_attention_of_scores_of_minus_infinity(dtype, far):
    """Keys of -inf under queries above zero: such tokens add nothing beside others, and a row that sees no others is zero, in drafted and in cached tokens."""
    pk, gen = _pk(), torch.Generator().manual_seed(far)
    counts, lens, Hq, H, P, D = [3, 2], [far, far], 4, 2, 16, 64
    pool, q, cu, lens, table = ragged_tree(gen, dtype, Hq, H, P, D, lens, counts)
    q = q.abs() + 0.1
    lost = [(0, t) for t in range(1, far + 1)] + [(1, t) for t in range(far + 1)]      # of the second sequence all but the last drafted one
    for b, t in lost:
        page, place = ref.place_of(pool, table[b], t)
        pool[0, page, 0, :, place] = -math.inf
    args = [q.to(DEV), cu.to(DEV), lens.to(DEV), table.to(DEV)]
    got = pk.focus_tree_attention(pool.to(DEV), 0, *args).cpu()
    assert bool((got[3] == 0.0).all())
    rows = [0, 1, 2, 4]
    want = ref.attention(pool, 0, q, cu, lens, table, None, D ** -0.5)
    for b, t in lost:                                      # the bound is that of the scores that count
        page, place = ref.place_of(pool, table[b], t)
        pool[0, page, 0, :, place] = 0.0
    spread = ref.attention(pool, 0, q, cu, lens, table, None, D ** -0.5)[2]
    held_against(got[rows], want[0][rows], want[1][rows], spread[rows], want[3][rows], D)


# -- compaction ----------------------------------------------------------------------------------------
def forms(keep, start):
    """What the batches of a sequence's moves are: 'few' (one batch), or for each 64 places 'whole' or 'single' (its tokens lie further apart than what is held of a row)."""
    skip = start & 63
    if skip + len(keep) <= 32:
        return {"few"}
    found = set()
    for j0 in range(0, skip + len(keep), 64):
        mine = [keep[j - skip] + (start & 7) for j in range(max(j0, skip), min(j0 + 64, skip + len(keep)))]
        if mine:
            found.add("single" if mine[-1] >= mine[0] // 8 * 8 + 256 else "whole")
    return found


def moved(pool, start, cu, keep, table, to_table):
    """The plain form with all tokens of a layer at once."""
    H, P, D = pool.shape[3:]
    src, dst = [], []
    for b in range(len(start)):
        for i in range(int(cu[b + 1]) - int(cu[b])):
            x, y = ref.place_of(pool, table[b], int(start[b]) + int(keep[int(cu[b]) + i])), ref.place_of(pool, to_table[b], int(start[b]) + i)
            if x is not None and y is not None:
                src.append(x), dst.append(y)
    (p, a), (r, c) = (tuple(torch.tensor(v).view(-1, 2).unbind(1)) for v in (src, dst))
    want, v = pool.clone(), pool.clone()[:, :, 1].reshape(*pool.shape[:2], H, D, P)
    want[:, r, 0, :, c] = pool[:, p, 0, :, a]
    v[:, r, :, :, c] = pool[:, :, 1].reshape(*pool.shape[:2], H, D, P)[:, p, :, :, a]
    want[:, :, 1] = v.reshape(*pool.shape[:2], H, P, D)
    return want


def check_compact(gen, dtype, layers, H, P, D, spans, keeps, start, in_place, holes=0):
    pk = _pk()
    pages = [-(-(a + b) // P) for a, b in zip(spans, start)]
    both, n_pages = ragged_table(gen, pages + pages)
    table, to = both[:len(spans)].clone(), both[len(spans):].clone()
    for t in (table, to):
        for _ in range(holes):                             # an entry that is no page, one that is none of the pool's
            t.view(-1)[torch.randint(0, t.numel(), (2,), generator=gen)] = i32([-1, n_pages])
    pool = make_pool(gen, layers, n_pages, H, P, D, dtype)
    cu, flat, start = starts([len(k) for k in keeps]), i32([x for k in keeps for x in k]), i32(start)
    want = moved(pool, start, cu, flat, table, table if in_place else to)
    got = pool.to(DEV)
    pk.focus_kv_compact(got, start.to(DEV), cu.to(DEV), flat.to(DEV), table.to(DEV), None if in_place else to.to(DEV))
    as_bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
    assert torch.equal(got.cpu().view(as_bits), want.view(as_bits))


def shares(gen, span, share):
    """Tokens that stay, of a span whose parts stay with one share after the other."""
    n = len(share)
    return [x for x in range(span) if float(torch.rand(1, generator=gen)) < share[x * n // span]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("in_place", [True, False])
def test_compact_of_many_heads(dtype, D, in_place):
    """More than 1024 (sequence, head, layer) triples: a workgroup takes all columns of its head.  One of few tokens, dense and sparse ones, and none."""
    gen = torch.Generator().manual_seed(D)
    layers, H, P = 4, 8, 16
    spans = [0, 1, 2, 3, 5, 9, 17, 33, 40, 64, 65, 130, 300, 700] + [8] * 24
    start = [int(torch.randint(0, 70, (1,), generator=gen)) for _ in spans]
    keeps = [shares(gen, s, [0.9, 0.3, 0.1] if s > 200 else [0.6]) for s in spans]
    keeps[1] = [0]
    assert len(spans) * H * layers > 1024
    found = set().union(*(forms(k, s) for k, s in zip(keeps, start)))
    assert found == {"few", "whole", "single"}
    check_compact(gen, dtype, layers, H, P, D, spans, keeps, start, in_place)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("P,D,start", [(8, 64, [3, 0, 61]), (24, 128, [7, 100, 64]), (64, 64, [0, 13, 63]), (64, 128, [1, 8, 250])])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("many", [False, True])
def test_compact_of_dense_and_sparse_stretches(dtype, P, D, start, in_place, many):
    """Batches whose rows of V^T are held whole and batches of single columns in turn; `many`: beside enough others that a workgroup takes all columns."""
    gen = torch.Generator().manual_seed(P + D)
    share = [[0.95, 0.05, 0.9, 0.12, 0.2, 0.05, 1.0, 0.05], [0.2, 0.15], [0.05, 0.99, 0.04]]
    spans = [3000, 2501, 1999]
    keeps = [shares(gen, a, b) for a, b in zip(spans, share)]
    assert all("single" in forms(k, s) for k, s in zip(keeps, start)) and all("whole" in forms(keeps[b], start[b]) for b in (0, 2))
    if many:
        spans, keeps, start = spans + [4] * 1100, keeps + [[0, 2]] * 1100, start + [5] * 1100
    assert (len(spans) > 1024) == many
    check_compact(gen, dtype, 1, 1, P, D, spans, keeps, start, in_place)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_compact_of_long_stretches_leaves_out_tokens_without_a_page(dtype):
    gen = torch.Generator().manual_seed(5)
    spans, start = [2000, 900], [9, 64]
    keeps = [shares(gen, 2000, [0.9, 0.1]), shares(gen, 900, [0.5])]
    for in_place in (True, False):
        check_compact(gen, dtype, 2, 2, 16, 64, spans, keeps, start, in_place, holes=12)


# -- reservation -----------------------------------------------------------------------------------------
def test_reserve_writes_what_lacks_over_the_lengths():
    pk = _pk()
    lens, refs = i32([20, 0, 50]).to(DEV), i32([0, 1, 0, 0, 0]).to(DEV)
    table = i32([[1, -1, -1], [-1, -1, -1], [-1, -1, -1]]).to(DEV)
    got = pk.focus_kv_reserve(lens, 1, table, refs, 16, lacking=lens)
    assert got is lens and lens.tolist() == [0, 0, 2] and refs.tolist() == [1] * 5       # 50 + 1 tokens want four pages: two were left, and the row has three entries
    assert table.tolist() == [[1, 0, -1], [2, -1, -1], [3, 4, -1]]


# -- beams that tie ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab,pad", [(70, 1), (4097, 3), (20011, 5)])
def test_beams_of_the_same_logits_tie(dtype, vocab, pad):
    """The lower beam comes first wherever its row begins, and the same logits are taken from every beam before the next ones."""
    pk, gen = _pk(), torch.Generator().manual_seed(vocab)
    n, beams, k = 50, 3, 6
    wide = torch.zeros(n * beams, vocab + pad, dtype=dtype, device=DEV)
    for scale in (0.5, 3.0):
        l = (torch.randn(n, vocab, generator=gen) * scale).to(dtype)
        l[:, 17], l[:, 40] = 19.0, 18.0                    # the best two by far
        wide[:, :vocab] = l.repeat_interleave(beams, 0).to(DEV)
        scores = (-torch.rand(n, 1, generator=gen) * 7).repeat(1, beams).to(DEV)
        rows, tokens, new = pk.focus_beam_select(wide[:, :vocab], scores, k)
        assert torch.equal(rows.cpu(), i32([0, 1, 2, 0, 1, 2]) + beams * torch.arange(n, dtype=torch.int32).view(n, 1))
        assert tokens.tolist() == [[17] * 3 + [40] * 3] * n
        assert torch.equal(new[:, :1].expand(n, 3), new[:, :3]) and torch.equal(new[:, 3:4].expand(n, 3), new[:, 3:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [300, 4096, 9001])
def test_beams_of_the_same_logits_at_other_tokens(dtype, vocab):
    """Their log-sums are 4e-12 apart at most, so the multiples of 2^-34 = 5.8e-11 that they round to are the same or neighbours; the chance that they are neighbours is 7 % at most."""
    pk, gen = _pk(), torch.Generator().manual_seed(vocab)
    n = 256
    l = torch.randn(n, vocab, generator=gen).to(dtype)
    l[:, 5] = 12.0
    order = torch.stack([torch.randperm(vocab, generator=gen) for _ in range(n)])
    logits = torch.stack([l, torch.gather(l, 1, order)], 1).view(2 * n, vocab)
    scores = torch.full((n, 2), -1.0)
    rows, tokens, new = (t.cpu() for t in pk.focus_beam_select(logits.to(DEV), scores.to(DEV), 2))
    place = torch.stack([torch.full((n,), 5), (order == 5).int().argmax(1)], 1)
    first = rows[:, 0] - 2 * torch.arange(n)
    assert torch.equal(rows.sort(1).values, torch.arange(2 * n, dtype=torch.int32).view(n, 2))
    assert torch.equal(tokens.long(), torch.where(first.view(n, 1) == 0, place, place.flip(1)))
    want = -1.0 + (12.0 - torch.logsumexp(l.double(), 1, keepdim=True))
    assert bool(((new.double() - want).abs() <= want.abs() * 2.0 ** -24 * 1.001 + 2.0 ** -34).all())
    assert int((first == 1).sum()) <= 40                    # of 256: 18 at that chance, and five times their spread


def test_captured_selection_of_many_picks():
    """As many beams and picks as there may be: a launch with more shared memory than it has by itself, captured, and replayed over other logits."""
    pk, gen = _pk(), torch.Generator().manual_seed(71)
    n, beams, vocab, k = 2, 64, 5000, 64
    logits, scores = torch.zeros(n * beams, vocab, device=DEV), torch.zeros(n, beams, device=DEV)
    out = [torch.zeros(n, k, dtype=t, device=DEV) for t in (torch.int32, torch.int32, torch.float32)]
    sets = [(torch.randn(n * beams, vocab, generator=gen).to(DEV), (-torch.rand(n, beams, generator=gen)).to(DEV)) for _ in range(4)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        pk.focus_beam_select(logits, scores, k, rows=out[0], tokens=out[1], new_scores=out[2], stream=side)
    for _ in range(3):
        for l, s in sets:
            logits.copy_(l)
            scores.copy_(s)
            torch.cuda.synchronize()
            graph.replay()
            want = pk.focus_beam_select(l, s, k)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want))
