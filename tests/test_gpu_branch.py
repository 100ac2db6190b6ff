"""Tree attention, page bookkeeping and beam selection on the GPU, through the public entry points, against plain 64-bit forms (branch_reference.py)."""
import math

import pytest
import torch

import branch_reference as ref

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
NAN = math.nan


def _pk():
    import paper_2601_23278_amd as pk
    return pk


def i32(v):
    return torch.tensor(v, dtype=torch.int32)


def starts(counts):
    return i32([sum(counts[:i]) for i in range(len(counts) + 1)])


def bits(words):
    """int64 whose bits are those of unsigned numbers."""
    return torch.tensor([[w - (1 << 64) if w >> 63 else w for w in row] for row in words], dtype=torch.int64)


def make_pool(gen, layers, pages, H, P, D, dtype, fill=None):
    if fill is not None:
        return torch.full((layers, pages, 2, H, P, D), fill, dtype=dtype)
    return torch.randn(layers, pages, 2, H, P, D, generator=gen).to(dtype)


def tables(gen, n, stride, spare=0):
    return torch.randperm(n * stride + spare, generator=gen)[:n * stride].to(torch.int32).view(n, stride)


def tree_masks(gen, counts, words, kind):
    """Rows of `words` unsigned 64-bit numbers: ancestors in a random tree, everything, nothing, or bits of all kinds (beyond the sequence's rows too)."""
    rows = []
    for n in counts:
        sets = []
        for i in range(n):
            if kind == "tree":
                parent = int(torch.randint(-1, i, (1,), generator=gen)) if i else -1
                s = (sets[parent] if parent >= 0 else 0) | 1 << i
            elif kind == "noise":
                s = sum(int(torch.randint(0, 1 << 32, (1,), generator=gen)) << (32 * x) for x in range(2 * words))
            else:
                s = {"none": 0, "all": (1 << (64 * words)) - 1}[kind]
            sets.append(s)
        rows += [[(s >> (64 * w)) & ((1 << 64) - 1) for w in range(words)] for s in sets]
    return bits(rows).view(-1, words)


# -- append -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,P,D,counts,lens,pad", [
    (1, 8, 64, [1], [0], 0), (2, 16, 128, [3, 0, 70, 1], [5, 9, 13, 0], 0), (3, 64, 64, [64, 130], [0, 63], 5), (2, 24, 128, [17, 31], [23, 24], 3), (1, 128, 128, [129], [1], 8)])
def test_append(dtype, H, P, D, counts, lens, pad):
    pk, gen = _pk(), torch.Generator().manual_seed(P + len(counts))
    n, rows, stride = len(counts), sum(counts), max(-(-(a + b) // P) for a, b in zip(counts, lens)) + 1
    pool, table = make_pool(gen, 2, n * stride + 3, H, P, D, dtype), tables(gen, n, stride, 3)
    both = torch.randn(rows + 2, 2 * H * D + pad, generator=gen).to(dtype)       # two rows behind the last sequence
    cu, lens = starts(counts), i32(lens)
    want = pool.clone()
    ref.append(want, 1, both[:rows, :H * D].contiguous(), both[:rows, H * D:2 * H * D].contiguous(), cu, lens, table)
    got, b = pool.to(DEV), both.to(DEV)
    pk.focus_kv_append(got, 1, b[:, :H * D], b[:, H * D:2 * H * D], cu.to(DEV), lens.to(DEV), table.to(DEV))
    assert torch.equal(got.cpu(), want)


def test_append_leaves_out_tokens_without_a_page():
    pk, gen = _pk(), torch.Generator().manual_seed(1)
    pool = make_pool(gen, 1, 6, 2, 16, 64, torch.bfloat16)
    table = i32([[0, -1, 2], [6, 1, 3], [4, 5, -7]])           # a hole, a page behind the pool's last one, a negative one
    cu, lens = starts([40, 50, 20]), i32([2, 3, 40])
    x = torch.randn(110, 2 * 2 * 64, generator=gen).to(torch.bfloat16)
    want = pool.clone()
    ref.append(want, 0, x[:, :128], x[:, 128:], cu, lens, table)
    got = pool.to(DEV)
    pk.focus_kv_append(got, 0, x.to(DEV)[:, :128], x.to(DEV)[:, 128:], cu.to(DEV), lens.to(DEV), table.to(DEV))
    assert torch.equal(got.cpu(), want) and not torch.equal(want, pool)


# -- tree attention -----------------------------------------------------------------------------
def check_tree(pool, q, cu, lens, table, seen, scale=None, ldo=None, **kw):
    pk = _pk()
    D = pool.shape[5]
    rows, width = q.shape
    live = int(cu[-1])
    want, size, spread, count = ref.attention(pool, 0, q[:live], cu, lens, table, seen, D ** -0.5 if scale is None else scale)
    wide = torch.full((rows, ldo or width), 7.0, dtype=q.dtype, device=DEV)
    out = wide[:, :width]
    args = [pool.to(DEV), 0, q.to(DEV), cu.to(DEV), lens.to(DEV), table.to(DEV)]
    s = None if seen is None else seen.to(DEV)
    pk.focus_tree_attention(*args, seen=s, out=out, scale=scale, **kw)
    first = wide.cpu()
    wide.fill_(7.0)
    pk.focus_tree_attention(*args, seen=s, out=out, scale=scale, **kw)
    as_bits = torch.int16 if q.dtype == torch.bfloat16 else torch.int32
    assert torch.equal(first.view(as_bits), wide.cpu().view(as_bits))
    assert bool((first[live:] == 7.0).all()) and bool((first[:, width:] == 7.0).all())
    got = first[:live, :width].double()
    # A score is a sum of D products (off by D 2^-24 of the sum of their sizes), its distance from the maximum is rounded once more, and the exponential is
    # off by 2^-22 and by what 2^-23 of its argument (at most twice the spread) makes; weights are off by twice that, as their sum is too.  Sums over n tokens add n 2^-24.
    # bf16: weights are rounded (2^-8), and so is the result.
    weight = 2 * ((2 * D + 8) * 2.0 ** -24 * spread + 2.0 ** -22 + 2 * 2.0 ** -23 * spread) + (count.unsqueeze(1) + 16) * 2.0 ** -24
    half = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -24
    bound = (weight + (half if q.dtype == torch.bfloat16 else 0.0)) * 1.01 * size + half * want.abs() + 1e-30
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    off = torch.where(torch.isnan(want), 0.0, (got - want).abs())
    bound = torch.where(torch.isnan(want), 0.0, bound)
    assert bool((off <= bound).all()), (float((off - bound).max()), int((off > bound).sum()), torch.nonzero(off > bound)[:4].tolist())


def tree_case(gen, dtype, Hq, H, P, D, lens, counts, extra_rows=0, poison=True):
    """A pool that is NaN wherever no sequence has a token."""
    n, stride = len(lens), max(-(-(a + b) // P) for a, b in zip(lens, counts)) + 1
    table = tables(gen, n, stride, 2)
    pool = make_pool(gen, 1, n * stride + 2, H, P, D, dtype, NAN if poison else 0.0)
    cu, lens = starts(counts), i32(lens)
    everything = starts([int(a) + b for a, b in zip(lens, counts)])
    x = torch.randn(int(everything[-1]), 2 * H * D, generator=gen).to(dtype)
    ref.append(pool, 0, x[:, :H * D], x[:, H * D:], everything, torch.zeros_like(lens), table)
    q = torch.randn(int(cu[-1]) + extra_rows, Hq * D, generator=gen).to(dtype)
    return pool, q, cu, lens, table


SHAPES = [(1, 1, 64, 128), (8, 2, 64, 128), (6, 2, 16, 64), (5, 1, 24, 128), (4, 4, 128, 64), (32, 2, 64, 64), (3, 1, 8, 64), (2, 2, 32, 128)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,H,P,D", SHAPES)
@pytest.mark.parametrize("kind", ["tree", "noise", "none", "all", None])
def test_tree_attention(dtype, Hq, H, P, D, kind):
    gen = torch.Generator().manual_seed(Hq * 100 + P + D)
    lens, counts = [0, 1, 63, 64, 130, 0, 200, 7], [1, 2, 1, 9, 0, 17, 33, 64]
    pool, q, cu, lens, table = tree_case(gen, dtype, Hq, H, P, D, lens, counts, extra_rows=3)
    seen = None if kind is None else torch.cat([tree_masks(gen, counts, 1, kind), torch.full((3, 1), -1, dtype=torch.int64)])
    check_tree(pool, q, cu, lens, table, seen, max_rows=64, max_len=233)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tree_attention_of_more_than_64_drafted_tokens(dtype):
    gen = torch.Generator().manual_seed(5)
    counts = [150, 65, 1]
    pool, q, cu, lens, table = tree_case(gen, dtype, 4, 2, 64, 128, [40, 0, 100], counts)
    for words in (1, 2, 3):
        for kind in ("tree", "noise"):
            seen = tree_masks(gen, counts, 3, kind)[:, :words].contiguous()
            check_tree(pool, q, cu, lens, table, seen, max_rows=150, max_len=190)
    check_tree(pool, q, cu, lens, table, None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("P,D", [(64, 128), (16, 64), (128, 64)])
@pytest.mark.parametrize("hint", [(0, 0), (1, 1), (8, 4000), (64, 1 << 20)])
def test_tree_attention_of_long_caches(dtype, P, D, hint):
    """Caches that are cut into parts, whatever the host knows of the lengths."""
    gen = torch.Generator().manual_seed(9)
    counts = [8, 3, 1, 8]
    pool, q, cu, lens, table = tree_case(gen, dtype, 4, 2, P, D, [3001, 1, 1500, 640], counts)
    check_tree(pool, q, cu, lens, table, tree_masks(gen, counts, 1, "tree"), max_rows=hint[0], max_len=hint[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tree_attention_strides_and_scales(dtype):
    gen = torch.Generator().manual_seed(11)
    counts = [3, 9]
    pool, q, cu, lens, table = tree_case(gen, dtype, 4, 2, 32, 64, [70, 20], counts)
    seen = tree_masks(gen, counts, 1, "tree")
    for pad in (1, 8, 64):
        wide = torch.zeros(q.shape[0], q.shape[1] + pad, dtype=dtype)
        wide[:, :q.shape[1]] = q
        check_tree(pool, wide[:, :q.shape[1]], cu, lens, table, seen, ldo=q.shape[1] + 2 * pad)
    for scale in (0.0, 1.0, -0.3, 3.0):
        check_tree(pool, q, cu, lens, table, seen, scale=scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_tree_attention_of_masked_tokens_that_are_no_numbers(dtype, bad):
    """Drafted tokens that hold NaN or infinities count for the rows that see them and for no other."""
    gen = torch.Generator().manual_seed(13)
    counts, lens = [12, 5, 30], [50, 0, 190]
    pool, q, cu, lens, table = tree_case(gen, dtype, 4, 2, 64, 128, lens, counts)
    where = [(0, 50 + 3), (0, 50 + 9), (1, 2), (2, 190 + 1), (2, 190 + 20)]
    seen = torch.full((47, 1), -1, dtype=torch.int64)
    for b, t in where:
        page, place = ref.place_of(pool, table[b], t)
        pool[0, page, 0, :, place, :] = bad
        pool[0, page, 1].view(2, 128, 64)[:, :, place] = bad
        seen &= ~(1 << (t - int(lens[b]))) if b == 2 else -1
    for b, t in where:
        rows = slice(int(cu[b]), int(cu[b + 1]))
        seen[rows] &= ~(1 << (t - int(lens[b])))
    check_tree(pool, q, cu, lens, table, seen)
    # rows that do see one: not a number there (V of +-inf may also give +-inf), the others unchanged
    pk = _pk()
    args = [pool.to(DEV), 0, q.to(DEV), cu.to(DEV), lens.to(DEV), table.to(DEV)]
    clean = pk.focus_tree_attention(*args, seen=seen.to(DEV)).cpu()
    seen[4] |= 1 << 3
    seen[20] |= 1 << 20
    got = pk.focus_tree_attention(*args, seen=seen.to(DEV)).cpu()
    others = [r for r in range(47) if r not in (4, 20)]
    assert torch.equal(got[others], clean[others])
    if bad != -math.inf:
        assert not bool(torch.isfinite(got[4]).any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tree_attention_values_that_are_no_numbers_for_some_rows_only(dtype):
    """V alone: rows that do not see the token have their own sums."""
    gen = torch.Generator().manual_seed(14)
    counts = [20]
    pool, q, cu, lens, table = tree_case(gen, dtype, 8, 2, 64, 128, [60], counts)
    for t in (62, 70, 64):
        page, place = ref.place_of(pool, table[0], t)
        pool[0, page, 1].view(2, 128, 64)[:, 5, place] = math.inf if t != 64 else math.nan
    seen = tree_masks(gen, counts, 1, "tree")
    pk = _pk()
    want, _, _, _ = ref.attention(pool, 0, q, cu, lens, table, seen, 128 ** -0.5)
    got = pk.focus_tree_attention(pool.to(DEV), 0, q.to(DEV), cu.to(DEV), lens.to(DEV), table.to(DEV), seen=seen.to(DEV)).cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), fine)
    assert bool(((got - want).abs()[fine] <= 0.02).all()) and not bool(fine.all())


def test_tree_attention_leaves_out_tokens_without_a_page():
    gen = torch.Generator().manual_seed(15)
    for dtype in (torch.bfloat16, torch.float32):
        pool, q, cu, lens, table = tree_case(gen, dtype, 4, 2, 16, 64, [70, 33, 20, 5], [3, 9, 4, 2])
        table[0, 2], table[1, 0], table[2] = -1, pool.shape[1], -1
        lens[3] = 10 ** 9                                       # beyond the table
        table[3, :] = table[3, 0]
        for kind in ("tree", "all"):
            check_tree(pool, q, cu, lens, table, tree_masks(gen, [3, 9, 4, 2], 1, kind))


def test_tree_attention_without_rows():
    pk = _pk()
    pool = torch.zeros(1, 2, 2, 1, 16, 64, device=DEV)
    q = torch.zeros(0, 64, device=DEV)
    assert pk.focus_tree_attention(pool, 0, q, i32([0, 0]).to(DEV), i32([3]).to(DEV), i32([[0]]).to(DEV)).shape == (0, 64)
    q = torch.ones(2, 64, device=DEV)
    out = torch.full_like(q, 5.0)
    pk.focus_tree_attention(pool, 0, q, i32([0, 0, 0]).to(DEV), i32([3, 0]).to(DEV), i32([[0], [1]]).to(DEV), out=out)
    assert bool((out == 5.0).all())


# -- compaction -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,P,D,spans,start,share", [
    (1, 8, 64, [1], [0], 1.0), (2, 16, 128, [40, 0, 9, 100], [3, 0, 16, 50], 0.5), (2, 64, 64, [200, 5], [0, 60], 0.3), (1, 24, 128, [130, 64], [7, 24], 0.8), (3, 64, 128, [300], [1], 0.1)])
@pytest.mark.parametrize("in_place", [True, False])
def test_compact(dtype, H, P, D, spans, start, share, in_place):
    pk, gen = _pk(), torch.Generator().manual_seed(P + len(spans))
    n, stride = len(spans), max(-(-(a + b) // P) for a, b in zip(spans, start)) + 1
    both = tables(gen, 2 * n, stride)
    pool = make_pool(gen, 3, 2 * n * stride, H, P, D, dtype)
    keep = [[x for x in range(s) if float(torch.rand(1, generator=gen)) <= share] for s in spans]
    table, to = both[:n].contiguous(), both[n:].contiguous()
    cu, flat, start = starts([len(x) for x in keep]), i32([x for k in keep for x in k]), i32(start)
    want = pool.clone()
    ref.compact(want, start, cu, flat, table, table if in_place else to)
    got = pool.to(DEV)
    pk.focus_kv_compact(got, start.to(DEV), cu.to(DEV), flat.to(DEV), table.to(DEV), None if in_place else to.to(DEV))
    assert torch.equal(got.cpu(), want)


def test_compact_into_a_table_that_shares_its_first_pages():
    """The accepted tokens go on in pages of their own while the full pages before them stay shared: to_table begins with the same pages."""
    pk, gen = _pk(), torch.Generator().manual_seed(3)
    pool = make_pool(gen, 2, 12, 2, 16, 64, torch.bfloat16)
    table, to = i32([[0, 1, 2, 3], [0, 4, 5, 6]]), i32([[0, 1, 7, -1], [0, 4, 8, -1]])
    start, cu, keep = i32([20, 30]), i32([0, 14, 17]), i32(list(range(0, 28, 2)) + [0, 3, 7])
    want = pool.clone()
    ref.compact(want, start, cu, keep, table, to)
    got = pool.to(DEV)
    pk.focus_kv_compact(got, *(t.to(DEV) for t in (start, cu, keep, table, to)))
    assert torch.equal(got.cpu(), want)


def test_compact_leaves_out_tokens_without_a_page():
    pk, gen = _pk(), torch.Generator().manual_seed(4)
    pool = make_pool(gen, 1, 8, 1, 16, 64, torch.float32)
    table, to = i32([[0, -1, 9, 1], [2, 3, 4, -1]]), i32([[5, 8], [6, 7]])
    start, cu, keep = i32([0, 0]), i32([0, 30, 62]), i32(list(range(1, 61, 2)) + list(range(5, 37)))
    want = pool.clone()
    ref.compact(want, start, cu, keep, table, to)
    got = pool.to(DEV)
    pk.focus_kv_compact(got, *(t.to(DEV) for t in (start, cu, keep, table, to)))
    assert torch.equal(got.cpu(), want)


# -- fork and reserve -------------------------------------------------------------------------------
def random_rows(gen, n, P, stride, n_pages, groups=3):
    """Rows that share their first pages in groups, with lengths inside what they hold; and the counts."""
    order, table, lens = torch.randperm(n_pages, generator=gen).tolist(), [], []
    refs, shared = [0] * n_pages, {}
    for b in range(n):
        g = b % groups
        if g not in shared:
            shared[g] = [order.pop() for _ in range(int(torch.randint(0, stride // 2 + 1, (1,), generator=gen)))]
        mine = [order.pop() for _ in range(int(torch.randint(0, stride - len(shared[g]) + 1, (1,), generator=gen)))]
        row = shared[g] + mine
        for p in row:
            refs[p] += 1
        low, high = len(shared[g]) * P, len(row) * P
        lens.append(int(torch.randint(low, high + 1, (1,), generator=gen)))
        table.append(row + [-1] * (stride - len(row)))
    return table, lens, refs


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_old,n_new,P,H,D,stride,spare", [(1, 1, 8, 1, 64, 2, 4), (1, 5, 16, 2, 128, 4, 40), (7, 7, 64, 2, 64, 3, 30), (12, 30, 24, 1, 128, 5, 60), (12, 30, 16, 1, 64, 5, 4),
                                                           (5, 0, 16, 1, 64, 4, 3), (0, 3, 16, 1, 64, 4, 3), (70, 300, 8, 1, 64, 3, 20)])
def test_fork_then_reserve(dtype, n_old, n_new, P, H, D, stride, spare):
    pk, gen = _pk(), torch.Generator().manual_seed(n_old * 10 + n_new + P)
    n_pages = max(1, n_old * stride + spare - n_old * stride // 3)
    table, lens, refs = random_rows(gen, n_old, P, stride, max(n_pages, n_old * stride))
    n_pages = len(refs)
    pool = make_pool(gen, 2, n_pages, H, P, D, dtype)
    parents = torch.randint(-1, n_old + 1, (n_new,), generator=gen).tolist()       # some outside
    want_pool, want_refs, want_table = pool.clone(), list(refs), None
    want_lens, want_table, want_lack = ref.fork(want_pool, parents, lens, table, want_refs, stride)
    got_pool, got_refs = pool.to(DEV), i32(refs).to(DEV)
    old = i32(table).view(n_old, stride).to(DEV)
    before = old.clone()
    got_lens, got_table, lack = pk.focus_kv_fork(got_pool, i32(parents).to(DEV), i32(lens).to(DEV), old, got_refs)
    assert got_lens.tolist() == want_lens and got_table.tolist() == want_table and lack.tolist() == want_lack
    assert got_refs.tolist() == want_refs and torch.equal(old, before)
    assert torch.equal(got_pool.cpu(), want_pool)
    held = [0] * n_pages                                                           # counts are what the tables hold
    for row in want_table:
        for p in row[:ref.held(row)]:
            held[p] += 1
    assert held == want_refs
    for room in (0, 1, P, 3 * P):
        want = ref.reserve(want_lens, room, want_table, want_refs, P)
        got = pk.focus_kv_reserve(got_lens, room, got_table, got_refs, P)
        assert got.tolist() == want and got_table.tolist() == want_table and got_refs.tolist() == want_refs


def test_a_pool_that_runs_out():
    pk = _pk()
    P, pool = 16, torch.zeros(1, 6, 2, 1, 16, 64, device=DEV)
    refs = i32([1, 1, 0, 1, 0, 1]).to(DEV)
    lens, table, lack = pk.focus_kv_fork(pool, i32([0, 0, 0, 0]).to(DEV), i32([20]).to(DEV), i32([[0, 1, -1, -1]]).to(DEV), refs)
    assert table.tolist() == [[0, 1, -1, -1], [0, 2, -1, -1], [0, 4, -1, -1], [0, -1, -1, -1]]
    assert lens.tolist() == [20, 20, 20, 16] and lack.tolist() == [0, 0, 0, 1] and refs.tolist() == [4, 1, 1, 1, 1, 1]
    assert pk.focus_kv_reserve(lens, 13, table, refs, P).tolist() == [1, 1, 1, 1]
    lens, table, lack = pk.focus_kv_fork(pool, i32([3, 1]).to(DEV), lens, table, refs)
    assert table.tolist() == [[0, -1, -1, -1], [0, 2, -1, -1]] and lens.tolist() == [16, 20] and refs.tolist() == [2, 1 - 1, 1, 1, 0, 1]
    assert pk.focus_kv_reserve(lens, 32, table, refs, P).tolist() == [0, 2]
    assert table.tolist() == [[0, 1, 4, -1], [0, 2, -1, -1]]
    pk.focus_kv_fork(pool, i32([]).to(DEV), lens, table, refs)
    assert refs.tolist() == [0, 0, 0, 1, 0, 1]
    assert pk.focus_kv_reserve(i32([10 ** 9]).to(DEV), 2 ** 31 - 1, i32([[-1, -1]]).to(DEV), refs, P).tolist() == [-(-(10 ** 9 + 2 ** 31 - 1) // P) - 2]


def test_many_pages():
    """More pages than a workgroup looks at in one go, the free ones at the end; wants of several pages a row."""
    pk, gen = _pk(), torch.Generator().manual_seed(2)
    n_pages, n, P, stride = 50001, 33, 8, 40
    refs = [1] * n_pages
    for p in torch.randint(n_pages - 20000, n_pages, (700,), generator=gen).tolist():
        refs[p] = 0
    lens = torch.randint(0, 300, (n,), generator=gen).tolist()
    table = [[-1] * stride for _ in range(n)]
    want_refs, lacks = list(refs), []
    got_table, got_refs = torch.full((n, stride), -1, dtype=torch.int32, device=DEV), i32(refs).to(DEV)
    for room in (5, 90):                                       # enough pages, then too few
        want = ref.reserve(lens, room, table, want_refs, P)
        got = pk.focus_kv_reserve(i32(lens).to(DEV), room, got_table, got_refs, P)
        assert got.tolist() == want and got_table.tolist() == table and got_refs.tolist() == want_refs
        lacks.append(sum(want))
    assert lacks[0] == 0 and lacks[1] > 0


# -- beam selection -----------------------------------------------------------------------------------
def check_beam(logits, scores, k, done=None, end_token=3):
    """logits: a CPU tensor [n * beams, vocab], possibly a view of columns."""
    pk = _pk()
    wide = torch.zeros(logits.shape[0], logits.stride(0) if logits.shape[0] > 1 else logits.shape[1], dtype=logits.dtype, device=DEV)
    view = wide[:, :logits.shape[1]]
    view.copy_(logits)
    want = ref.beam(logits, scores, k, done, end_token)
    got = pk.focus_beam_select(view, scores.to(DEV), k, done=None if done is None else done.to(DEV), end_token=end_token)
    again = pk.focus_beam_select(view, scores.to(DEV), k, done=None if done is None else done.to(DEV), end_token=end_token)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    assert got[0].tolist() == want[0] and got[1].tolist() == want[1]
    g, w = got[2].cpu().double(), torch.tensor(want[2], dtype=torch.float64)
    none = torch.isinf(w)
    assert torch.equal(torch.isinf(g), none)
    # rounded once to fp32; the 64-bit values before are off by far less
    assert bool(((g - w).abs()[~none] <= w.abs()[~none] * 2.0 ** -24 * 1.001 + 1e-12).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,beams,vocab,k,pad", [(1, 1, 1, 1, 0), (1, 4, 3, 8, 0), (2, 1, 1000, 64, 0), (3, 5, 513, 10, 3), (1, 64, 70, 64, 1), (2, 3, 4099, 6, 5), (1, 2, 40000, 16, 0),
                                                (5, 12, 257, 24, 7), (1, 2, 151936, 4, 0)])
def test_beam_select(dtype, n, beams, vocab, k, pad):
    gen = torch.Generator().manual_seed(vocab + k)
    logits = (torch.randn(n * beams, vocab + pad, generator=gen) * 3).to(dtype)[:, :vocab]
    scores = -torch.rand(n, beams, generator=gen) * 4
    check_beam(logits, scores, k)
    done = torch.rand(n, beams, generator=gen) < 0.4
    check_beam(logits, scores, k, done)
    check_beam(logits, scores, k, torch.ones(n, beams, dtype=torch.uint8), end_token=-5)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_beam_select_ties_and_values_that_are_no_numbers(dtype):
    gen = torch.Generator().manual_seed(21)
    n, beams, vocab = 16, 4, 300
    l = torch.randn(n, beams, vocab, generator=gen).to(dtype)
    scores = -torch.rand(n, beams, generator=gen)
    l[0] = 0.0                                             # all equal
    l[1] = torch.round(l[1])                               # many equal
    l[2, 1] = l[2, 0]                                      # equal beams
    scores[2] = -1.0
    l[3, 0] = -math.inf
    l[4, :, 10:] = -math.inf                               # fewer than k that count
    l[5, 1, 7] = math.nan
    l[6, 2, 7] = math.inf
    l[7] = -math.inf
    scores[8, 1:] = -math.inf                              # the first step: one beam
    scores[9] = math.nan
    l[10] = math.nan
    scores[11, 0], scores[11, 1] = math.inf, math.nan
    l[12] = l[12] * 1000
    l[13] = torch.finfo(dtype).min                          # the lowest value as a mask
    l[13, :, 5:25] = torch.randn(4, 20, generator=gen).to(dtype)
    l[14, 0, ::2], l[14, 0, 1::2] = 0.0, -0.0
    l[15, :, 0] = 80.0
    done = torch.zeros(n, beams, dtype=torch.bool)
    done[9, 0] = done[10, 2] = done[11, 0] = done[2, 3] = True
    for k in (1, 8, 24, 64):
        check_beam(l.view(n * beams, vocab), scores, k)
        check_beam(l.view(n * beams, vocab), scores, k, done)


@pytest.mark.parametrize("order", ["rising", "falling", "equal", "late"])
def test_beam_select_of_sorted_logits(order):
    vocab = 30011
    base = torch.linspace(-8, 8, vocab)
    row = {"rising": base, "falling": base.flip(0), "equal": torch.full((vocab,), 1.5), "late": torch.cat([torch.zeros(vocab - 40), torch.linspace(1, 2, 40)])}[order]
    for dtype in (torch.float32, torch.bfloat16):
        check_beam(torch.stack([row, row.flip(0)]).to(dtype), torch.tensor([[-1.0, -1.25]]), 32)


def test_beam_select_close_calls_are_those_of_64_bits():
    """Two beams whose best candidates differ by less than fp32 sums could tell."""
    gen = torch.Generator().manual_seed(23)
    for seed in range(6):
        l = torch.randn(2, 5000, generator=gen)
        lse = torch.logsumexp(l.double(), 1)
        top = l.max(1).values.double()
        scores = torch.zeros(1, 2)
        scores[0, 1] = float((top[0] - lse[0]) - (top[1] - lse[1]))
        check_beam(l, scores, 2)


# -- together ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_tree_is_drafted_verified_and_compacted(dtype):
    """Drafted tokens go into the cache, attention follows the tree, the accepted path is moved together; a single token after that sees exactly that path."""
    pk, gen = _pk(), torch.Generator().manual_seed(31)
    H, Hq, P, D, layers, stride = 2, 8, 16, 64, 2, 8
    lens, counts = [0, 17, 60], [9, 5, 12]
    n = len(lens)
    pool, refs = torch.full((layers, n * stride + 4, 2, H, P, D), NAN, dtype=dtype).to(DEV), torch.zeros(n * stride + 4, dtype=torch.int32, device=DEV)
    table = torch.full((n, stride), -1, dtype=torch.int32, device=DEV)
    cached = [torch.randn(layers, x, 2 * H * D, generator=gen).to(dtype) for x in lens]
    drafted = torch.randn(layers, sum(counts), 2 * H * D, generator=gen).to(dtype)
    q = torch.randn(sum(counts), Hq * D, generator=gen).to(dtype).to(DEV)
    cu, held = starts(counts).to(DEV), i32(lens).to(DEV)
    assert pk.focus_kv_reserve(held, 12, table, refs, P).tolist() == [0, 0, 0]
    for l in range(layers):
        x = torch.cat([c[l] for c in cached]).to(DEV)
        pk.focus_kv_append(pool, l, x[:, :H * D], x[:, H * D:], starts(lens).to(DEV), torch.zeros_like(held), table)
        d = drafted[l].to(DEV)
        pk.focus_kv_append(pool, l, d[:, :H * D], d[:, H * D:], cu, held, table)
    seen = tree_masks(gen, counts, 1, "tree")
    paths = []                                               # the accepted path of each: ancestors of its last token, in order
    for b, c in enumerate(counts):
        word = int(seen[int(cu[b]) + c - 1])
        paths.append([j for j in range(c) if word >> j & 1])
    verified = pk.focus_tree_attention(pool, 1, q, cu, held, table, seen=seen.to(DEV), max_rows=12, max_len=72)
    pk.focus_kv_compact(pool, held, starts([len(p) for p in paths]).to(DEV), i32([j for p in paths for j in p]).to(DEV), table)
    held = held + i32([len(p) for p in paths]).to(DEV)
    for b in range(n):
        # the last row of the tree saw the cache and its path: so does a single row now whose token is the path's last
        r = int(cu[b]) + counts[b] - 1
        dense = torch.cat([cached[b][1], drafted[1][int(cu[b]):int(cu[b + 1])][paths[b]]])
        k, v = dense[:, :H * D].double().view(-1, H, D), dense[:, H * D:].double().view(-1, H, D)
        one = pk.focus_tree_attention(pool, 1, q[r:r + 1], i32([0, 1]).to(DEV), held[b:b + 1] - 1, table[b:b + 1])
        for h in range(Hq):
            w = torch.softmax(k[:, h // 4] @ q[r, h * D:(h + 1) * D].double().cpu() * D ** -0.5, 0) @ v[:, h // 4]
            size = float(v.abs().max())
            for got in (one[0], verified[r]):
                assert float((got[h * D:(h + 1) * D].cpu().double() - w).abs().max()) <= (2 * 2.0 ** -8 if dtype == torch.bfloat16 else 1e-5) * size


def beam_search(pk, gen, embed, pool, refs, table, lens, steps, n, beams, H, D, P, stream=None, histories=None):
    """A toy decoder of one layer: the token's row is its key, value and query; logits are its attention against the embedding."""
    scores = torch.full((n, beams), -math.inf, device=DEV)
    scores[:, 0] = 0.0
    token = torch.zeros(n * beams, dtype=torch.long, device=DEV)
    rows = torch.arange(n * beams + 1, dtype=torch.int32, device=DEV)
    for step in range(steps):
        pk.focus_kv_reserve(lens, 1, table, refs, P)
        x = embed[token]
        pk.focus_kv_append(pool, 0, x[:, :H * D], x[:, H * D:2 * H * D], rows, lens, table)
        out = pk.focus_tree_attention(pool, 0, x[:, 2 * H * D:].contiguous(), rows, lens, table, max_rows=1)
        lens = lens + 1
        picked, tokens, new = pk.focus_beam_select((out.float() @ embed[:, 2 * H * D:].float().t()).contiguous(), scores, beams)
        lens, table, lacking = pk.focus_kv_fork(pool, picked.view(-1), lens, table, refs)
        assert not bool(lacking.any())
        scores, token = new, tokens.view(-1).long()
        if histories is not None:
            histories = [histories[p] + [int(t)] for p, t in zip(picked.view(-1).tolist(), token.tolist())]
    return scores, lens, table, histories


def test_beam_search_over_shared_pages():
    """Beams that share and copy pages have the scores of their own histories, worked out from scratch in 64 bits."""
    pk, gen = _pk(), torch.Generator().manual_seed(37)
    n, beams, H, D, P, vocab, steps, stride = 2, 3, 1, 64, 8, 50, 21, 6
    embed = (torch.randn(vocab, 3 * H * D, generator=gen)).to(DEV)
    pool = torch.full((1, 60, 2, H, P, D), NAN, device=DEV)
    refs, table = torch.zeros(60, dtype=torch.int32, device=DEV), torch.full((n * beams, stride), -1, dtype=torch.int32, device=DEV)
    lens = torch.zeros(n * beams, dtype=torch.int32, device=DEV)
    scores, lens, table, histories = beam_search(pk, gen, embed, pool, refs, table, lens, steps, n, beams, H, D, P, histories=[[0] for _ in range(n * beams)])
    e = embed.double().cpu()
    for i in range(n * beams):
        x = e[histories[i][:-1]]
        total = 0.0
        for t in range(steps):
            w = torch.softmax(x[:t + 1, :D] @ x[t, 2 * D:] * D ** -0.5, 0) @ x[:t + 1, D:2 * D]
            l = e[:, 2 * D:] @ w
            total += float(l[histories[i][t + 1]] - torch.logsumexp(l, 0))
        assert abs(float(scores.view(-1)[i]) - total) <= 2e-4 * max(1.0, abs(total))
    assert lens.tolist() == [steps] * (n * beams)
    for parents in (list(range(n * beams)), [0] * 4 + [5, 5], [2, 1, 5, 4, 3, 0]):
        lens, table, lacking = pk.focus_kv_fork(pool, i32(parents).to(DEV), lens, table, refs)
        held = [0] * 60
        for row in table.tolist():
            for p in row[:ref.held(row)]:
                held[p] += 1
        assert refs.tolist() == held and not bool(lacking.any())
    assert max(held) == 4
    pk.focus_kv_fork(pool, i32([]).to(DEV), lens, table, refs)
    assert not bool(refs.any())
