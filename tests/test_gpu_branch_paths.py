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
