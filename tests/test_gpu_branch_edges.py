"""Branching generation on the GPU where calls meet: graphs, streams, workspaces, many sequences, offsets past 32 bits, a context; and what the binding refuses."""
import math

import pytest
import torch

import branch_reference as ref
import focus_inputs as fi
from test_gpu_branch import DEV, beam_search, check_beam, check_tree, i32, make_pool, starts, tables, tree_case, tree_masks

pytestmark = pytest.mark.gpu


def _pk():
    import paper_2601_23278_amd as pk
    return pk


# -- sizes that other paths take -------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("room", [None, 0, 4096])
def test_tree_attention_of_many_sequences(dtype, room):
    """More sequences than a workgroup sums up for itself, some without rows; with the workspace, without one, and with one for the starts alone."""
    gen = torch.Generator().manual_seed(41)
    n = 300
    lens = torch.randint(0, 90, (n,), generator=gen).tolist()
    counts = torch.randint(0, 4, (n,), generator=gen).tolist()
    pool, q, cu, lens, table = tree_case(gen, dtype, 2, 1, 16, 64, lens, counts)
    kw = {} if room is None else dict(workspace=torch.empty(max(room, 1), dtype=torch.uint8, device=DEV)[:room])
    check_tree(pool, q, cu, lens, table, tree_masks(gen, counts, 1, "tree"), max_rows=3, max_len=93, **kw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tree_attention_with_less_workspace(dtype):
    gen = torch.Generator().manual_seed(42)
    counts = [8, 30, 1]
    pool, q, cu, lens, table = tree_case(gen, dtype, 8, 2, 64, 128, [700, 64, 2000], counts)
    for size in (0, 256, 100000):
        check_tree(pool, q, cu, lens, table, tree_masks(gen, counts, 1, "tree"), workspace=torch.empty(size, dtype=torch.uint8, device=DEV))


@pytest.mark.parametrize("heads,H", [(1, 1), (7, 7), (24, 8), (16, 1), (64, 16)])
def test_tree_attention_head_layouts(heads, H):
    gen = torch.Generator().manual_seed(heads)
    counts = [1, 5, 3]
    for dtype in (torch.bfloat16, torch.float32):
        pool, q, cu, lens, table = tree_case(gen, dtype, heads, H, 16, 64, [900, 3, 70], counts)
        check_tree(pool, q, cu, lens, table, tree_masks(gen, counts, 1, "tree"), max_rows=5, max_len=905)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_compact_of_thousands_of_tokens_in_place(dtype):
    pk, gen = _pk(), torch.Generator().manual_seed(43)
    n, P, stride = 3, 64, 50
    table = tables(gen, n, stride)
    pool = make_pool(gen, 1, n * stride, 1, P, 64, dtype)
    spans, start = [3000, 1, 2500], i32([100, 0, 13])
    keep = [[x for x in range(s) if float(torch.rand(1, generator=gen)) < share] for s, share in zip(spans, (0.5, 1.1, 0.95))]
    cu, flat = starts([len(x) for x in keep]), i32([x for k in keep for x in k])
    want = pool.clone()
    ref.compact(want, start, cu, flat, table, table)
    got = pool.to(DEV)
    pk.focus_kv_compact(got, start.to(DEV), cu.to(DEV), flat.to(DEV), table.to(DEV))
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("n_old,n_new,stride", [(3, 7, 300), (2, 3, 777), (300, 9000, 2)])
def test_fork_and_reserve_of_long_tables_and_many_rows(n_old, n_new, stride):
    """Rows longer than a workgroup looks at in one go, and more wants than are held at once."""
    pk, gen = _pk(), torch.Generator().manual_seed(stride)
    P, n_pages = 8, n_old * stride + n_new + 5
    order = torch.randperm(n_pages, generator=gen).tolist()
    table, lens, refs = [], [], [0] * n_pages
    for b in range(n_old):
        held = int(torch.randint(stride // 2, stride, (1,), generator=gen))
        row = [order.pop() for _ in range(held)]
        for p in row:
            refs[p] += 1
        table.append(row + [-1] * (stride - held))
        lens.append(int(torch.randint((held - 1) * P, held * P + 1, (1,), generator=gen)) if held else 0)
    pool = make_pool(gen, 1, n_pages, 1, P, 64, torch.bfloat16)
    parents = torch.randint(0, n_old, (n_new,), generator=gen).tolist()
    if n_new > 1000:                                       # the reference walks the pool for every page: the copies alone are compared
        old = i32(table).to(DEV)
        got_refs, got_pool = i32(refs).to(DEV), pool.to(DEV)
        new_lens, new_table, lack = (t.cpu() for t in pk.focus_kv_fork(got_pool, i32(parents).to(DEV), i32(lens).to(DEV), old, got_refs))
        held = torch.zeros(n_pages, dtype=torch.int32)
        held.index_add_(0, new_table[new_table >= 0].long(), torch.ones(int((new_table >= 0).sum()), dtype=torch.int32))
        assert torch.equal(held, got_refs.cpu())
        first = set()
        free = sorted(set(p for p in range(n_pages) if refs[p] == 0) | set(p for b in range(n_old) if b not in set(parents) for p in table[b] if p >= 0))
        at = 0
        for i, b in enumerate(parents):
            whole, left = lens[b] // P, lens[b] % P
            if b in first and left:
                assert int(lack[i]) == (at >= len(free)) and (at >= len(free) or int(new_table[i, whole]) == free[at])
                at += 1
            first.add(b)
            assert new_table[i, :whole].tolist() == table[b][:whole]
        assert at > 4096
        more = pk.focus_kv_reserve(new_lens.to(DEV), P, new_table.to(DEV), got_refs, P)
        assert int(more.sum()) > 0 and int((got_refs == 0).sum()) == 0
        return
    want_refs = list(refs)
    want_pool = pool.clone()
    want = ref.fork(want_pool, parents, lens, table, want_refs, stride)
    got_pool, got_refs = pool.to(DEV), i32(refs).to(DEV)
    got = pk.focus_kv_fork(got_pool, i32(parents).to(DEV), i32(lens).to(DEV), i32(table).to(DEV), got_refs)
    assert [t.tolist() for t in got] == list(want) and got_refs.tolist() == want_refs and torch.equal(got_pool.cpu(), want_pool)
    lacks = ref.reserve(want[0], 3 * P, want[1], want_refs, P)
    assert pk.focus_kv_reserve(got[0], 3 * P, got[1], got_refs, P).tolist() == lacks
    assert got[1].tolist() == want[1] and got_refs.tolist() == want_refs


@pytest.mark.parametrize("n,beams,vocab,k", [(1, 64, 70000, 64), (2, 16, 30000, 64), (40, 3, 9000, 6)])
def test_beam_select_of_many_lists(n, beams, vocab, k):
    gen = torch.Generator().manual_seed(vocab)
    for dtype in (torch.float32, torch.bfloat16):
        check_beam((torch.randn(n * beams, vocab, generator=gen) * 2).to(dtype), -torch.rand(n, beams, generator=gen), k)


def test_beam_select_writes_scores_in_place():
    pk, gen = _pk(), torch.Generator().manual_seed(8)
    logits, scores = torch.randn(40 * 6, 5003, generator=gen).to(DEV), (-torch.rand(40, 6, generator=gen)).to(DEV)
    want = pk.focus_beam_select(logits, scores, 6)
    got = pk.focus_beam_select(logits, scores, 6, new_scores=scores)
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and got[2] is scores


# parts alike instead of a short last one, a part of less than a wavefront's loads, and more picks than wavefronts that are full can rule out
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [4096 * 2 + 1, 4096 * 2 + 2047, 4096 * 2 + 2048, 4096 * 5 + 65, 255, 256, 257, 511, 513, 767, 1025])
def test_beam_select_of_parts_that_do_not_come_out_even(dtype, vocab):
    gen = torch.Generator().manual_seed(vocab)
    check_beam((torch.randn(6, vocab, generator=gen) * 2).to(dtype), -torch.rand(2, 3, generator=gen), 64)
    check_beam(torch.randn(6, vocab, generator=gen).round().to(dtype), -torch.rand(2, 3, generator=gen), 5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_beam_select_of_logits_far_from_zero(dtype):
    """Maxima and masks far apart: weights that vanish, references that have to move."""
    gen = torch.Generator().manual_seed(47)
    V = 9001
    l = torch.randn(12, V, generator=gen)
    l[0] -= 5000.0
    l[1] += 3.0e5
    l[2, :8000] = -math.inf
    l[2, 8000:] -= 2000.0
    l[3, :8000] = torch.finfo(dtype).min
    l[4] = torch.linspace(-3000, 3000, V)
    l[5] = torch.linspace(3000, -3000, V)
    l[6] *= 1e30
    l[7, 17] = 1e38
    l[8, :] = -1e38
    l[9, 5000:] += 650.0
    l[10, ::2] -= 900.0
    check_beam(l.to(dtype), -torch.rand(6, 2, generator=gen), 4)
    check_beam(l.to(dtype), -torch.rand(1, 12, generator=gen), 24)


# -- offsets past 32 bits --------------------------------------------------------------------------
def test_pools_of_more_than_4_gib():
    """The same tables in a small pool and at the end of a large one."""
    pk, gen = _pk(), torch.Generator().manual_seed(51)
    H, P, D, pages, far = 8, 64, 128, 40, 18000
    counts, lens = [5, 9], [300, 700]
    small, q, cu, lens, table = tree_case(gen, torch.bfloat16, 16, H, P, D, lens, counts, poison=False)
    pages = small.shape[1]
    large = torch.zeros(1, far + pages, 2, H, P, D, dtype=torch.bfloat16, device=DEV)
    large[:, far:] = small.to(DEV)
    small = small.to(DEV)
    new = torch.randn(14, 2 * H * D, generator=gen).to(torch.bfloat16).to(DEV)
    out = []
    for pool, t in ((small, table), (large, table + far)):
        t = t.to(DEV)
        args = (cu.to(DEV), lens.to(DEV), t)
        pk.focus_kv_append(pool, 0, new[:, :H * D], new[:, H * D:], *args)
        a = pk.focus_tree_attention(pool, 0, q.to(DEV), *args, max_rows=9)
        pk.focus_kv_compact(pool, lens.to(DEV), i32([0, 2, 5]).to(DEV), i32([1, 3, 0, 4, 8]).to(DEV), t)
        b = pk.focus_tree_attention(pool, 0, q.to(DEV), *args, max_rows=9)
        refs = torch.ones(pool.shape[1], dtype=torch.int32, device=DEV)
        refs[:far] = 1
        refs[-1] = 0                                        # the last page is free
        t[t == pool.shape[1] - 1] = -1
        _, forked, lack = pk.focus_kv_fork(pool, i32([0, 0]).to(DEV), lens.to(DEV), t, refs)
        out.append((a, b, pool[:, -pages:].clone(), torch.where(forked >= 0, forked - (pool.shape[1] - pages), forked), lack))
    for x, y in zip(*out):
        assert torch.equal(x, y)


def test_logits_of_more_than_4_gib():
    pk = _pk()
    n, beams, V = 1900, 8, 151936
    logits = torch.empty(n * beams, V, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(3)
    for r in range(0, n * beams, 1024):
        logits[r:r + 1024].normal_(generator=gen)
    scores = -torch.rand(n, beams, device=DEV, generator=gen)
    rows, tokens, new = pk.focus_beam_select(logits, scores, 4)
    last = slice((n - 2) * beams, n * beams)
    part = pk.focus_beam_select(logits[last].clone(), scores[-2:].clone(), 4)
    assert torch.equal(rows[-2:] - (n - 2) * beams, part[0]) and torch.equal(tokens[-2:], part[1]) and torch.equal(new[-2:], part[2])


# -- graphs and streams ------------------------------------------------------------------------------
class Step:
    """One step of a toy decoder with everything in it: room, append, attention, beam selection, fork; its buffers stay where they are."""

    def __init__(self, seed, n, beams, dtype):
        gen = torch.Generator().manual_seed(seed)
        self.n, self.beams, self.H, self.D, self.P = n, beams, 2, 64, 16
        rows, width = n * beams, 2 * 64
        self.embed = torch.randn(40, 3 * width, generator=gen).to(dtype).to(DEV)
        self.pool = torch.zeros(1, rows * 8 + 20, 2, 2, 16, 64, dtype=dtype, device=DEV)
        self.cu = torch.arange(rows + 1, dtype=torch.int32, device=DEV)
        self.state = [torch.zeros(rows, dtype=torch.int32, device=DEV), torch.full((rows, 8), -1, dtype=torch.int32, device=DEV),
                      torch.zeros(rows * 8 + 20, dtype=torch.int32, device=DEV), -torch.rand(n, beams, generator=gen).to(DEV),
                      torch.randint(0, 40, (rows,), generator=gen).to(DEV)]
        self.first = [t.clone() for t in self.state]

    def reset(self):
        self.pool.zero_()
        for t, f in zip(self.state, self.first):
            t.copy_(f)

    def __call__(self, stream=None):
        pk = _pk()
        lens, table, refs, scores, token = self.state
        w = self.H * self.D
        pk.focus_kv_reserve(lens, 1, table, refs, self.P, stream=stream)
        x = self.embed[token]
        pk.focus_kv_append(self.pool, 0, x[:, :w], x[:, w:2 * w], self.cu, lens, table, stream=stream)
        out = pk.focus_tree_attention(self.pool, 0, x[:, 2 * w:], self.cu, lens, table, max_rows=1, stream=stream)
        logits = (out.float() @ self.embed[:, 2 * w:].float().t()).contiguous()
        rows, tokens, new = pk.focus_beam_select(logits, scores, self.beams, stream=stream)
        lens1, table1, _ = pk.focus_kv_fork(self.pool, rows.view(-1), lens + 1, table, refs, stream=stream)
        pk.focus_kv_compact(self.pool, torch.zeros_like(lens1), self.cu, torch.zeros_like(lens1), table1, stream=stream)       # moves nothing
        for t, v in zip((lens, table, scores, token), (lens1, table1, new, tokens.view(-1).long())):
            t.copy_(v)

    def seen(self):
        return [t.clone() for t in self.state] + [self.pool.clone()]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_steps_replay_and_share_nothing(dtype):
    """Two captured steps of different sizes, replayed in turn with eager steps of others between; every replay equals the eager step."""
    steps = [Step(1, 3, 4, dtype), Step(2, 1, 2, dtype)]
    eager = [Step(1, 3, 4, dtype), Step(2, 1, 2, dtype)]
    side = torch.cuda.Stream()
    graphs = []
    for s in steps:
        s()                                               # once before
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            s(stream=side)
        s.reset()
        graphs.append(g)
    for _ in range(20):
        for g, s, e in zip(graphs, steps, eager):
            torch.cuda.synchronize()
            g.replay()
            e()
            torch.cuda.synchronize()
            for a, b in zip(s.seen(), e.seen()):
                assert torch.equal(a, b)


def test_calls_on_streams_at_once():
    streams = [torch.cuda.Stream() for _ in range(3)]
    want, steps = [], [Step(5 + i, 2 + i, 3, torch.bfloat16) for i in range(3)]
    for i in range(3):
        e = Step(5 + i, 2 + i, 3, torch.bfloat16)
        for _ in range(6):
            e()
        torch.cuda.synchronize()
        want.append(e.seen())
    torch.cuda.synchronize()
    for _ in range(6):
        for s, stream in zip(steps, streams):
            with torch.cuda.stream(stream):
                s(stream=stream)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(s.seen(), w))


def test_a_stream_that_is_not_the_current_one():
    """Outputs and workspaces belong to the call's stream."""
    pk, gen = _pk(), torch.Generator().manual_seed(61)
    counts = [4, 7]
    pool, q, cu, lens, table = tree_case(gen, torch.bfloat16, 4, 2, 64, 128, [500, 900], counts)
    args = [t.to(DEV) for t in (q, cu, lens, table)]
    pool = pool.to(DEV)
    want = pk.focus_tree_attention(pool, 0, *args, max_rows=7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [pk.focus_tree_attention(pool, 0, *args, max_rows=7, stream=side) for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


# -- a context -----------------------------------------------------------------------------------------
def test_a_prefilled_context_is_forked():
    """Three samples of one prompt: its full pages are shared, the page it ends in is copied, and every sample's steps are those of a sequence that was prefilled alone."""
    pk = _pk()
    from paper_2601_23278_amd import runner
    wl = fi.workload("c1_tiny", batch=1, prefix_lo=40, prefix_hi=40)       # 40 tokens in pages of 16, blocks of 16
    alone = runner.open_session(wl, DEV)
    cfg = runner.config_from_workload(wl, max_batch=3, max_prefix_len=40, n_pages=14)
    embed, lm_head, norm, layers = alone.weights
    pool = torch.full((wl.n_layers, 14, 2, wl.n_kv_heads, wl.page_size, wl.head_dim), math.nan, device=DEV)
    f = pk.Focus(cfg, embed, lm_head, norm, layers, pool)
    refs, table = torch.zeros(14, dtype=torch.int32, device=DEV), torch.full((1, 4), -1, dtype=torch.int32, device=DEV)
    lens = i32([40]).to(DEV)
    assert int(pk.focus_kv_reserve(lens, 16, table, refs, 16).sum()) == 0
    prompt = wl.prompt_tokens(wl.prefix_lens())
    f.focus_prefill_kv([40], table.tolist(), prompt)
    lens, table, lack = pk.focus_kv_fork(pool, i32([0, 0, 0]).to(DEV), lens, table, refs)
    assert int(pk.focus_kv_reserve(lens, 16, table, refs, 16).sum()) == 0 and not bool(lack.any())
    rows = table.tolist()
    assert rows[0][:2] == rows[1][:2] == rows[2][:2] and len({r[2] for r in rows}) == 3 and refs[rows[0][0]] == 3
    f.focus_prefill_kv([40] * 3, rows, None)
    B, n = wl.block_size, 3
    for _ in range(4):
        got, want = torch.zeros(n, B, dtype=torch.int32, device=DEV), torch.zeros(1, B, dtype=torch.int32, device=DEV)
        h3, h1 = torch.zeros(n * B, wl.hidden, device=DEV), torch.zeros(B, wl.hidden, device=DEV)
        c3, c1 = torch.zeros(n + 1, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
        f.focus_step(n, out=pk.make_step_out(tokens=got, hidden_packed=h3, cu_seqlens=c3))
        alone.focus.focus_step(1, out=pk.make_step_out(tokens=want, hidden_packed=h1, cu_seqlens=c1))
        torch.cuda.synchronize()
        assert all(got[i].tolist() == want[0].tolist() for i in range(n))
        rows_1 = int(c1[1])
        for i in range(n):
            mine = h3[int(c3[i]):int(c3[i + 1])]
            assert mine.shape[0] == rows_1
            # fp32 model, other orders of the same sums
            assert float((mine - h1[:rows_1]).abs().max()) <= 1e-4 * float(h1[:rows_1].abs().max())
    f.focus_free()
    alone.focus.focus_free()


def test_beam_search_with_bf16_cache():
    pk, gen = _pk(), torch.Generator().manual_seed(38)
    n, beams, H, D, P = 2, 4, 2, 64, 16
    embed = torch.randn(60, 3 * H * D, generator=gen).to(torch.bfloat16).to(DEV)
    refs, table = torch.zeros(90, dtype=torch.int32, device=DEV), torch.full((n * beams, 6), -1, dtype=torch.int32, device=DEV)
    lens = torch.zeros(n * beams, dtype=torch.int32, device=DEV)
    pool = torch.full((1, 90, 2, H, P, D), math.nan, dtype=torch.bfloat16, device=DEV)
    scores, lens, table, _ = beam_search(pk, gen, embed, pool, refs, table, lens, 40, n, beams, H, D, P)
    assert bool(torch.isfinite(scores).all()) and lens.tolist() == [40] * (n * beams)
    assert bool((scores[:, :-1] >= scores[:, 1:]).all())


# -- what the binding refuses ----------------------------------------------------------------------------
def test_the_binding_refuses():
    pk = _pk()
    pool = torch.zeros(1, 4, 2, 2, 16, 64, device=DEV)
    cu, lens, table = i32([0, 2]).to(DEV), i32([3]).to(DEV), i32([[0, 1]]).to(DEV)
    q, k = torch.zeros(2, 256, device=DEV), torch.zeros(2, 128, device=DEV)
    logits, scores = torch.zeros(4, 10, device=DEV), torch.zeros(2, 2, device=DEV)
    refs, one = torch.zeros(4, dtype=torch.int32, device=DEV), i32([0]).to(DEV)
    bad = [
        lambda: pk.focus_kv_append(pool[0], 0, k, k, cu, lens, table), lambda: pk.focus_kv_append(pool.half(), 0, k, k, cu, lens, table),
        lambda: pk.focus_kv_append(pool.transpose(4, 5), 0, k, k, cu, lens, table), lambda: pk.focus_kv_append(pool, 1, k, k, cu, lens, table),
        lambda: pk.focus_kv_append(pool, 0, k[:, :64], k, cu, lens, table), lambda: pk.focus_kv_append(pool, 0, k.bfloat16(), k, cu, lens, table),
        lambda: pk.focus_kv_append(pool, 0, k, k[:1], cu, lens, table), lambda: pk.focus_kv_append(pool, 0, k, k, lens, lens, table),
        lambda: pk.focus_kv_append(pool, 0, k, k, cu, cu, table), lambda: pk.focus_kv_append(pool, 0, k, k, cu.long(), lens, table),
        lambda: pk.focus_kv_append(pool, 0, k, k, cu, lens, table.t()), lambda: pk.focus_kv_append(pool, 0, k, k.cpu(), cu, lens, table),
        lambda: pk.focus_tree_attention(pool, 0, q[:, :100], cu, lens, table), lambda: pk.focus_tree_attention(pool, 0, q[:, :192], cu, lens, table),
        lambda: pk.focus_tree_attention(pool, 0, q.bfloat16(), cu, lens, table), lambda: pk.focus_tree_attention(pool, 0, q, cu, lens, table, seen=cu),
        lambda: pk.focus_tree_attention(pool, 0, q, cu, lens, table, seen=torch.zeros(3, dtype=torch.int64, device=DEV)),
        lambda: pk.focus_tree_attention(pool, 0, q, cu, lens, table, seen=torch.zeros(2, 17, dtype=torch.int64, device=DEV)),
        lambda: pk.focus_tree_attention(pool, 0, q, cu, lens, table, out=q[:1]), lambda: pk.focus_tree_attention(pool, 0, q, cu, lens, table, scale=math.nan),
        lambda: pk.focus_tree_attention(pool, 0, q, cu, lens, table, max_rows=-1), lambda: pk.focus_tree_attention(pool, 2 ** 40, q, cu, lens, table),
        lambda: pk.focus_tree_attention(pool, 0, q, cu, lens, table, workspace=torch.zeros(64)),
        lambda: pk.focus_kv_compact(pool, lens, cu, one, table, i32([[0], [1]]).to(DEV)), lambda: pk.focus_kv_compact(pool, cu, cu, one, table),
        lambda: pk.focus_kv_compact(pool, lens, cu, one.view(1, 1), table), lambda: pk.focus_kv_compact(pool, lens, cu, one.long(), table),
        lambda: pk.focus_kv_fork(pool, one, lens, table, refs[:3]), lambda: pk.focus_kv_fork(pool, one, cu, table, refs), lambda: pk.focus_kv_fork(pool, one.long(), lens, table, refs),
        lambda: pk.focus_kv_fork(pool, one, lens, table, refs, new_table=table), lambda: pk.focus_kv_fork(pool, one, lens, table, refs, new_table=i32([[0]]).to(DEV)),
        lambda: pk.focus_kv_fork(pool, one, lens, table, refs, workspace=torch.zeros(4, dtype=torch.uint8, device=DEV)),
        lambda: pk.focus_kv_reserve(lens, -1, table, refs, 16), lambda: pk.focus_kv_reserve(lens, 1, table, refs, 12), lambda: pk.focus_kv_reserve(cu, 1, table, refs, 16),
        lambda: pk.focus_kv_reserve(lens, 2 ** 33, table, refs, 16), lambda: pk.focus_kv_reserve(lens, 1, table, refs.view(2, 2), 16),
        lambda: pk.focus_beam_select(logits, scores[:1], 2), lambda: pk.focus_beam_select(logits, scores, 0), lambda: pk.focus_beam_select(logits, scores, 65),
        lambda: pk.focus_beam_select(logits, scores.double(), 2), lambda: pk.focus_beam_select(logits.half(), scores, 2), lambda: pk.focus_beam_select(logits.t(), scores, 2),
        lambda: pk.focus_beam_select(logits, scores, 2, done=scores), lambda: pk.focus_beam_select(logits, scores, 2, rows=one),
        lambda: pk.focus_beam_select(logits, scores, 2, workspace=torch.zeros(8, dtype=torch.uint8, device=DEV)), lambda: pk.focus_beam_select(logits.view(-1), scores, 2),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(pk.FocusError):
            call()
            pytest.fail("call %d was not refused" % i)
