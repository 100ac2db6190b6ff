"""Calls of the expert router and the MXFP4 operators at the edges of what their documentation allows, against plain 64-bit forms (mx_reference.py)."""
import gc
import math
import weakref

import pytest
import torch

import mx_reference as ref
from test_gpu_mx import DEV, MATRICES, _pk, check_route, experts_case, gpu, product_bound, small

pytestmark = pytest.mark.gpu


# -- router -----------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("a", [10.0, 100.0, 1e3, 1e4])
@pytest.mark.parametrize("spread", [1.0, 0.02])
def test_groups_whose_biases_cancel(kind, a, spread):
    """A group's two choices are rounded at the size of their biases, however small their sum is: groups closer than that, all of them so or every other."""
    E, G = 128, 64
    gen = torch.Generator().manual_seed(int(a))
    l = torch.randn(48, E, generator=gen) * spread
    both = torch.tensor([a, -a]).repeat(G)
    half = both.clone().view(G, 2)
    half[1::2] = 0.0
    for bias in (both, half.view(-1)):
        check_route(l, bias, kind, G, 8, 2, 8, 1, 1.0)


def test_scores_that_32_bits_do_not_hold():
    """An expert whose score is too small for 32 bits still comes before those with none at all; scores near the smallest numbers keep their order."""
    inf = float("inf")
    l = torch.full((8, 16), -inf)
    l[0, [1, 3, 4]] = torch.tensor([0.0, -1.0, -150.0])
    l[1, [15, 7, 14]] = torch.tensor([-400.0, 5.0, -300.0])
    l[2, [2, 9]] = torch.tensor([3e38, 2e38])
    l[3, 5:] = -110.0 - torch.arange(11) * 0.25
    l[3, 8] = 0.0
    l[4] = torch.tensor([0.0, -150.0]).repeat(8)
    l[5, 12] = 88.0
    l[5, [10, 11]] = torch.tensor([-61.9, -62.0])
    l[6, [0, 2, 3]] = torch.tensor([-150.0, -140.0, 0.0])
    l[7, [9, 11, 15]] = torch.tensor([-500.0, -499.0, 1.0])
    for kind in ("softmax", "sigmoid"):
        for renorm in (0, 1):
            for k in (2, 3, 5, 16):
                check_route(l, None, kind, 1, 1, 1, k, renorm, 1.0)
                check_route(l, torch.zeros(16), kind, 4, 2, 2, min(k, 8), renorm, 1.0)
    gen = torch.Generator().manual_seed(5)
    l = -87.0 - 17.0 * torch.rand(60, 64, generator=gen)
    l[:, 1::2] = l[:, ::2] + torch.randint(-2, 3, (60, 32), generator=gen) * 2.0 ** -17      # neighbours in fp32
    l[:, 63] = 0.0
    for kind in ("softmax", "sigmoid"):
        check_route(l, None, kind, 1, 1, 1, 32, 0, 1.0)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k", [(64, 28), (200, 20), (512, 32)])
def test_a_score_that_its_bias_cancels_against_small_scores(kind, E, k):
    """One expert's score of 0.9 is known to some 1e-7 in 32 bits, and so is its choice, 1e-6 by its bias; the small scores around it lie 2e-8 apart and are
    known far better.  Whether it is among the picks, and where, is not a matter of its neighbours' distances alone."""
    gen = torch.Generator().manual_seed(E)
    rows = 160
    w = torch.empty(rows, E, dtype=torch.float64)
    w[:, 1:9] = 0.0125 * (1 + 0.01 * torch.arange(8, dtype=torch.float64))
    small = 1e-6 + 2e-8 * torch.arange(E - 9, dtype=torch.float64) * (1 + 0.1 * torch.rand(rows, E - 9, generator=gen, dtype=torch.float64))
    w[:, 9:] = small[:, torch.randperm(E - 9, generator=gen)]
    last = float(small.sort(dim=1, descending=True).values[:, k - 9].mean())       # about the last of the k
    w[:, 0] = 0.9 + 3e-7 * torch.randn(rows, generator=gen, dtype=torch.float64)
    bias = torch.zeros(E)
    bias[0] = last - 0.9
    logits = torch.log(w) if kind == "softmax" else torch.log(w / (1 - w))
    if kind == "softmax":
        bias[0] = last - float((w[:, 0] / w.sum(1)).mean())
    check_route(logits.float(), bias, kind, 1, 1, 1, k, 1, 1.0)


# -- products ---------------------------------------------------------------------------------
@pytest.mark.parametrize("a_type", ["bf16", "mx4"])
@pytest.mark.parametrize("k", [96, 512])
def test_gemm_with_the_smallest_scales_against_large_rows(a_type, k):
    """Weights from 2^-128 on, most of them below the smallest normal number, times rows around 2^100: normal results, to which every weight counts."""
    pk, _ = _pk()
    m, n = 40, 140
    gen = torch.Generator().manual_seed(k)
    codes = torch.randint(0, 256, (n, k // 2), generator=gen, dtype=torch.uint8)
    scales = torch.randint(0, 4, (n, k // 32), generator=gen, dtype=torch.uint8)
    scales[:20], scales[20:40] = 0, 1
    wv = ref.values(codes, scales)
    if a_type == "bf16":
        a = (torch.randn(m, k, generator=gen) * 2.0 ** 100).to(torch.bfloat16)
        av, ga = a.double(), a.to(DEV)
    else:
        am = ref.random_mx(gen, m, k)
        am[1].add_(100)
        av, ga = ref.values(*am), gpu(*am)
    c = pk.focus_mx_gemm(ga, gpu(codes, scales), torch.empty(m, n, device=DEV)).cpu().double()
    want = av @ wv.t()
    assert float(want.abs().median()) > 2.0 ** -40                  # the bound's own smallest numbers are nothing beside them
    assert bool(((c - want).abs() <= product_bound(av, wv, torch.float32)).all())


@pytest.mark.parametrize("scale", [251, 252, 253, 254])
def test_gemm_with_the_largest_scales(scale):
    """Rows in MXFP4: every weight counts with its value.  Rows in bf16: weights of 2^128 and more, beyond bf16, count as infinite; those that the quantiser writes
    (scales up to 252) are smaller."""
    pk, _ = _pk()
    n, k = 16, 64
    codes = torch.zeros(n, k // 2, dtype=torch.uint8)
    codes[:, 5] = torch.arange(n, dtype=torch.uint8) << 4            # element 11 of row c is code c, all others are zero
    w = codes, torch.full((n, k // 32), scale, dtype=torch.uint8)
    value = ref.values(*w)[:, 11]
    a = torch.zeros(3, k)
    a[0, 11], a[1, 11], a[2, 11] = 2.0 ** -20, -1.5, 2.0 ** -125
    want = a.double()[:, 11:12] * value
    want = torch.where(want.abs() < 2.0 ** 128, want, torch.sign(want) * math.inf)
    got = pk.focus_mx_gemm(pk.focus_mx_quantize(a.to(DEV)), gpu(*w), torch.empty(3, n, device=DEV)).cpu().double()
    assert torch.equal(got, want)
    want = torch.where(value.abs() < 2.0 ** 128, want, torch.sign(a[:, 11:12].double()) * torch.sign(value) * math.inf)
    got = pk.focus_mx_gemm(a.to(torch.bfloat16).to(DEV), gpu(*w), torch.empty(3, n, device=DEV)).cpu().double()
    assert torch.equal(got, want)
    top = torch.full((1, 32), torch.finfo(torch.float32).max)
    for dtype in (torch.float32, torch.bfloat16):
        assert pk.focus_mx_quantize(top.to(dtype).clamp(max=torch.finfo(dtype).max).to(DEV))[1].tolist() == [[252]]


# -- inside a context -------------------------------------------------------------------------
@pytest.mark.parametrize("E,k,batch,ratio,kept,hint", [
    (64, 4, 5, 0.25, 0x00010001, 10),      # ten rows and a hint of ten: tiles of 32 rows, their list behind the counts
    (64, 4, 5, 0.25, 0xFFFFFFFF, 8),       # the same launches with 160 rows in them
    (300, 8, 5, 0.25, 0xFFFFFFFF, 5),      # 1280 entries of 300 experts where 40 were expected
    (64, 4, 2, 0.25, 0xFFFF0FF1, 0),       # 64 rows and no hint: still 32-row tiles
    (48, 2, 1, 1 / 32, None, 0)])          # one row a step, whose counts leave no room for the tiles behind them
def test_context_in_tiles_of_32_rows(E, k, batch, ratio, kept, hint):
    """Few rows an expert, as the row hint has it, which need not be true: every row's residual stream against a context on the same values in bf16, and against
    one whose experts give nothing, so that a row that lost an expert shows.  Only the experts differ, so that all select the same positions.  The same values are
    summed in another order and rounded to bf16 between kernels: the tolerance of the bf16 model's parity tests, of what the experts give."""
    pk, runner = _pk()
    wl = small(n_experts=E, experts_per_token=k, batch=batch, keep_ratio=ratio)
    n = wl.batch
    forced = None if kept is None else torch.full((n,), kept, dtype=torch.int64, device=DEV)
    routes = torch.tensor(wl.route_override(n), dtype=torch.int32, device=DEV)
    got = {}
    for which in ("bf16", "mx", "none"):
        sess = runner.open_session(wl, DEV)
        layers = []
        for w in sess.weights[3]:
            pairs = {}
            for name in MATRICES[2:4]:
                if name in w:
                    t = w[name]
                    c, s = pk.focus_mx_quantize(t.reshape(-1, t.shape[-1]))
                    pk.focus_mx_dequantize(c, s, t.view(-1, t.shape[-1]))
                    pairs[name] = (c.view(*t.shape[:-1], -1) * (which == "mx"), s.view(*t.shape[:-1], -1))
            layers.append(pairs)
        if which != "bf16":
            sess.focus.focus_set_mx_weights(layers)
        sess.focus.focus_set_route_override(routes)
        if hint:
            sess.focus.focus_set_row_hint(hint, wl.block_size)
        hidden = torch.zeros(n * wl.block_size, wl.hidden, device=DEV)
        cu = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
        sess.focus.focus_step(n, out=pk.make_step_out(hidden_packed=hidden, cu_seqlens=cu), keep_override=forced)
        torch.cuda.synchronize()
        got[which] = hidden[:int(cu[n])].double().cpu()
        sess.focus.focus_free()
    assert got["mx"].shape[0] == n * (1 if kept is None else bin(kept).count("1"))
    given = (got["bf16"] - got["none"]).norm(dim=1)
    assert bool((given > 0).all()) and bool(((got["mx"] - got["bf16"]).norm(dim=1) <= 2e-2 * given).all()), float(((got["mx"] - got["bf16"]).norm(dim=1) / given).max())


def expert_pairs(pk, E, ffn, hidden):
    up, down = pk.focus_mx_quantize(torch.ones(E * 2 * ffn, hidden, device=DEV)), pk.focus_mx_quantize(torch.ones(E * hidden, ffn, device=DEV))
    return dict(w_expert_gate_up=tuple(t.view(E, 2 * ffn, -1) for t in up), w_expert_down=tuple(t.view(E, hidden, -1) for t in down))


def test_a_context_keeps_what_it_borrows():
    """The caller's lists and dicts may change or go once a setter has returned; a refused call keeps what was there."""
    pk, runner = _pk()
    sess = runner.open_session(small(), DEV)
    f, E = sess.focus, 16
    layers = [{}, expert_pairs(pk, E, 128, 512), expert_pairs(pk, E, 128, 512)]
    biases = [torch.zeros(E, device=DEV) for _ in range(3)]
    router = pk.focus_router(n_experts=E, experts_per_token=4, score=1, n_groups=4, groups_kept=2, group_top=2, renormalize=1, route_scale=1.0)
    tensors = [weakref.ref(t) for l in layers for pair in l.values() for t in pair] + [weakref.ref(b) for b in biases]
    f.focus_set_mx_weights(layers)
    f.focus_set_router(router, biases)
    layers[1].clear()
    layers.clear()
    biases.clear()
    gc.collect()
    assert len(tensors) == 11 and all(t() is not None for t in tensors)
    with pytest.raises(pk.FocusError):
        f.focus_set_mx_weights([{}])
    with pytest.raises(pk.FocusError):
        f.focus_set_router(router, [None])
    gc.collect()
    assert all(t() is not None for t in tensors)
    f.focus_step(sess.wl.batch)
    torch.cuda.synchronize()
    f.focus_set_mx_weights(None)
    f.focus_set_router(None)
    gc.collect()
    assert all(t() is None for t in tensors)
    f.focus_free()


def test_setters_refuse_names_that_no_matrix_has():
    pk, runner = _pk()
    sess = runner.open_session(small(), DEV)
    good = expert_pairs(pk, 16, 128, 512)
    for name in ("w_expert_gateup", "w_qkv", "gate_up"):
        with pytest.raises(pk.FocusError):
            sess.focus.focus_set_mx_weights([{}, dict(good, **{name: good["w_expert_down"]}), good])
    sess.focus.focus_free()


def test_context_refuses_mx_matrices_wider_than_its_kernels_take():
    """K, and the distance of rows, of at most 2^22, as for the product without a context.  Nothing is read: the context is never run."""
    pk, _ = _pk()
    for ffn, ok in ((2 ** 22, True), (2 ** 22 + 32, False)):
        cfg = pk.focus_config(n_layers=2, hidden=64, n_q_heads=1, n_kv_heads=1, head_dim=64, ffn=ffn, vocab=64, dtype=pk.FOCUS_BF16, rms_eps=1e-6, rope_base=1e4,
                              block_size=1, mask_token_id=63, max_batch=1, max_prefix_len=8, page_size=16, n_pages=1, evict_layer=1, maxpool_k=3, budget_mode=1,
                              keep_ratio=1.0, conf_threshold=0.9)
        one = torch.zeros(64, dtype=torch.bfloat16, device=DEV)
        pool = torch.zeros(pk.focus_kv_pool_bytes(cfg), dtype=torch.uint8, device=DEV)
        f = pk.Focus(cfg, one, one, one, [{n: one for n in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down")}] * 2, pool)
        up, down = (tuple(torch.empty(r, c // per, dtype=torch.uint8, device=DEV) for per in (2, 32)) for r, c in ((2 * ffn, 64), (64, ffn)))
        if ok:
            f.focus_set_mx_weights([dict(w_gate_up=up, w_down=down)] * 2)
        else:
            with pytest.raises(pk.FocusError, match="layer 0"):
                f.focus_set_mx_weights([dict(w_gate_up=up, w_down=down)] * 2)
        f.focus_free()


def test_weights_of_scores_below_the_smallest_normal_number():
    """Biases pick experts whose scores 32 bits hold with few bits or not at all, beside others that they do hold: the quotients count in full."""
    for rows, E, k, seed, size in ((40, 32, 20, 1, 100.0), (40, 16, 7, 2, 60.0), (7, 256, 22, 3, 30.0)):
        gen = torch.Generator().manual_seed(seed)
        l = torch.randn(rows, E, generator=gen) * size
        check_route(l, torch.randn(E, generator=gen) * 100, "softmax", 1, 1, 1, k, 1, 2.5)
        check_route(l, torch.randn(E, generator=gen) * 100, "sigmoid", 4, 3, 2, min(k, 3 * E // 4), 1, 2.5)
