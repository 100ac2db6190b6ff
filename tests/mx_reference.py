"""Plain 64-bit forms of the expert router and of the MXFP4 operators, on the CPU, written from their definitions (include/focus.h)."""
import math

import numpy as np
import torch

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def scores_of(logits, kind):
    """Scores of one row of float64 logits; NaN has score 0."""
    l = np.asarray(logits, dtype=np.float64)
    ok = ~np.isnan(l)
    s = np.zeros(len(l))
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            s[ok] = 1.0 / (1.0 + np.exp(-l[ok]))
        return s
    top = np.max(l[ok]) if ok.any() else -np.inf
    if top == -np.inf:
        return s
    if top == np.inf:
        s[ok] = (l[ok] == np.inf).astype(np.float64)
    else:
        s[ok] = np.exp(l[ok] - top)
    return s / s.sum()


def route_row(logits, bias, kind, groups, kept, top, k, renorm, scale, forced=None):
    """(experts, weights) of one row."""
    s = scores_of(logits, kind)
    E = len(s)
    if forced is None:
        c = s + (0.0 if bias is None else np.asarray(bias, dtype=np.float64))
        c = [-math.inf if math.isnan(logits[e]) or math.isnan(c[e]) else float(c[e]) for e in range(E)]
        size = E // groups
        values = []
        for g in range(groups):
            v = sum(sorted(c[g * size:(g + 1) * size], reverse=True)[:top])
            values.append(-math.inf if math.isnan(v) else v)
        best = sorted(range(groups), key=lambda g: (-values[g], g))[:kept]
        pool = [e for e in range(E) if e // size in best]
        forced = sorted(pool, key=lambda e: (-c[e], e))[:k]
    total = sum(s[e] for e in forced)
    scale = float(np.float32(scale))
    return list(forced), [(scale * s[e] / total if total > 0 else 0.0) if renorm else scale * s[e] for e in forced]


def quantize(x):
    """Codes (one per element, uint8) and scales of float64 rows [rows, cols]; a row's last block is filled with zeros."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    blocks = -(-cols // 32)
    p = np.zeros((rows, blocks * 32))
    p[:, :cols] = x
    p = p.reshape(rows, blocks, 32)
    codes = np.zeros(p.shape, dtype=np.uint8)
    scales = np.zeros((rows, blocks), dtype=np.uint8)
    for r in range(rows):
        for b in range(blocks):
            v = p[r, b]
            if not np.all(np.isfinite(v)):
                scales[r, b] = 255
                continue
            most = np.max(np.abs(v))
            power = -127 if most == 0 else min(127, max(-127, math.frexp(most)[1] - 1 - 2))
            scales[r, b] = power + 127
            for i in range(32):
                t = abs(v[i]) / 2.0 ** power
                near = min(range(8), key=lambda q: (abs(t - GRID[q]), q & 1))      # a tie goes to the even mantissa
                codes[r, b, i] = near + (8 if math.copysign(1.0, v[i]) < 0 else 0)
    return codes.reshape(rows, blocks * 32), scales


def pack(codes):
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def values(packed, scales):
    """float64 values of packed codes [..., K / 2] and scales [..., K / 32], torch uint8 tensors."""
    q = torch.stack([packed & 15, packed >> 4], dim=-1).flatten(-2).long()
    grid = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64)
    s = torch.exp2(scales.double() - 127.0)
    s[scales == 255] = float("nan")
    return grid[q] * s.repeat_interleave(32, dim=-1)


def random_mx(gen, *shape, spread=3):
    """Random codes and scales of a matrix [..., K]; scales over 2^(-spread) .. 2^spread times 2^-4."""
    codes = torch.randint(0, 256, (*shape[:-1], shape[-1] // 2), generator=gen, dtype=torch.uint8)
    scales = torch.randint(123 - spread, 124 + spread, (*shape[:-1], shape[-1] // 32), generator=gen, dtype=torch.uint8)
    return codes, scales


def experts(x, gate_up, down, picks, weights):
    """(out, bound of the error) in float64: x [rows, hidden], values of gate_up [E, 2 F, hidden] and down [E, hidden, F].

    The bound counts, for a kernel that sums in fp32 and rounds the inner activations to bf16: K additions of at most half an ulp each, doubled for
    matrix units that truncate; SiLU's slope (at most 1.1) times the gate's error; its exponential (error grows with its argument); half
    a bf16 step of the activation."""
    rows, hidden = x.shape
    E, two_f, _ = gate_up.shape
    F = two_f // 2
    out, bound = torch.zeros(rows, hidden, dtype=torch.float64), torch.zeros(rows, hidden, dtype=torch.float64)
    for r in range(rows):
        for j in range(picks.shape[1]):
            e, w = int(picks[r, j]), float(weights[r, j])
            if not 0 <= e < E:
                continue
            both, size = gate_up[e] @ x[r], gate_up[e].abs() @ x[r].abs()
            g, u = both[:F], both[F:]
            silu = g / (1 + torch.exp(-g))
            act = silu * u
            e_act = (hidden * 2.0 ** -23) * (1.1 * size[:F] * u.abs() + silu.abs() * size[F:]) + act.abs() * (2.0 ** -8 + 2.0 ** -20 * (1 + g.abs()))
            out[r] += w * (down[e] @ act)
            bound[r] += abs(w) * (down[e].abs() @ (e_act + act.abs() * (F * 2.0 ** -23 + 4 * 2.0 ** -24 * picks.shape[1])))
    return out, bound
