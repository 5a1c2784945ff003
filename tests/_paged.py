"""Plain 64-bit restatement (CPU) of the rotary and paged-cache operators, and error bounds by counting roundings."""
import math

import torch

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step, relative


def frequencies(dims, base, factor=1.0, trained=0.0, low=1.0, high=32.0):
    f = torch.tensor([base ** (-2.0 * i / dims) for i in range(dims // 2)], dtype=torch.float64)
    g = torch.zeros_like(f)
    if trained:
        g = ((trained * f / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
    return f * (g + (1 - g) / factor)


def rotate(x, positions, freq, layout, weight=None, eps=1e-6, magnitude=1.0):
    """x [n, H, d] (any type), positions [n] -> 64 bits.  freq None: the norm alone."""
    y = x.double()
    if weight is not None:
        y = y * weight.double() / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
    if freq is None:
        return y
    rd = 2 * len(freq)
    ang = positions.double()[:, None, None] * freq
    c, s = magnitude * ang.cos(), magnitude * ang.sin()
    ia = torch.arange(rd // 2) if layout == "half" else torch.arange(0, rd, 2)
    ib = ia + rd // 2 if layout == "half" else ia + 1
    out = y.clone()
    out[..., ia] = y[..., ia] * c - y[..., ib] * s
    out[..., ib] = y[..., ib] * c + y[..., ia] * s
    return out


def rotate_bound(want, dtype, normed):
    """One rounding to the type; in 32 bits: cos, sin, two products and a sum (5 roundings of values up to the row's largest, 2 of them
    in a pair), with the norm a sum of squares in 16 + 3 steps, its root, its reciprocal and two products ahead: 32 in all."""
    top = want.abs().amax(-1, keepdim=True) * 2 ** 0.5
    return HALF[dtype] * want.abs() + (40 if normed else 8) * 2.0 ** -24 * top + 1e-30


def key_rows(table_row, n, page, pages, pages_per_seq):
    """(key, page, row) of the keys 0 .. n - 1 that lie in pages that exist."""
    out = []
    for j in range(min(n, page * pages_per_seq)):
        p = int(table_row[j // page])
        if 0 <= p < pages:
            out.append((j, p, j % page))
    return out


def attend(q, K, V, starts, lens, table, window=0, scale=None):
    """q [T, Hq, d]; K, V [pages, Hkv, P, d]; lists / CPU tensors.  Returns (out, lse, sum of weights * |V|, largest sum of |q k| scale),
    in 64 bits; rows of tokens that belong to no sequence are NaN."""
    T, Hq, d = q.shape
    pages, Hkv, P, _ = K.shape
    G = Hq // Hkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    out = torch.full((T, Hq, d), math.nan, dtype=torch.float64)
    mass, absq = out.clone(), torch.zeros((T, Hq), dtype=torch.float64)
    lse = torch.full((T, Hq), math.nan, dtype=torch.float64)
    for s in range(len(lens)):
        a, b = int(starts[s]), min(int(starts[s + 1]), T)
        if a >= b:
            continue
        n, new = max(int(lens[s]), 0), int(starts[s + 1]) - a
        rows = key_rows(table[s], n, P, pages, table.shape[1])
        j = torch.tensor([r[0] for r in rows], dtype=torch.long)
        pg, rw = torch.tensor([r[1] for r in rows], dtype=torch.long), torch.tensor([r[2] for r in rows], dtype=torch.long)
        pos = torch.arange(n - new, n - new + (b - a))
        seen = j[None] <= pos[:, None]
        if window:
            seen &= j[None] > pos[:, None] - window
        for h in range(Hkv):
            k, v = K[pg, h, rw].double(), V[pg, h, rw].double()
            for g in range(h * G, h * G + G):
                x = q[a:b, g].double()
                for i in range(b - a):
                    m = seen[i]
                    if not bool(m.any()):
                        out[a + i, g], mass[a + i, g], lse[a + i, g] = 0, 0, -math.inf
                        continue
                    ki, vi = k[m], v[m]
                    logits = (ki * x[i]).sum(-1) * scale
                    w = torch.softmax(logits, 0)
                    out[a + i, g] = (w[:, None] * vi).sum(0)
                    mass[a + i, g] = (w[:, None] * vi.abs()).sum(0)
                    lse[a + i, g] = torch.logsumexp(logits, 0)
                    absq[a + i, g] = ((ki * x[i]).abs().sum(-1) * scale).max()
    return out, lse, mass, absq


def attend_bounds(want, lse, mass, absq, dtype, d, weights_rounded):
    """Bounds of out and lse.  A logit is off by d roundings of partial sums of size absq, two by the scaling and the reference (all in
    32 bits), hence a weight by twice as much relative (it and its sum); the sums over keys add a rounding of 32 bits for each level
    (64 granted).  bf16 weights (weights_rounded) are off by half a step of bf16, the output by half a step of its type."""
    logit = (d + 4) * 2.0 ** -24 * absq[..., None]
    rel = 2 * logit + 64 * 2.0 ** -24 + (HALF[torch.bfloat16] if weights_rounded else 0.0)
    top = want.abs().nan_to_num(0.0, 0.0, 0.0)
    return rel * mass + HALF[dtype] * (top + rel * mass) + 1e-30, logit[..., 0] + 64 * 2.0 ** -24 * (1 + lse.abs().nan_to_num(0.0, 0.0, 0.0))
