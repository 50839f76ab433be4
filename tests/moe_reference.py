"""The mixture-of-experts operators and the AdamW step in 64 bits on the CPU, from their definitions: loops over tokens and
groups, no code of the package."""
import math

import numpy as np
import torch

E4M3, E5M2 = torch.float8_e4m3fn, torch.float8_e5m2
FMAX = {E4M3: 448.0, E5M2: 57344.0}


def route(logits, k, renorm):
    """dict of gates (float64), experts, offsets, row_token, slot_row from logits [T, E] (any float tensor)."""
    x = logits.double().numpy()
    T, E = x.shape
    gates, experts = np.zeros((T, k)), np.full((T, k), -1)
    for t in range(T):
        can = [e for e in range(E) if x[t, e] > -math.inf]      # (not NaN either)
        chosen = sorted(can, key=lambda e: (-x[t, e], e))[:k]
        if not chosen:
            continue
        top = x[t, chosen[0]]
        ex = {e: math.exp(x[t, e] - top) for e in can}
        total = sum(ex[e] for e in (chosen if renorm else can))
        for j, e in enumerate(chosen):
            experts[t, j], gates[t, j] = e, ex[e] / total
    slots = sorted((experts[t, j], t, j) for t in range(T) for j in range(k) if experts[t, j] >= 0)
    row_token, slot_row, counts = np.full(T * k, -1), np.full((T, k), -1), np.zeros(E, dtype=np.int64)
    for r, (e, t, j) in enumerate(slots):
        row_token[r], slot_row[t, j] = t, r
        counts[e] += 1
    return {"gates": gates, "experts": experts, "offsets": np.concatenate([[0], np.cumsum(counts)]), "row_token": row_token, "slot_row": slot_row}


def route_bwd(logits, dgates, gates, experts, renorm):
    x = logits.double().numpy()
    T, E = x.shape
    out = np.zeros((T, E))
    for t in range(T):
        inner = sum(dgates[t, j] * gates[t, j] for j in range(experts.shape[1]) if experts[t, j] >= 0)
        d = {experts[t, j]: dgates[t, j] for j in range(experts.shape[1]) if experts[t, j] >= 0}
        g = {experts[t, j]: gates[t, j] for j in range(experts.shape[1]) if experts[t, j] >= 0}
        can = [e for e in range(E) if x[t, e] > -math.inf]
        if not d:
            continue
        total = sum(math.exp(x[t, e] - max(x[t, can])) for e in can)
        for e in can:
            p = g.get(e, 0.0) if renorm else math.exp(x[t, e] - max(x[t, can])) / total
            out[t, e] = p * (d.get(e, 0.0) - inner)
    return out


def values(x, dim, fmt, pow2):
    """x behind its codes (float64), one scale per line along dim."""
    x = x.float()
    s = (FMAX[fmt] / x.abs().amax(dim, keepdim=True).double().clamp(min=1e-12)).float()
    if pow2:
        s = (s.view(torch.int32) & -0x800000).view(torch.float32)
    return (x * s).clamp(-FMAX[fmt], FMAX[fmt]).to(fmt).double() / s.double()


def product(a, b):
    """a b^T and the same of the magnitudes, which bounds what the order of the sums does."""
    return a @ b.T, a.abs() @ b.abs().T


def rows_of(x, row_token):
    """x's rows by token, zeros where there is none."""
    t = row_token.long()
    return torch.where(((t >= 0) & (t < x.shape[0]))[:, None], x[t.clamp(0, max(x.shape[0] - 1, 0))], torch.zeros((), dtype=x.dtype))


def grouped_fwd(xr, w, offsets, fmt_x, fmt_w, pow2):
    """(Y, magnitudes) from rows xr [M, K]."""
    y = torch.zeros((xr.shape[0], w.shape[1]), dtype=torch.float64)
    s = torch.zeros_like(y)
    for e in range(w.shape[0]):
        at = slice(int(offsets[e]), int(offsets[e + 1]))
        if at.stop > at.start:
            y[at], s[at] = product(values(xr[at], 1, fmt_x, pow2), values(w[e], 1, fmt_w, pow2))
    return y, s


def grouped_bwd(dy, xr, w, offsets, fmt_dy, fmt_x, fmt_w, pow2):
    """((dX, magnitudes), (dW, magnitudes))"""
    dx = torch.zeros((dy.shape[0], w.shape[2]), dtype=torch.float64)
    dw = torch.zeros(w.shape, dtype=torch.float64)
    sx, sw = torch.zeros_like(dx), torch.zeros_like(dw)
    for e in range(w.shape[0]):
        at = slice(int(offsets[e]), int(offsets[e + 1]))
        if at.stop > at.start:
            dx[at], sx[at] = product(values(dy[at], 1, fmt_dy, pow2), values(w[e], 0, fmt_w, pow2).T)
            dw[e], sw[e] = product(values(dy[at], 0, fmt_dy, pow2).T, values(xr[at], 0, fmt_x, pow2).T)
    return (dx, sx), (dw, sw)


def assert_product(got, want, size):
    """A bfloat16 result against 64 bits: half a bfloat16 step of the value, and 2^-13 of the sum of the products' magnitudes for
    the order of the fp32 sums and the matrix instruction's alignment of its 128 products to a common exponent."""
    off = (got.double() - want).abs()
    bound = want.abs() * 2.0 ** -8 + size * 2.0 ** -13
    assert torch.isfinite(got.double()).all()
    assert (off <= bound).all(), (off - bound).max()


def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step, c):
    """(p, m, v) after a step, and what bounds the roundings of each: all float64."""
    g = g * c
    m1, v1 = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    den = v1.sqrt() / math.sqrt(1 - beta2 ** step) + eps
    rate = lr / (1 - beta1 ** step)
    p1 = p * (1 - lr * weight_decay) - rate * m1 / den
    # roundings of fp32 (2^-24 of the value each): of m two products, a sum, the three factors; of v two more; the root halves v's
    # and adds its own, the denominator three more; the quotient, the rate and its product; of p the decay, a product, the difference
    u = 2.0 ** -24
    off_m = 6 * u * (beta1 * m.abs() + (1 - beta1) * g.abs())
    off_v = 8 * u * v1
    off_p = 3 * u * p.abs() + rate * (off_m + 12 * u * m1.abs()) / den + u * p1.abs()
    return (p1, off_p), (m1, off_m), (v1, off_v)
