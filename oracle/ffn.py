"""The operators of a decode step's feed-forward half in 64 bits (numpy), written from their formulas: products with an
epilogue, routing to experts, the experts' products.  Test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")      # by their number in the C ABI
LIPSCHITZ = 1.13                                          # no activation's slope is larger

_erf = np.vectorize(math.erf, otypes=[np.float64])


def activation(z, act: int) -> np.ndarray:
    z = np.asarray(z, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        if act == 1:
            return np.where(z < 0, 0.0, z)
        if act == 2:
            return z / (1.0 + np.exp(-z))
        if act == 3:
            return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
        if act == 4:
            return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def nt_act(x, Wt, act: int, gated: bool, bias=None, residual=None):
    """The values of nmm_gemv_nt_act before their rounding, and how far fp32 sums of K products may take them.

    A sum of K products passes at most K additions and 33 roundings per 32 of them inside the matrix cores; the waves' sums,
    the bias and the product's own additions are 16 more at most.  Each is half a step, 2^-24, of the sum of magnitudes.
    An activation moves by at most LIPSCHITZ times that, and its own evaluation by 2^-20."""
    x, Wt = np.asarray(x, dtype=np.float64), np.asarray(Wt, dtype=np.float64)
    K = x.shape[1]
    z, mag = x @ Wt.T, np.abs(x) @ np.abs(Wt).T
    if bias is not None:
        z, mag = z + bias, mag + np.abs(bias)
    dz = (K + 33 * (K / 32 + 1) + 16) * 2.0 ** -24 * mag
    N = Wt.shape[0] // 2 if gated else Wt.shape[0]
    v = activation(z[:, :N], act)
    err = LIPSCHITZ * dz[:, :N] + (2.0 ** -20 * np.abs(v) + 2.0 ** -20 * np.abs(z[:, :N]) * (act > 2) if act > 1 else 0.0)
    if gated:
        up = z[:, N:]
        err = err * np.abs(up) + (np.abs(v) + err) * dz[:, N:] + 2.0 ** -24 * np.abs(v * up)
        v = v * up
    if residual is not None:
        v = v + residual
        err = err + 2.0 ** -24 * np.abs(v)
    return v, err


def route(logits, top_k: int, softmax: bool, bias=None, groups: int = 1, top_groups: int = 1, group_top: int = 1,
          renormalize: bool = False, scale: float = 1.0, mask=None):
    """chosen, weights, offsets and the ordered pairs of nmm_moe_route."""
    l = np.asarray(logits, dtype=np.float64)
    T, E = l.shape
    with np.errstate(all="ignore"):
        if softmax:
            top = np.fmax.reduce(l, axis=1, keepdims=True)
            s = np.exp(l - top)
            s = s / s.sum(1, keepdims=True)
        else:
            s = 1.0 / (1.0 + np.exp(-l))
        c = s if bias is None else s + np.asarray(bias, dtype=np.float64)
    c = np.where(np.isnan(c), -np.inf, c)
    chosen = np.full((T, top_k), -1, dtype=np.int64)
    weights = np.zeros((T, top_k))
    size = E // groups
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        open_ = np.arange(E)
        if groups > 1:
            best = -np.sort(-c[t].reshape(groups, size), axis=1)
            with np.errstate(invalid="ignore"):
                total = best[:, 0] + best[:, 1] if group_top == 2 and size > 1 else best[:, 0]
            total = np.where(np.isnan(total), -np.inf, total)
            kept = sorted(range(groups), key=lambda g: (-total[g], g))[:top_groups]
            open_ = np.array([e for e in range(E) if e // size in kept])
        order = sorted(open_, key=lambda e: (-c[t, e], e))[:top_k]
        chosen[t] = order
        w = s[t, order]
        with np.errstate(all="ignore"):
            weights[t] = (w / w.sum() if renormalize else w) * scale
    flat = chosen.reshape(-1)
    pairs = np.argsort(np.where(flat < 0, E, flat), kind="stable")[:np.count_nonzero(flat >= 0)]
    offsets = np.concatenate(([0], np.cumsum(np.bincount(flat[flat >= 0], minlength=E))))
    return chosen, weights, offsets, pairs


def experts(x, w1, w2, chosen, weights, first: int, act: int, half_step: float, residual=None):
    """The values of nmm_moe_experts before y's rounding, and how far they may be off: the up product's sums as in nt_act, h's
    rounding (half_step of its magnitude, and of the least normal number), the down product's sums and top_k additions."""
    x, w1, w2 = (np.asarray(a, dtype=np.float64) for a in (x, w1, w2))
    T, hidden = x.shape
    local, inner = w1.shape[0], w1.shape[1] // 2
    y, err = np.zeros((T, hidden)), np.zeros((T, hidden))
    for e in range(local):
        for t, i in np.argwhere(chosen == first + e):
            h, dh = nt_act(x[t:t + 1], w1[e], act, True)
            dh = dh + half_step * (np.abs(h) + dh) + 2.0 ** -25
            w = float(weights[t, i])
            part, mag = (h @ w2[e].T)[0], (np.abs(h) @ np.abs(w2[e]).T)[0]
            y[t] += w * part
            off = (dh @ np.abs(w2[e]).T)[0] + (inner + 33 * (inner / 32 + 1) + 16) * 2.0 ** -24 * mag
            err[t] += abs(w) * (off + 2.0 ** -22 * mag)
    err = err * (1 + 2.0 ** -20) + 2.0 ** -22 * np.abs(y)
    if residual is not None:
        y = y + residual
        err = err + 2.0 ** -24 * np.abs(y)
    return y, err
