"""The operators of a batched decode in 64 bits (numpy), written from their formulas: 8-bit latent-cache rows,
attention over a paged cache with a shared prefix, products with 4-bit weights.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

BLOCK, SCALE_BYTES, MIN_EXP = 32, 16, -117


def bf16_round(v) -> np.ndarray:
    """Nearest bf16 values, ties to even, of fp64 values in the normal range (and zeros, infinities, NaN)."""
    v = np.asarray(v, dtype=np.float64)
    m, e = np.frexp(np.where(np.isfinite(v), v, 0.0))
    r = np.ldexp(np.rint(m * 256.0), e - 8)
    r = np.where(np.abs(r) > 3.3895313892515355e38, np.copysign(np.inf, r), r)
    return np.where(np.isfinite(v), r, v)


def bf16_decode(bits) -> np.ndarray:
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def bf16_encode(v) -> np.ndarray:
    """The bits of values that are bf16 numbers."""
    return (np.asarray(v, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def e4m3_values() -> np.ndarray:
    """The 256 values of e4m3: sign, 4 exponent bits (bias 7), 3 of mantissa, no infinity, 0x7F NaN."""
    c = np.arange(256)
    ex, man = (c >> 3) & 15, (c & 7).astype(np.float64)
    v = np.where(ex == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * 2.0 ** (ex - 7.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >= 128, -v, v)


def e4m3_encode(v) -> np.ndarray:
    """Codes of fp64 values of magnitude at most 448: nearest, ties to the even code; NaN 0x7F."""
    v = np.asarray(v, dtype=np.float64)
    nan = np.isnan(v)
    a = np.where(nan, 0.0, np.abs(v))
    assert np.all(a <= 448)
    grid = e4m3_values()[:127]
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.signbit(v), code + 128, code)
    return np.where(nan, 127, code).astype(np.uint8)


def cache_entry(src, kv: int, rope: int, gamma=None, eps: float = 0.0, positions=None, theta: float = 1e4) -> np.ndarray:
    """[RMSNorm | RoPE] of the rows of src, unrounded."""
    src = np.asarray(src, dtype=np.float64)
    c, k = src[:, :kv], src[:, kv:kv + rope]
    if gamma is not None:
        c = c / np.sqrt((c * c).mean(1, keepdims=True) + eps) * np.asarray(gamma, dtype=np.float64)
    if positions is not None and rope:
        a = np.asarray(positions, dtype=np.float64)[:, None] * float(theta) ** (-2.0 * np.arange(rope // 2) / rope)
        cs, sn = np.cos(a), np.sin(a)
        k = np.stack((k[:, 0::2] * cs - k[:, 1::2] * sn, k[:, 0::2] * sn + k[:, 1::2] * cs), -1).reshape(k.shape)
    return np.concatenate((c, k), 1)


def quantise_rows(rows, kv: int) -> np.ndarray:
    """8-bit rows (bytes) of bf16 values [n, kv + rope]."""
    rows = np.asarray(rows, dtype=np.float64)
    n, rope = rows.shape[0], rows.shape[1] - kv
    v = rows[:, :kv].reshape(n, -1, BLOCK)
    fin = np.isfinite(v)
    amax = np.where(fin, np.abs(v), 0.0).max(-1)
    m, x = np.frexp(amax)                                  # 448 = 0.875 * 2^9
    e = np.where(amax == 0, MIN_EXP, np.maximum(x - 9 + (m > 0.875), MIN_EXP))
    codes = e4m3_encode(np.where(fin, v, np.nan) * np.exp2(-e.astype(np.float64))[..., None]).reshape(n, kv)
    scales = np.full((n, SCALE_BYTES), 127, dtype=np.uint8)
    scales[:, :kv // BLOCK] = e + 127
    tail = bf16_encode(rows[:, kv:]).reshape(n, rope).view(np.uint8) if rope else np.zeros((n, 0), np.uint8)
    return np.concatenate((codes, scales, tail), 1)


def dequantise_rows(data, kv: int, rope: int) -> np.ndarray:
    """What 8-bit rows stand for, fp64 [n, kv + rope]: bf16 numbers, 2^128 and more as infinity (e4m3 rounds bf16's
    largest values up to 2^128)."""
    data = np.ascontiguousarray(data)
    v = e4m3_values()[data[:, :kv]].reshape(len(data), -1, BLOCK)
    v = v * np.exp2(data[:, kv:kv + kv // BLOCK].astype(np.float64) - 127)[..., None]
    k = bf16_decode(np.ascontiguousarray(data[:, kv + SCALE_BYTES:kv + SCALE_BYTES + 2 * rope]).view(np.uint16))
    v = np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)
    return np.concatenate((v.reshape(len(data), kv), k.reshape(len(data), rope)), 1)


def attention_batch(q, rows, scale: float, kv: int, page: int, pages, lens, max_len: int, prefix_pages=(),
                    prefix_len: int = 0):
    """out [B, T, H, kv] and sum_j p_j |v_j| of q [B, T, H, d] over cache rows [n, d] (fp64 values).  Positions
    on a page outside the pool do not exist; a row with no position gives zeros."""
    q = np.asarray(q, dtype=np.float64)
    B, T, H, _ = q.shape
    n_pages = len(rows) // page
    out, mag = np.zeros((B, T, H, kv)), np.zeros((B, T, H, kv))

    def locate(table, n):
        pos = np.arange(max(0, n))
        p = np.asarray(table, dtype=np.int64)[pos // page]
        ok = (p >= 0) & (p < n_pages)
        return pos, np.where(ok, p * page + pos % page, -1)

    _, shared = locate(prefix_pages, prefix_len)
    for b in range(B):
        n = min(max(0, int(lens[b])), max_len)
        _, mine = locate(pages[b], n)
        for t in range(T):
            at = np.concatenate((shared, mine[:max(0, n - (T - 1 - t))]))
            at = at[at >= 0]
            if len(at) == 0:
                continue
            ctx = rows[at]
            s = scale * (q[b, t] @ ctx.T)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[b, t], mag[b, t] = p @ ctx[:, :kv], p @ np.abs(ctx[:, :kv])
    return out, mag


E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])


def w4_decode(codes, scales, group: int, K: int, zeros=None, mx: bool = False) -> np.ndarray:
    """The weight [N, K] that packed codes [N, >= ceil(K / 2)], scales [N, groups] and zero points stand for."""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(len(codes), -1)[:, :K]
    g = np.arange(K) // group
    if mx:
        return E2M1[c] * np.exp2(scales.astype(np.float64) - 127)[:, g]
    z = 8.0 if zeros is None else zeros.astype(np.float64)[:, g]
    return (c - z) * np.asarray(scales, dtype=np.float64)[:, g]
