"""A served decoding step in 64 bits (test infrastructure, shares nothing with the product): the paged cache of 8-bit values, attention
over it and products with 4-bit weights, token by token as include/astra.h states them.  Pinned by tests/test_oracle_serving.py."""
from __future__ import annotations

import math

import numpy as np


def e4m3_values() -> np.ndarray:
    """Value of each of the 256 codes: 1 sign, 4 exponent (bias 7), 3 mantissa bits; exponent and mantissa all ones is the only NaN."""
    code = np.arange(256)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((code & 127) == 127, np.nan, v)
    return np.where(code & 128, -v, v)


def e4m3_code(x) -> np.ndarray:
    """Code of the value nearest to x (|x| <= 448), ties to the even code; NaN to NaN."""
    x = np.asarray(x, dtype=np.float64)
    grid = e4m3_values()[:127]                                    # ascending, code = index
    a = np.abs(x)
    hi = np.clip(np.searchsorted(grid, np.where(np.isnan(a), 0.0, a)), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isnan(x), 127, code).astype(np.uint8)
    return code | (np.signbit(x) & ~np.isnan(x)).astype(np.uint8) * np.uint8(128)


def block_scale(most: float) -> float:
    """The smallest power of two s with most <= 448 s, 2^-100 <= s <= 2^110."""
    e = -100
    while e < 110 and most > math.ldexp(448.0, e):
        e += 1
    return math.ldexp(1.0, e)


def turned(x: np.ndarray, position: int, base: float) -> np.ndarray:
    """x [..., dh]: pair j by position * base^(-2j/dh)."""
    dh = x.shape[-1]
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * position * base ** (-np.arange(0, dh, 2) / dh))
    return np.stack((z.real, z.imag), -1).reshape(x.shape)


def _pages(table, s, t, page, n_pages):
    at = t // page
    if at >= table.shape[1]:
        return -1
    p = int(table[s, at])
    return p if 0 <= p < n_pages else -1


def cache_append(table, lens, first, shift, q, k, v, k_pages, v_pages, k_scales, v_scales, base=0.0):
    """q [n, Hq, dh] or None, k, v [n, Hkv, dh]; pages uint8 [n_pages, Hkv, page, dh], scales fp32 [n_pages, Hkv].  Returns (q turned, k_pages,
    v_pages, k_scales, v_scales, exact): new arrays; exact[m] maps (page, head, offset) to the unrounded value of a new row of m = 0 keys, 1 values."""
    n_pages, hkv, page, dh = k_pages.shape
    out_q = None if q is None else q.astype(np.float64).copy()
    pages, scales = [k_pages.copy(), v_pages.copy()], [k_scales.astype(np.float64), v_scales.astype(np.float64)]
    val, exact = e4m3_values(), [{}, {}]
    for s in range(len(lens)):
        rows = []
        for i, r in enumerate(range(first[s], first[s + 1])):
            t = int(lens[s]) + i
            m = t + (0 if shift is None else int(shift[s]))
            kr = k[r].astype(np.float64)
            if base > 0:
                kr = turned(kr, m, base)
                if q is not None:
                    out_q[r] = turned(q[r].astype(np.float64), m, base)
            p = _pages(table, s, t, page, n_pages)
            if p >= 0:
                rows.append((p, t, (kr, v[r].astype(np.float64))))
        for p in dict.fromkeys(p for p, _, _ in rows):
            mine = [(t, x) for q_, t, x in rows if q_ == p]
            held = mine[0][0] % page
            for j in range(2):
                for h in range(hkv):
                    x = np.stack([a[j][h] for _, a in mine])
                    ok = np.isfinite(x)
                    scale = block_scale(np.abs(x[ok]).max(initial=0.0))
                    old = scales[j][p, h]
                    if held:
                        scale = max(scale, old)
                        if scale > old:
                            pages[j][p, h, :held] = e4m3_code(val[pages[j][p, h, :held]] * (old / scale))
                    scales[j][p, h] = scale
                    code = e4m3_code(np.where(ok, np.clip(np.where(ok, x, 0) / scale, -448, 448), np.nan))
                    for (t, _), c, u in zip(mine, code, x):
                        pages[j][p, h, t % page] = c
                        exact[j][p, h, t % page] = u
    return out_q, pages[0], pages[1], scales[0], scales[1], exact


def cache_attention(table, lens, first, q, k_pages, v_pages, k_scales, v_scales, scale=None, prior=None, prior_lse=None):
    """(out [n, Hq, dh], lse [n, Hq]); rows that no sequence has are NaN."""
    n, hq, dh = q.shape
    n_pages, hkv, page, _ = k_pages.shape
    val, f = e4m3_values(), 1.0 / math.sqrt(dh) if scale is None else scale
    out, lse = np.full(q.shape, np.nan), np.full((n, hq), np.nan)
    for s in range(len(lens)):
        total = int(lens[s]) + first[s + 1] - first[s]
        at = [(t, _pages(table, s, t, page, n_pages)) for t in range(total)]
        at = [(t, p) for t, p in at if p >= 0]
        tok = np.array([t for t, _ in at], dtype=np.int64)
        rows = [np.stack([val[pg[p, :, t % page]] * sc[p].astype(np.float64)[:, None] for t, p in at]) if at else np.zeros((0, hkv, dh))
                for pg, sc in ((k_pages, k_scales), (v_pages, v_scales))]
        for i, r in enumerate(range(first[s], first[s + 1])):
            seen = tok <= int(lens[s]) + i
            for h in range(hq):
                kk, vv = rows[0][seen, h // (hq // hkv)], rows[1][seen, h // (hq // hkv)]
                z = (kk @ q[r, h].astype(np.float64)) * f
                if prior is not None:
                    z = np.append(z, np.float64(prior_lse[r, h]))
                    vv = np.concatenate((vv, np.where(np.isneginf(prior_lse[r, h]), 0.0, prior[r, h].astype(np.float64))[None]))
                top = z.max(initial=-np.inf)
                if np.isneginf(top):
                    out[r, h], lse[r, h] = 0.0, -np.inf
                    continue
                w = np.exp(z - top)
                out[r, h], lse[r, h] = (w / w.sum()) @ vv, top + np.log(w.sum())
    return out, lse


def w4_linear(x, codes, scales, zeros=None, bias=None, group=128):
    """x [T, in]; codes [out, in / 2], scales and zeros [out, in / group]."""
    n_out, half = codes.shape
    q = np.zeros((n_out, 2 * half))
    for k in range(2 * half):
        q[:, k] = (codes[:, k // 2] >> (4 * (k % 2))) & 15
    z = 8.0 if zeros is None else np.repeat((np.asarray(zeros) & 15).astype(np.float64), group, 1)
    w = (q - z) * np.repeat(np.asarray(scales, dtype=np.float64), group, 1)
    y = np.asarray(x, dtype=np.float64) @ w.T
    return y if bias is None else y + np.asarray(bias, dtype=np.float64)
