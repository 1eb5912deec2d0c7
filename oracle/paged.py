"""Rotary positions, the paged 8-bit cache and dense attention over it (test infrastructure only), in fp64.

The attention is Eq. 2's softmax attention with the causal row sets of the step, over a cache whose stored values are
scale * code.  The codes' rounding is the definition's: to nearest, ties to even, of the exact quotient; the scale of a page
and head is max * fp32(1 / 127) in fp32 (int8) or the least power of two that keeps the largest value within 448 (e4m3), and grows by
powers of two while a sequence fills the page.  Nothing here is vectorized over sequences or pages.
"""
from __future__ import annotations

import math

import numpy as np


def e4m3_values():
    """The 256 OCP e4m3 numbers by code (NaN at 0x7F and 0xFF)."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
        out[c] = math.nan if (c & 127) == 127 else (-v if c & 128 else v)
    return out


E4M3 = e4m3_values()
_POS = E4M3[:127]                       # 0 .. 448, ascending with the code


def e4m3_encode(x):
    """Codes of x (|x| <= 448, or NaN), to nearest, ties to the even code."""
    a = np.abs(np.asarray(x, np.float64))
    bad, a = np.isnan(a), np.nan_to_num(a)
    hi = np.clip(np.searchsorted(_POS, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(bad, 127, code)
    return np.where(np.signbit(x), code | 128, code).astype(np.uint8)


def decode(codes, fmt):
    """fp64 values of raw code bytes."""
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else E4M3[codes]


def encode(x, fmt):
    if fmt == "int8":
        return np.clip(np.rint(x), -127, 127).astype(np.int8).view(np.uint8)
    return e4m3_encode(x)


# ---- rotary positions -----------------------------------------------------------------------------------
def frequencies(rot, base=10000.0, scaling="none", factor=1.0, orig_len=0, low=1.0, high=32.0):
    """The pairs' frequencies and the factor of the table."""
    f, m = [], 1.0
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "ntk" else base
        x = b ** (-2.0 * i / rot)
        if scaling == "linear":
            x /= factor
        if scaling == "yarn":
            g = min(max((orig_len * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            x = x * (g + (1 - g) / factor)
        f.append(x)
    if scaling == "yarn":
        m = 1 + 0.1 * math.log(factor)
    return np.array(f), m


def table(n_pos, rot, **kw):
    f, m = frequencies(rot, **kw)
    a = np.arange(n_pos)[:, None] * f
    return m * np.stack([np.cos(a), np.sin(a)], axis=-1)


def rotate(x, cs, layout="half", inverse=False):
    """x [..., d] fp64 with cs [..., rot / 2, 2] broadcast over the heads: [T, H, d] and [T, rot / 2, 2]."""
    y = np.array(x, np.float64)
    half = cs.shape[-2]
    c, s = cs[..., 0].astype(np.float64)[:, None], cs[..., 1].astype(np.float64)[:, None]
    s = -s if inverse else s
    i = np.arange(half)
    i0, i1 = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
    y[..., i0] = x[..., i0] * c - x[..., i1] * s
    y[..., i1] = x[..., i0] * s + x[..., i1] * c
    return y


# ---- the cache --------------------------------------------------------------------------------------------
def need_of(a, fmt):
    """The scale that values of magnitude up to a need."""
    if not np.isfinite(a):
        return np.float32(np.nan)
    if a < 2.0 ** -100:
        return np.float32(0)
    if fmt == "int8":
        return np.float32(a) * np.float32(1 / 127)
    e = math.frexp(a)[1] - 9                 # a < 2^(e + 9) = 512 * 2^e
    while a > math.ldexp(448, e):
        e += 1
    while a <= math.ldexp(448, e - 1):
        e -= 1
    return np.float32(math.ldexp(1, e))


def append(x, cu, lens, block_table, codes, scale, fmt):
    """Store rows x [T, H, d] (fp64 holding fp32 values) into codes uint8 [pages, H, page, d] and scale fp32 [pages, H], in
    place."""
    n_pages, H, page, _ = codes.shape
    for b in range(len(lens)):
        n = int(cu[b + 1] - cu[b])
        start = int(lens[b]) - n
        pos = np.arange(max(start, 0), int(lens[b]))
        for p in sorted(set(pos // page)):
            if p >= block_table.shape[1] or not 0 <= block_table[b, p] < n_pages:
                continue
            pid = block_table[b, p]
            mine = pos[pos // page == p]
            rows = cu[b] + mine - start
            for h in range(H):
                v = x[rows, h]
                a = np.max(np.abs(v)) if np.all(np.isfinite(v)) else np.inf
                need, old = need_of(a, fmt), scale[pid, h]
                went_on = mine[0] % page > 0
                s = need
                if went_on and old != 0:
                    if not np.isfinite(need) or not np.isfinite(old):
                        s = np.float32(np.nan)
                    else:
                        k = 0
                        while float(old) * 2.0 ** k < float(need):
                            k += 1
                        s = np.float32(float(old) * 2.0 ** k)
                        if k:                # (all of the page: what the call writes is written below)
                            codes[pid, h] = encode(decode(codes[pid, h], fmt) / 2.0 ** k, fmt)
                scale[pid, h] = s
                ok = np.isfinite(s) and s > 0
                codes[pid, h, mine % page] = encode(v / float(s), fmt) if ok else 0


# ---- attention --------------------------------------------------------------------------------------------
def seen_by(i, n, window, n_sink):
    j = np.arange(min(i + 1, n))
    return j[(j > i - window) | (j < n_sink)] if window else j


def attend(q, cu, lens, block_table, k_codes, v_codes, k_scale, v_scale, fmt, sm_scale, window=0, n_sink=0):
    """q [T, Hq, d] fp64, already rotated.  Returns o [T, Hq, d], lse [T, Hq] (NaN at rows of no sequence), and what bounds
    rounding errors: sum_j p_j |v_j| [T, Hq, d], max_j sm_scale sum_e |q_e k_je| [T, Hq], and with the values' scales s_j and
    codes c_j max_j (p_j s_j) sum_j |c_j| [T, Hq, d]."""
    T, Hq, d = q.shape
    n_pages, Hkv, page, _ = k_codes.shape
    G = Hq // Hkv
    o, lse = np.full((T, Hq, d), np.nan), np.full((T, Hq), np.nan)
    av, aq, aw = np.zeros((T, Hq, d)), np.zeros((T, Hq)), np.zeros((T, Hq, d))
    with np.errstate(invalid="ignore"):
        for b in range(len(lens)):
            n = int(cu[b + 1] - cu[b])
            L = min(int(lens[b]), block_table.shape[1] * page)
            ids = block_table[b, :-(-L // page)] if L > 0 else block_table[b, :0]
            there = np.repeat((ids >= 0) & (ids < n_pages), page)[:max(L, 0)]
            safe = np.clip(ids, 0, n_pages - 1)
            for h in range(Hkv):
                k, v = ((decode(c[safe, h], fmt) * np.where(np.isfinite(s[safe, h]), s[safe, h].astype(np.float64), np.nan)
                         [:, None, None]).reshape(-1, d) for c, s in ((k_codes, k_scale), (v_codes, v_scale)))
                vc = np.abs(decode(v_codes[safe, h], fmt)).reshape(-1, d)
                vs = np.repeat(v_scale[safe, h].astype(np.float64), page)
                for t in range(n):
                    r, i = int(cu[b]) + t, int(lens[b]) - n + t
                    j = seen_by(i, L, window, n_sink) if i >= 0 else np.arange(0)
                    j = j[there[j]]
                    for g in range(G):
                        hq = h * G + g
                        if len(j) == 0:
                            o[r, hq], lse[r, hq] = 0.0, -np.inf
                            continue
                        x = sm_scale * (k[j] @ q[r, hq])
                        top = x.max()
                        p = np.exp(x - top)
                        lse[r, hq] = top + math.log(p.sum()) if np.isfinite(top) else np.nan
                        p = p / p.sum()
                        o[r, hq] = p @ v[j]
                        av[r, hq] = p @ np.abs(v[j])
                        aw[r, hq] = (p * vs[j]).max() * vc[j].sum(axis=0)
                        aq[r, hq] = sm_scale * (np.abs(k[j]) @ np.abs(q[r, hq])).max()
    return o, lse, av, aq, aw
