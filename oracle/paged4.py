"""The paged 4-bit cache, packed prompts and dense attention over either (test infrastructure only), in fp64.

The codes' rounding is the definition's: int4 groups of 32 channels with z = the largest fp16 at most their minimum, s = the smallest
fp16 with 15 s >= max - z and c = rint((x - z) / s); e2m1 groups with the least power of two that keeps the largest value within 6
and the nearest of the sixteen numbers, ties to the even code.  The attention is Eq. 2's softmax attention with the causal row sets
of the step.  Nothing here is vectorized over sequences or positions.
"""
from __future__ import annotations

import math

import numpy as np

from oracle.paged import seen_by

GROUP, MOST = 32, 32768.0
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
S_MOST, E_LEAST, E_MOST = 4372.0, -23, 13
TOP = 65520.0                              # what rounds to an infinity in fp16


def half_down(x):
    """Largest fp16 at most x, never -0."""
    h = np.float16(x)
    if float(h) > x:
        h = np.nextafter(h, np.float16(-np.inf))
    return np.float16(0) if h == 0 else h


def encode_group(x, fmt):
    """Codes 0..15 of 32 values and the group's numbers: (s, z) in fp16 or the exponent's byte."""
    if not np.all(np.isfinite(x)):
        return np.zeros(len(x), np.uint8), (np.float16(np.nan), np.float16(np.nan)) if fmt == "int4" else 255
    y = np.clip(np.asarray(x, np.float64), -MOST, MOST)
    if fmt == "int4":
        z = half_down(y.min())
        span = y.max() - float(z)
        s = np.float16(span / 15)
        while 15 * float(s) < span:
            s = np.nextafter(s, np.float16(np.inf))
        while s > 0 and 15 * float(np.nextafter(s, np.float16(-np.inf))) >= span:
            s = np.nextafter(s, np.float16(-np.inf))
        s = np.float16(0) if s == 0 else s
        c = np.clip(np.rint((y - float(z)) / float(s)), 0, 15) if s > 0 else np.zeros(len(y))
        return c.astype(np.uint8), (s, z)
    a, e = np.abs(y).max(), E_LEAST
    while a > 6 * 2.0 ** e:
        e += 1
    c = np.empty(len(y), np.uint8)
    for i, v in enumerate(y):
        d = np.abs(E2M1 - abs(v) / 2.0 ** e)
        near = np.flatnonzero(d == d.min())
        c[i] = (near[0] if near[0] % 2 == 0 else near[-1]) | (8 if math.copysign(1, v) < 0 else 0)
    return c, e + 127


def decode_group(c, meta, fmt):
    """fp64 values of codes; NaN where the numbers are none that an append writes."""
    c = c.astype(int)
    if fmt == "int4":
        s, z = float(meta[0]), float(meta[1])
        ok = 0 <= s <= S_MOST and abs(z) <= MOST and z + 15 * s < TOP and not (s == 0 and math.copysign(1, s) < 0)
        return z + s * c if ok else np.full(len(c), np.nan)
    e = int(meta) - 127
    if not E_LEAST <= e <= E_MOST:
        return np.full(len(c), np.nan)
    return np.where(c > 7, -1.0, 1.0) * E2M1[c & 7] * 2.0 ** e


def pack(c):
    return (c[0::2] | (c[1::2] << 4)).astype(np.uint8)


def unpack(w):
    return np.stack([w & 15, w >> 4], axis=-1).reshape(*w.shape[:-1], 2 * w.shape[-1])


def empty(n_pages, H, page, d, fmt, rng=None):
    """(codes, numbers) of one side of a cache, with valid numbers drawn when rng is given."""
    codes = np.zeros((n_pages, H, page, d // 2), np.uint8)
    meta = np.zeros((n_pages, H, page, d // GROUP, 2), np.float16) if fmt == "int4" else np.full((n_pages, H, page, d // GROUP), 127, np.uint8)
    if rng is not None:
        codes[:] = np.frombuffer(rng.bytes(codes.size), np.uint8).reshape(codes.shape)
        if fmt == "int4":
            meta[..., 0] = np.exp(rng.normal(size=meta.shape[:-1]) * 0.5) * 0.3
            meta[..., 1] = -rng.uniform(3, 12, meta.shape[:-1]) * meta[..., 0]
        else:
            meta[:] = rng.integers(124, 129, meta.shape)
    return codes, meta


def row_of(w, m, fmt):
    """fp64 values [d] of one position and head."""
    c = unpack(w)
    return np.concatenate([decode_group(c[GROUP * g:GROUP * (g + 1)], m[g], fmt) for g in range(m.shape[0])])


def rows_of(codes, meta, fmt):
    """fp64 values [..., d], the same as row_of of each, by tables."""
    c = unpack(codes).reshape(*codes.shape[:-1], 2 * codes.shape[-1] // GROUP, GROUP).astype(int)
    if fmt == "int4":
        s, z = meta[..., 0].astype(np.float64), meta[..., 1].astype(np.float64)
        ok = (s >= 0) & (s <= S_MOST) & (np.abs(z) <= MOST) & (z + 15 * s < TOP) & ~((s == 0) & np.signbit(s))
        x = np.where(ok, z, 0.0)[..., None] + np.where(ok, s, 0.0)[..., None] * c
    else:
        e = meta.astype(int) - 127
        ok = (e >= E_LEAST) & (e <= E_MOST)
        x = np.where(c > 7, -1.0, 1.0) * E2M1[c & 7] * np.exp2(np.clip(e, E_LEAST, E_MOST).astype(np.float64))[..., None]
    return np.where(ok[..., None], x, np.nan).reshape(*codes.shape[:-1], 2 * codes.shape[-1])


def places(cu, lens, block_table, n_pages, page):
    """(row, sequence, position, page or -1) of every row of a sequence."""
    for b in range(len(lens)):
        n = int(cu[b + 1] - cu[b])
        for t in range(n):
            p = int(lens[b]) - n + t
            pid = -1
            if 0 <= p < block_table.shape[1] * page:
                pid = int(block_table[b, p // page])
            yield int(cu[b]) + t, b, p, pid if 0 <= pid < n_pages else -1


def append(x, cu, lens, block_table, codes, meta, fmt):
    """Store rows x [T, H, d] (fp64 holding fp32 values) in place; returns the rows that the codes stand for (NaN: dropped)."""
    n_pages, H, page, _ = codes.shape
    out = np.full(x.shape, np.nan)
    dropped = np.ones(x.shape[0], bool)
    for r, _, p, pid in places(cu, lens, block_table, n_pages, page):
        if pid < 0:
            continue
        dropped[r] = False
        for h in range(H):
            for g in range(x.shape[2] // GROUP):
                c, m = encode_group(x[r, h, GROUP * g:GROUP * (g + 1)], fmt)
                codes[pid, h, p % page, GROUP // 2 * g:GROUP // 2 * (g + 1)] = pack(c)
                meta[pid, h, p % page, g] = m
                out[r, h, GROUP * g:GROUP * (g + 1)] = decode_group(c, np.array(m, np.float16) if fmt == "int4" else m, fmt)
    return out, dropped


def read(cu, lens, block_table, codes, meta, T, fmt):
    """Rows [T, H, d] (0 where a page is not there); rows of no sequence are NaN and marked."""
    n_pages, H, page, half = codes.shape
    out, none = np.full((T, H, 2 * half), np.nan), np.ones(T, bool)
    for r, _, p, pid in places(cu, lens, block_table, n_pages, page):
        none[r] = False
        out[r] = 0 if pid < 0 else np.stack([row_of(codes[pid, h, p % page], meta[pid, h, p % page], fmt) for h in range(H)])
    return out, none


# ---- attention --------------------------------------------------------------------------------------------
def attend_rows(q, k, v, i, there, sm_scale, window, n_sink):
    """One sequence and key/value head: q [n, G, d] at positions i over k, v [L, d].  Returns o, lse and what bounds rounding
    errors: sum_j p_j |v_j|, max_j sm_scale sum |q_e k_je|, and (max_j p_j) sum_j |v_j| over what a row sees."""
    n, G, d = q.shape
    o, lse = np.zeros((n, G, d)), np.full((n, G), -np.inf)
    av, aq, aw = np.zeros((n, G, d)), np.zeros((n, G)), np.zeros((n, G, d))
    with np.errstate(invalid="ignore", over="ignore"):
        for t in range(n):
            j = seen_by(int(i[t]), len(k), window, n_sink) if i[t] >= 0 else np.arange(0)
            j = j[there[j]]
            if len(j) == 0:
                continue
            x = sm_scale * (q[t] @ k[j].T)                        # [G, keys]
            top = x.max(axis=1)
            p = np.exp(x - top[:, None])
            total = p.sum(axis=1)
            with np.errstate(divide="ignore"):
                lse[t] = np.where(np.isneginf(top), -np.inf, top + np.log(total))
            p = np.where(np.isneginf(top)[:, None], 0.0, p / total[:, None])
            o[t], av[t] = p @ v[j], p @ np.abs(v[j])
            aw[t] = p.max(axis=1)[:, None] * np.abs(v[j]).sum(axis=0)
            aq[t] = sm_scale * (np.abs(q[t]) @ np.abs(k[j]).T).max(axis=1)
    return o, lse, av, aq, aw


def attend(q, seqs, Hkv, sm_scale, window=0, n_sink=0):
    """q [T, Hq, d]; seqs yields (first row, end row, length, k [L, Hkv, d], v, there [L]) per sequence.  Rows of no sequence: NaN."""
    T, Hq, d = q.shape
    G = Hq // Hkv
    out = [np.full((T, Hq, d), np.nan), np.full((T, Hq), np.nan), np.zeros((T, Hq, d)), np.zeros((T, Hq)), np.zeros((T, Hq, d))]
    for r0, r1, length, k, v, there in seqs:
        i = np.arange(length - (r1 - r0), length)
        for h in range(Hkv):
            heads = slice(h * G, h * G + G)
            got = attend_rows(q[r0:r1, heads], k[:, h], v[:, h], i, there, sm_scale, window, n_sink)
            for whole, part in zip(out, got):
                whole[r0:r1, heads] = part
    return out


def packed_seqs(k, v, cu_q, cu_k):
    for b in range(len(cu_q) - 1):
        n = int(cu_k[b + 1] - cu_k[b])
        yield int(cu_q[b]), int(cu_q[b + 1]), n, k[cu_k[b]:cu_k[b + 1]], v[cu_k[b]:cu_k[b + 1]], np.ones(n, bool)


def paged_seqs(cu, lens, block_table, sides, fmt):
    """sides: ((codes, numbers) of the keys, of the values).  A position with a group that reads as NaN is NaN altogether."""
    n_pages, H, page, _ = sides[0][0].shape
    for b in range(len(lens)):
        L = max(min(int(lens[b]), block_table.shape[1] * page), 0)
        ids = block_table[b, :-(-L // page)]
        there = np.repeat((ids >= 0) & (ids < n_pages), page)[:L]
        safe = np.clip(ids, 0, n_pages - 1)
        k, v = (rows_of(c[safe], m[safe], fmt).transpose(0, 2, 1, 3).reshape(-1, H, 2 * c.shape[3])[:L] for c, m in sides)
        bad = np.isnan(k).any(axis=2) | np.isnan(v).any(axis=2)
        yield int(cu[b]), int(cu[b + 1]), int(lens[b]), np.where(bad[..., None], np.nan, k), np.where(bad[..., None], np.nan, v), there
