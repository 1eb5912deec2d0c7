"""The paged 4-bit cache and dense attention over it: the HIP path against the fp64 oracle.

Tolerances.  Codes and groups' numbers are equal.  Rows read back are rounded once to their type, from fp32: half a step and 2^-24 of
|z| + |s c|.  Attention: with fp16 queries each |q_e| is off by at most 2^-11 of itself (2^-25 of the row's largest below its normal
range) and each int4 key by 2^-11 of itself, so a score by e = 2^-11 A or 2^-10 A, A = max_j sm_scale sum |q_e k_je|, and
(d + 8) 2^-23 A for its fp32 sum; a probability by 2 e of itself, and it is rounded to fp16: 2^-11 of itself, or 2^-25 of the unit
below fp16's normal range, the unit being at most the row's largest probability; an int4 value by 2^-11 of itself.  The output's own
rounding adds half a step, fp32 sums over the keys (n + d) 2^-23."""
import numpy as np
import pytest
import torch

from gpu_util import REL_FRO, say
from oracle import paged, paged4

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return t.cpu().double().numpy()


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def up(a):
    return torch.from_numpy(a.copy()).cuda()


def bits(a):
    a = a.cpu().numpy() if isinstance(a, torch.Tensor) else a
    a = a.view(np.uint16) if a.dtype == np.float16 else a
    return np.where((a & 0x7FFF) > 0x7C00, 0x7E00, a) if a.dtype == np.uint16 else a      # one NaN


def batch(rng, new, past, page, spare=2, holes=()):
    lens = [a + b for a, b in zip(new, past)]
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    pages = [-(-n // page) for n in lens]
    order = rng.permutation(sum(pages) + spare)
    tab = np.full((len(new), max(pages) + 1), -1, np.int32)
    at = 0
    for b, n in enumerate(pages):
        tab[b, :n] = order[at:at + n]
        at += n
    for b, p in holes:
        tab[b, p] = -1
    return cu, np.array(lens, np.int32), tab, sum(pages) + spare


APPENDS = [
    # new, past, page, Hkv, d, rot
    ([1], [0], 16, 1, 64, 16),
    ([1, 1, 1, 1], [15, 16, 17, 0], 16, 2, 64, 64),
    ([33, 0, 1, 64, 7], [10, 5, 63, 64, 0], 32, 3, 128, 32),
    ([100, 5], [1, 127], 128, 2, 128, 128),
    ([60, 64, 33], [0, 0, 63], 64, 5, 64, 48),
    ([1] * 70, list(range(70)), 64, 1, 128, 128),
    ([1, 0, 2, 0, 0, 0, 0, 50, 1], [5, 3, 31, 0, 1, 2, 3, 9, 100], 64, 2, 64, 32),
    ([23, 1, 1, 1], [8, 127, 128, 1], 128, 3, 128, 64),
    ([3, 2], [5, 60], 16, 9, 128, 112),
]


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
@pytest.mark.parametrize("dtype,layout", [("bf16", "half"), ("f16", "interleaved"), ("bf16", None)])
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append_and_read(F, case, dtype, layout, fmt):
    new, past, page, H, d, rot = APPENDS[case]
    say(f"append case {case} {dtype} {layout} {fmt}")
    rng = np.random.default_rng(case)
    cu, lens, tab, n_pages = batch(rng, new, past, page)
    n, T, dt = int(cu[-1]), int(cu[-1]) + 3, DT[dtype]           # three rows of no sequence
    size = np.exp(rng.normal(size=(T, H, 1)) * 1.5)
    k, v = (torch.from_numpy(rng.normal(size=(T, H, d)) * size).to(dt) for _ in range(2))
    k[n:] = float("nan")
    rows = torch.cat((k, v), dim=1).cuda()
    kd, vd = rows[:, :H], rows[:, H:]
    sides = [paged4.empty(n_pages, H, page, d, fmt, rng) for _ in range(2)]
    cs = paged.table(tab.shape[1] * page, rot).astype(np.float32)
    table = None if layout is None else torch.from_numpy(cs).cuda()
    cache = [up(sides[0][0]), up(sides[1][0]), up(sides[0][1]), up(sides[1][1])]
    kr, vr = (torch.full((T, H, d), 7.0, dtype=dt, device="cuda") for _ in range(2))
    F.paged4_append(kd, vd, i32(cu), i32(lens), i32(tab), *cache, table=table, layout=layout or "half", k_rows=kr, v_rows=vr)
    torch.cuda.synchronize()
    kx = f64(k)
    if layout:
        pos = np.concatenate([np.arange(lens[b] - new[b], lens[b]) for b in range(len(new))] + [np.zeros(3, int)]).astype(int)
        with np.errstate(invalid="ignore"):
            kx = paged.rotate(kx, cs[pos], layout).astype(np.float32).astype(np.float64)
    wants = []
    for x, (c, m), gc, gm, gr in ((kx, sides[0], cache[0], cache[2], kr), (f64(v), sides[1], cache[1], cache[3], vr)):
        want, _ = paged4.append(x, cu, lens, tab, c, m, fmt)
        wants.append(want)
        assert np.array_equal(bits(gm), bits(m)), f"{np.argwhere(bits(gm) != bits(m))[:3]}"
        same = gc.cpu().numpy() == c
        assert same.all(), f"{(~same).sum()} bytes differ, first at {np.argwhere(~same)[0]}"
        assert torch.all(gr[n:] == 7)
        # |z| + |s c| is at most 3 times the group's largest magnitude
        big = np.abs(want[:n]).reshape(n, H, -1, 32).max(-1, keepdims=True).repeat(32, -1).reshape(n, H, d)
        assert np.all(np.abs(f64(gr)[:n] - want[:n]) <= half_step(dt) * np.abs(want[:n]) + 3 * 2.0 ** -24 * big + (2.0 ** -25 if dtype == "f16" else 0))
    # without the rows, in place, and back
    twin = [t.clone() for t in cache]
    F.paged4_append(kd, vd, i32(cu), i32(lens), i32(tab), *twin, table=table, layout=layout or "half")
    assert all(torch.equal(bits_t(a), bits_t(b)) for a, b in zip(cache, twin))
    F.paged4_append(kd, vd, i32(cu), i32(lens), i32(tab), *twin, table=table, layout=layout or "half", k_rows=kd, v_rows=vd)
    assert all(torch.equal(bits_t(a), bits_t(b)) for a, b in zip(cache, twin))
    assert torch.equal(kd[:n], kr[:n]) and torch.equal(vd[:n], vr[:n]) and torch.isnan(kd[n:]).all()
    out = torch.full((T, 2 * H, d), 7.0, dtype=dt, device="cuda")
    gk, gv = F.paged4_read(i32(cu), i32(lens), i32(tab), *cache, T, k_out=out[:, :H], v_out=out[:, H:])
    assert torch.equal(gk[:n], kr[:n]) and torch.equal(gv[:n], vr[:n]) and torch.all(out[n:] == 7)
    other = torch.float16 if dtype == "bf16" else torch.bfloat16
    gk, gv = F.paged4_read(i32(cu), i32(lens), i32(tab), *cache, T, dtype=other)
    for got, want in ((gk, wants[0]), (gv, wants[1])):
        assert got.dtype == other
        assert np.all(np.abs(f64(got)[:n] - want[:n]) <= half_step(other) * np.abs(want[:n]) + 2.0 ** -20 * np.abs(want[:n]).max())


def bits_t(t):
    return t.view(torch.int16) if t.dtype == torch.float16 else t


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_append_edges(F, fmt):
    """Zeros, constants, tiny and huge values, infinities and NaN, values on the borders between codes, pages that are not there,
    negative starts, sequences beyond the block table."""
    page, H, d = 16, 2, 64
    tab = np.array([[0, 1, -1], [2, 99, 3], [4, 5, 6]], np.int32)
    rng = np.random.default_rng(0)
    sides = [paged4.empty(8, H, page, d, fmt, rng) for _ in range(2)]
    cache = [up(sides[0][0]), up(sides[1][0]), up(sides[0][1]), up(sides[1][1])]

    def step(what, new, lens, fill):
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T = int(cu[-1]) + 1
        x = torch.from_numpy(rng.normal(size=(T, H, d))).to(torch.bfloat16)
        fill(x)
        kr, vr = (torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        F.paged4_append(x.cuda(), (-x).cuda(), i32(cu), i32(lens), i32(tab), *cache, k_rows=kr, v_rows=vr)
        torch.cuda.synchronize()
        for y, (c, m), gc, gm, gr in ((f64(x), sides[0], cache[0], cache[2], kr), (-f64(x), sides[1], cache[1], cache[3], vr)):
            want, dropped = paged4.append(y, cu, lens, tab, c, m, fmt)
            at = np.argwhere(bits(gm) != bits(m))
            assert len(at) == 0, (what, at[:3])
            at = np.argwhere(gc.cpu().numpy() != c)
            assert len(at) == 0, (what, at[:3])
            got = f64(gr)
            assert np.all(got[dropped] == 7), what
            assert np.array_equal(np.isnan(got[~dropped]), np.isnan(want[~dropped])), what
        cu_all, lens_all = np.array([0, 40, 88, 136]), np.array([40, 48, 48])
        gk, gv = F.paged4_read(i32(cu_all), i32(lens_all), i32(tab), *cache, 136)
        for got, (c, m) in ((gk, sides[0]), (gv, sides[1])):
            want, _ = paged4.read(cu_all, lens_all, tab, c, m, 136, fmt)
            got = f64(got)
            ok = np.isfinite(want)
            assert np.array_equal(np.isnan(got), ~ok), what
            assert np.all(np.abs(got - want)[ok] <= 2.0 ** -8 * np.abs(want)[ok] + 2.0 ** -20 * np.abs(want[ok]).max()), what

    def fill_with(f):
        def fill(x):
            x[:] = torch.from_numpy(f(x.shape)).to(x.dtype)
        return fill

    def special(x):
        x[0, 0, 3], x[1, 1, 0], x[2, 0, 40] = float("inf"), float("nan"), float("-inf")

    def borders(shape):                                           # halves of steps of both formats
        x = rng.integers(-12, 13, shape) * 0.25
        x[..., 0::32], x[..., 1::32] = 6.0, -6.0
        return x

    def steps(shape):                                             # 15 steps of a half, and their halves
        x = rng.integers(0, 31, shape) * 0.5
        x[..., 0::32], x[..., 1::32] = 0.0, 15.0
        return x

    step("holes", [40, 40, 20], [40, 40, 20], lambda x: None)     # sequence 0 runs into a page that is not there; 1 has a hole
    step("zeros", [3, 1, 2], [3, 18, 22], fill_with(np.zeros))
    step("negative zeros", [3, 1, 2], [3, 40, 22], fill_with(lambda s: -np.zeros(s)))
    step("constants", [3, 1, 2], [3, 40, 22], fill_with(lambda s: np.full(s, 0.3)))
    step("not finite", [3, 2, 0], [4, 40, 22], special)
    step("after it", [3, 2, 0], [4, 40, 22], lambda x: None)
    step("tiny", [3, 2, 2], [3, 2, 2], lambda x: x.mul_(2.0 ** -30))
    step("half tiny", [3, 2, 2], [3, 2, 2], lambda x: x.mul_(2.0 ** -23))
    step("huge", [3, 2, 2], [3, 2, 2], lambda x: x.mul_(30000.0))
    step("largest", [3, 2, 2], [3, 2, 2], lambda x: x.mul_(1e38))
    step("one sided", [8, 9, 9], [12, 12, 12], fill_with(lambda s: 1000.0 + rng.uniform(0, 4, s)))
    step("powers", [8, 9, 9], [12, 12, 12], fill_with(lambda s: np.exp2(rng.integers(-30, 16, s).astype(float)) * rng.choice([-1, 1], s)))
    for i in range(3):
        step("borders", [16, 16, 16], [16, 16, 16], fill_with(borders))
        step("steps", [16, 16, 16], [16, 16, 16], fill_with(steps))
    step("longer than their sequences", [5, 9, 4], [2, 9, 0], lambda x: None)
    step("beyond the block table", [7, 0, 30], [60, 0, 60], lambda x: None)


def test_append_of_every_key(F):
    """Many values: the fast rounding next to the definition's, on values that lie anywhere."""
    for fmt in ("int4", "e2m1"):
        rng = np.random.default_rng(5)
        T, page, d = 256, 64, 128
        x = torch.from_numpy(rng.normal(size=(T, 1, d)) * np.exp2(rng.integers(-12, 12, (T, 1, d)) * rng.integers(0, 2, (T, 1, 1)))).to(torch.float16)
        cache = F.paged4_cache(4, 1, page, d, fmt)
        F.paged4_append(x.cuda(), x.cuda(), i32([0, T]), i32([T]), i32([[3, 1, 0, 2]]), *cache)
        c, m = paged4.empty(4, 1, page, d, fmt)
        paged4.append(f64(x), np.array([0, T]), np.array([T]), np.array([[3, 1, 0, 2]]), c, m, fmt)
        for g in (0, 1):
            assert np.array_equal(cache[g].cpu().numpy(), c) and np.array_equal(bits(cache[2 + g]), bits(m))


def test_index_checks(F):
    page, H, d = 16, 1, 64
    x = torch.zeros(4, H, d, dtype=torch.float16, device="cuda")
    cache = F.paged4_cache(4, H, page, d)
    F.set_index_checks(True)
    try:
        calls = [lambda cu, lens, tab: F.paged4_append(x, x, i32(cu), i32(lens), i32(tab), *cache),
                 lambda cu, lens, tab: F.paged4_attn(x, i32(cu), i32(lens), i32(tab), *cache),
                 lambda cu, lens, tab: F.paged4_read(i32(cu), i32(lens), i32(tab), *cache, 4)]
        calls[0]([0, 2, 4], [2, 18], [[0, 1], [2, 3]])
        calls[1]([0, 2, 4], [2, 18], [[0, 1], [0, 3]])                       # sequences may share what they read
        calls[2]([0, 2, 4], [2, 18], [[0, 1], [0, -1]])
        for call in calls:
            for cu, lens in (([1, 2, 4], [2, 18]), ([0, 3, 2], [3, 18]), ([0, 2, 5], [2, 18]), ([0, 2, 4], [1, 18]),
                             ([0, 2, 4], [2, 33])):
                with pytest.raises(F.FlashLoopError, match="FL_E_RANGE"):
                    call(cu, lens, [[0, 1], [2, 3]])
        with pytest.raises(F.FlashLoopError, match="appended to twice"):
            calls[0]([0, 2, 4], [2, 18], [[3, 1], [2, 3]])
        with pytest.raises(F.FlashLoopError, match="outside"):
            calls[0]([0, 2, 4], [2, 18], [[0, 1], [2, -1]])
    finally:
        F.set_index_checks(False)


# ---- attention ---------------------------------------------------------------------------------------------
def spoil_numbers(m, where, fmt):
    m[where] = np.nan if fmt == "int4" else 255


def check_attn(F, rng, new, past, page, Hq, Hkv, d, dtype, fmt, layout=None, rot=0, window=0, n_sink=0, hints=((None, 0),),
               holes=(), spoil=False, amp=1.0, edit=None, lse=True):
    cu, lens, tab, n_pages = batch(rng, new, past, page, holes=holes)
    T = int(cu[-1]) + 2
    dt = DT[dtype]
    sides = [paged4.empty(n_pages, Hkv, page, d, fmt, rng) for _ in range(2)]
    if edit:
        edit(sides, tab)
    if spoil:              # what lies behind a sequence's end, and pages of nobody: numbers that read as NaN
        for b, L in enumerate(lens):
            if L % page and tab[b, L // page] >= 0:
                for _, m in sides:
                    spoil_numbers(m, (tab[b, L // page], slice(None), slice(L % page, None)), fmt)
        mine = set(tab[tab >= 0].tolist())
        for p in set(range(n_pages)) - mine:
            for _, m in sides:
                spoil_numbers(m, p, fmt)
    q = torch.from_numpy(rng.normal(size=(T, 2 * Hq * d)) * amp).to(dt)
    part = q.cuda()[:, Hq * d:].view(T, Hq, d)
    qx = f64(q)[:, Hq * d:].reshape(T, Hq, d)
    cs = None
    if layout:
        cs = paged.table(tab.shape[1] * page, rot).astype(np.float32)
        pos = np.concatenate([np.arange(lens[b] - new[b], lens[b]) for b in range(len(new))] + [np.zeros(2, int)]).astype(int)
        qx = paged.rotate(qx, cs[np.clip(pos, 0, len(cs) - 1)], layout)
    want, wlse, av, aq, aw = paged4.attend(qx, paged4.paged_seqs(cu, lens, tab, sides, fmt), Hkv, d ** -0.5, window, n_sink)
    args = (i32(cu), i32(lens), i32(tab), up(sides[0][0]), up(sides[1][0]), up(sides[0][1]), up(sides[1][1]))
    n = int(cu[-1])
    for max_q, max_len in hints:
        out = torch.full((T, 3 * Hq * d), 7.0, dtype=dt, device="cuda")
        o = out[:, Hq * d:2 * Hq * d].view(T, Hq, d)
        L = torch.full((T, Hq), 7.0, device="cuda") if lse else None
        F.paged4_attn(part, *args, table=None if cs is None else torch.from_numpy(cs).cuda(), layout=layout or "half",
                      window=window, n_sink=n_sink, max_q=max_q, max_len=max_len, out=o, lse=L)
        torch.cuda.synchronize()
        got = f64(o)
        assert np.all(got[n:] == 7) and torch.all(out[:, :Hq * d] == 7) and torch.all(out[:, 2 * Hq * d:] == 7)
        fin = np.isfinite(want[:n])
        what = f"new={list(new)[:5]} past={list(past)[:5]} page={page} {Hq}/{Hkv}x{d} {dtype} {fmt} w={window}+{n_sink} hint={max_q},{max_len}"
        at = np.argwhere(np.isnan(got[:n]) != ~fin)
        assert len(at) == 0, f"{len(at)} NaN where none belongs or the other way round, first at {at[0]}, {what}"
        keys = int(max(lens))
        wide = 2.0 ** -11 if fmt == "int4" else 0.0
        e = (2.0 ** -11 + wide + (d + 8) * 2.0 ** -23) * aq[:n]
        acc = (keys + d) * 2.0 ** -23
        with np.errstate(invalid="ignore"):
            tol = (2 * e[..., None] + 2.0 ** -11 + wide + acc) * av[:n] + 2.0 ** -25 * aw[:n] + half_step(dt) * np.abs(want[:n]) + 2.0 ** -24
            err = np.abs(got[:n] - want[:n])[fin]
        den = np.linalg.norm(want[:n][fin])
        rel = np.linalg.norm(err) / den if den else 0.0
        say(f"  {what}: rel={rel:.2e} worst={np.max(err / np.maximum(tol[fin], 1e-30)) if err.size else 0:.2f} of tol")
        assert np.all(err <= tol[fin])
        assert rel <= REL_FRO + half_step(dt)
        if lse:
            gl = f64(L)
            assert np.all(gl[n:] == 7)
            none = np.isneginf(wlse[:n])
            assert np.array_equal(np.isneginf(gl[:n]), none)
            ok = np.isfinite(wlse[:n]) & fin.all(axis=-1)
            assert np.all(np.abs(gl[:n][ok] - wlse[:n][ok]) <= (e + acc + 2.0 ** -20 * (1 + np.abs(wlse[:n])))[ok])
    return part, args


ATTN = [
    # new, past, page, Hq, Hkv, window, n_sink
    ([1], [0], 16, 1, 1, 0, 0),
    ([1], [299], 64, 16, 16, 0, 0),
    ([1, 1, 0, 1], [16, 15, 40, 17], 16, 6, 2, 0, 0),
    ([3, 0, 4, 1], [700, 0, 31, 1300], 32, 8, 1, 0, 0),
    ([2, 2], [500, 65], 128, 4, 4, 64, 4),
    ([1, 1, 1], [1000, 30, 200], 64, 8, 2, 100, 5),
    ([1, 2], [900, 400], 16, 3, 1, 1, 0),
    ([40], [0], 64, 2, 2, 0, 0),
    ([129, 1, 64], [0, 77, 300], 32, 6, 3, 0, 0),
    ([257, 30], [130, 5], 64, 4, 1, 96, 17),
    ([300], [20], 16, 2, 1, 33, 70),
    ([70, 90, 0], [513, 0, 12], 128, 5, 5, 0, 0),
    ([1] * 100 + [0] * 20 + [3] * 10, [7 * i % 211 for i in range(129)] + [1500], 16, 2, 1, 0, 0),     # more than 64 sequences
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "int4"), ("f16", "e2m1"), ("bf16", "e2m1"), ("f16", "int4")])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(F, case, dtype, fmt, d):
    new, past, page, Hq, Hkv, window, n_sink = ATTN[case]
    rng = np.random.default_rng(100 + case)
    layout, rot = [(None, 0), ("half", d), ("interleaved", d // 2), ("half", 16)][(case + d // 64) % 4]
    check_attn(F, rng, new, past, page, Hq, Hkv, d, dtype, fmt, layout, rot, window, n_sink,
               hints=((None, 0), (1, 5000), (1000, 1), (1000, 5000)), spoil=True)


@pytest.mark.parametrize("dtype,fmt,d,page,window,n_sink", [("bf16", "int4", 128, 64, 0, 0), ("f16", "e2m1", 64, 32, 700, 40),
                                                            ("bf16", "e2m1", 128, 16, 1500, 4), ("f16", "int4", 64, 128, 0, 0)])
def test_attention_of_long_chunks(F, dtype, fmt, d, page, window, n_sink):
    """Many row tiles over long contexts: shares of the work that begin and end inside row tiles, of one sequence and between
    sequences; also with a hint that leaves each tile to a workgroup, and with the kernel for few rows."""
    rng = np.random.default_rng(12)
    check_attn(F, rng, [300, 0, 1, 170], [1200, 50, 2000, 3], page, 4, 2, d, dtype, fmt, "half", d, window, n_sink,
               hints=((300, 2001), (300, 500), (300, 0), (1, 2001)), spoil=True)
    check_attn(F, rng, [33, 0, 64, 1], [2500, 0, 1100, 3], page, 2, 1, d, dtype, fmt, "half", d, window, n_sink,
               hints=((64, 2533),), spoil=True)


@pytest.mark.parametrize("dtype,fmt,d,page,window,n_sink", [("bf16", "int4", 128, 64, 0, 0), ("f16", "e2m1", 64, 32, 2600, 40),
                                                            ("bf16", "e2m1", 128, 16, 3000, 130), ("f16", "int4", 64, 128, 0, 0)])
def test_attention_of_chunks_after_long_contexts(F, dtype, fmt, d, page, window, n_sink):
    """Few row tiles over thousands of keys: shares as above, with and without a window."""
    rng = np.random.default_rng(23)
    check_attn(F, rng, [300, 0, 1, 170], [4200, 50, 5000, 3], page, 4, 2, d, dtype, fmt, "half", d, window, n_sink,
               hints=((300, 5001), (300, 0)), spoil=True, holes=((0, 40), (2, 3)))
    check_attn(F, rng, [33, 0, 64, 1], [3000, 0, 2500, 3], page, 2, 1, d, dtype, fmt, "half", d, window, n_sink,
               hints=((64, 3033),), spoil=True)


def test_thousands_of_sequences(F):
    """More sequences than a search looks at in one or two rounds, many of them without a row."""
    rng = np.random.default_rng(14)
    B, page, d = 5000, 16, 64
    new = (np.arange(B) % 3 > 0).astype(int)
    new[[0, 17, 4097, B - 1]] = [0, 20, 33, 0]
    past = np.arange(B) % 40
    check_attn(F, rng, new, past, page, 2, 1, d, "bf16", "int4", hints=((None, 0), (33, 73), (1, 73)), spoil=True)


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
@pytest.mark.parametrize("d", [64, 128])
def test_holes_empty_rows_and_lengths(F, fmt, d):
    """Pages that are not there, lengths below the new positions, of zero, and beyond the block table."""
    rng = np.random.default_rng(15)
    check_attn(F, rng, [2, 40, 1], [100, 60, 0], 16, 4, 2, d, "bf16", fmt, holes=((0, 0), (0, 3), (1, 0), (1, 1), (1, 5), (2, 0)),
               hints=((None, 0), (1, 0), (100, 0)), spoil=True)

    def odd(lens):
        cu, tab = [0, 3, 43, 44], rng.permutation(12).reshape(3, 4)
        sides = [paged4.empty(12, 1, 16, d, fmt, rng) for _ in range(2)]
        q = torch.from_numpy(rng.normal(size=(44, 2, d))).to(torch.float16)
        want, wlse, *_ = paged4.attend(f64(q), paged4.paged_seqs(cu, lens, tab, sides, fmt), 1, d ** -0.5)
        cache = [up(sides[0][0]), up(sides[1][0]), up(sides[0][1]), up(sides[1][1])]
        for max_q in (1, 16, 100):
            L = torch.empty(44, 2, device="cuda")
            got = f64(F.paged4_attn(q.cuda(), i32(cu), i32(lens), i32(tab), *cache, max_q=max_q, lse=L))
            assert np.abs(got - want).max() <= 2e-2 * np.abs(want).max()
            assert np.array_equal(np.isneginf(f64(L)), np.isneginf(wlse))
    odd([2, 20, 0])
    odd([0, 39, 64])
    odd([64, 64, 1])
    odd([70, 90, 100])


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
@pytest.mark.parametrize("d", [64, 128])
def test_groups_that_read_as_nan(F, fmt, d):
    """A spoilt group makes exactly the rows that see its position NaN, in single positions, several and chunks, across split keys."""
    rng = np.random.default_rng(16)
    page = 16

    def edit(where):
        def put(sides, tab):
            for side, b, pos, h, g in where:
                spoil_numbers(sides[side][1], (tab[b, pos // page], h, pos % page, g), fmt)
                if fmt == "int4":                                  # the other ways of being none
                    sides[side][1][tab[b, pos // page], h, pos % page, g] = [(np.nan, 0), (1, np.inf), (-1, 0), (4376, 0), (1, 40000)][(pos + g) % 5]
                else:
                    sides[side][1][tab[b, pos // page], h, pos % page, g] = [255, 0, 103, 141, 254][(pos + g) % 5]
        return put
    last = d // 32 - 1
    for new, past, where in (([4], [60], [(1, 0, 62, 0, last)]), ([4], [60], [(0, 0, 61, 1, 0)]), ([1, 1], [900, 40], [(1, 0, 500, 0, 0)]),
                             ([200, 3], [100, 90], [(1, 0, 250, 1, last), (0, 0, 150, 0, 0), (1, 1, 91, 0, 0)]),
                             ([3, 3], [2000, 1200], [(1, 0, 2001, 0, 0), (1, 1, 3, 1, last)])):
        for window, n_sink in ((0, 0), (64, 2)):
            check_attn(F, rng, new, past, page, 4, 2, d, "bf16", fmt, window=window, n_sink=n_sink, edit=edit(where),
                       hints=((None, 0), (1, 0), (200, 0)))


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_of_any_bytes(F, fmt, d):
    """Pages that were never cleared: every byte that no sequence holds is random, single numbers of it within their bounds and
    groups beyond them among it; and such groups where rows do see them."""
    rng = np.random.default_rng(20)

    def edit(sides, tab):
        for c, m in sides:
            c[:] = np.frombuffer(rng.bytes(c.size), np.uint8).reshape(c.shape)
            raw, keep = m.view(np.uint8), m.copy()
            raw[:] = np.frombuffer(rng.bytes(raw.size), np.uint8).reshape(raw.shape)
            if fmt == "int4":
                m[rng.random(m.shape[:-1]) < 0.3] = (4372, 32768)
            for b, L in enumerate(lens):                       # what the sequences hold
                for p in range(-(-L // page)):
                    m[tab[b, p], :, :L - p * page] = keep[tab[b, p], :, :L - p * page]
    page = 64
    for new, past in (([1, 2, 1], [700, 30, 0]), ([90, 1, 64], [301, 5, 64]), ([500, 3], [37, 2])):
        lens = [a + b for a, b in zip(new, past)]
        for window, n_sink in ((0, 0), (40, 3)):
            check_attn(F, rng, new, past, page, 4, 2, d, "bf16", fmt, window=window, n_sink=n_sink, edit=edit,
                       hints=((None, 0), (1, 0), (200, 0)))
    if fmt == "int4":
        def edge(sides, tab):                                  # just within, just beyond
            for i, (_, m) in enumerate(sides):
                m[tab[0, 4], 0, 3, 0] = [(2182, 32768), (2184, 32768)][i]
        check_attn(F, rng, [3, 300], [600, 1], page, 4, 2, d, "bf16", fmt, edit=edge, hints=((None, 0), (1, 0), (200, 0)))


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_values_of_any_size(F, fmt):
    """Groups whose values differ by far side by side, and as large and as small as the format has them."""
    rng = np.random.default_rng(17)

    def edit(sides, tab):
        for _, m in sides[1:]:
            if fmt == "int4":
                s = np.exp2(rng.uniform(-24, 12, m.shape[:-1]))
                m[..., 0] = s
                m[..., 1] = -np.minimum(s * rng.uniform(0, 15, s.shape), 32768)
            else:
                m[:] = rng.integers(104, 141, m.shape)
    for dtype in ("bf16",):
        check_attn(F, rng, [1, 60], [800, 100], 16, 4, 2, 128, dtype, fmt, edit=edit, hints=((None, 0), (1, 0), (60, 0)))


def test_queries_of_any_size(F):
    rng = np.random.default_rng(18)
    for fmt in ("int4", "e2m1"):
        for amp in (0.0, 2.0 ** -12, 20.0):
            check_attn(F, rng, [1, 40], [300, 20], 16, 4, 2, 64, "f16", fmt, "half", 64, amp=amp, hints=((None, 0), (1, 0)))
    q = torch.randn(2, 2, 64, device="cuda").to(torch.bfloat16)
    q[0, 0, 3], q[1, 1, 0] = float("nan"), float("-inf")
    cache = F.paged4_cache(4, 1, 16, 64)
    x = torch.randn(40, 1, 64, device="cuda").to(torch.bfloat16)
    F.paged4_append(x, x, i32([0, 40]), i32([40]), i32([[0, 1, 2, 3]]), *cache)
    for max_q in (1, 100):
        got = F.paged4_attn(q, i32([0, 2]), i32([40]), i32([[0, 1, 2, 3]]), *cache, max_q=max_q)
        assert torch.isnan(got[0, 0]).all() and torch.isnan(got[1, 1]).all() and torch.isfinite(got[0, 1]).all() and torch.isfinite(got[1, 0]).all()


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_far_positions(F, fmt):
    """A position and a chunk after hundreds of thousands, with and without a window, however the call is hinted."""
    rng = np.random.default_rng(21)
    for window, n_sink in ((0, 0), (5000, 70)):
        check_attn(F, rng, [1, 2], [300000, 17], 64, 4, 1, 64, "bf16", fmt, window=window, n_sink=n_sink, hints=((None, 0), (1, 300001), (200, 0)))
        check_attn(F, rng, [130, 1], [100000, 77], 128, 1, 1, 128, "f16", fmt, window=window, n_sink=n_sink, hints=((None, 0), (1, 0)))


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_empty_calls_and_one_side_alone(F, fmt):
    """Calls without rows write nothing; one side's rows can be had without the other's."""
    rng = np.random.default_rng(22)
    H, d, page, T = 3, 64, 16, 21
    cache = F.paged4_cache(4, H, page, d, fmt)
    for c in cache:
        c.view(torch.uint8).fill_(5)
    before = [c.clone() for c in cache]
    tab, none = i32([[2, 0]]), torch.empty(0, H, d, dtype=torch.bfloat16, device="cuda")
    F.paged4_append(none, none, i32([0, 0]), i32([9]), tab, *cache, k_rows=none, v_rows=none)
    F.paged4_read(i32([0, 0]), i32([9]), tab, *cache, 0)
    assert F.paged4_attn(none, i32([0, 0]), i32([9]), tab, *cache).shape == none.shape
    assert F.packed_attn(none, none, none, i32([0, 0])).shape == none.shape
    torch.cuda.synchronize()
    assert all(torch.equal(bits_t(a), bits_t(b)) for a, b in zip(cache, before))
    k, v = (torch.from_numpy(rng.normal(size=(T, H, d))).to(torch.bfloat16).cuda() for _ in range(2))
    batch_of = (i32([0, T]), i32([T]), tab)
    kr, vr, k1, v1 = (torch.full_like(k, 7.0) for _ in range(4))
    F.paged4_append(k, v, *batch_of, *cache, k_rows=kr, v_rows=vr)
    F.paged4_append(k, v, *batch_of, *cache, k_rows=k1)
    F.paged4_append(k, v, *batch_of, *cache, v_rows=v1)
    assert torch.equal(k1, kr) and torch.equal(v1, vr)
    # rows that see no key at all: the sequence has none
    q = torch.ones(2, H, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(2, H, device="cuda")
    assert torch.all(F.packed_attn(q, none, none, i32([0, 2]), i32([0, 0]), lse=lse) == 0) and torch.all(lse == -float("inf"))


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
@pytest.mark.parametrize("d", [64, 128])
def test_fp16_outputs_are_half_as_far_off_again(F, fmt, d):
    """Ordinary numbers, keys and values as appended: besides an output's own rounding to fp16 only one more rounding of the same relative
    size is in it (the probabilities', or the values'), so the norm of its error is at most sqrt(2) times, with 6 % for the rest 1.5
    times, that of rounding the exact output."""
    rng = np.random.default_rng(24)
    page, Hkv, Hq = 64, 2, 8
    for new, past in (([1, 1, 1], [900, 30, 5]), ([4, 2], [300, 60]), ([8], [500]), ([150, 40], [0, 400])):
        cu, lens, tab, n_pages = batch(rng, new, past, page)
        sides = [paged4.empty(n_pages, Hkv, page, d, fmt) for _ in range(2)]
        at = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        for c, m in sides:
            paged4.append(rng.normal(size=(int(at[-1]), Hkv, d)), at, lens, tab, c, m, fmt)
        q = torch.from_numpy(rng.normal(size=(int(cu[-1]), Hq, d))).half()
        want = paged4.attend(f64(q), paged4.paged_seqs(cu, lens, tab, sides, fmt), Hkv, d ** -0.5)[0]
        least = np.linalg.norm(want.astype(np.float16).astype(np.float64) - want)
        for max_q in (None, 8, 100):
            got = F.paged4_attn(q.cuda(), i32(cu), i32(lens), i32(tab), up(sides[0][0]), up(sides[1][0]), up(sides[0][1]), up(sides[1][1]),
                                max_q=max_q)
            err = np.linalg.norm(f64(got) - want)
            say(f"  {new} after {past} d={d} {fmt} max_q={max_q}: {err / least:.2f} times the rounding's")
            assert err <= 1.5 * least
