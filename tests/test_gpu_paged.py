"""Rotary positions, the paged 8-bit cache and dense attention over it: the HIP path against the fp64 oracle.

Tolerances.  Rotations are rounded once to their type from fp32 sums of two rounded products: half a step of the type plus
2^-22 (|x0 c| + |x1 s|).  Codes and scales are equal.  Attention: with fp16 queries each |q_e| is off by at most 2^-11 of
itself (2^-25 of the row's largest below its normal range), so a score by e = 2^-11 A, A = max_j sm_scale sum |q_e k_je|, a
probability by 2 e of itself, and it is rounded to fp16: 2^-11 of itself, or 2^-25 of the unit below fp16's normal range.  The unit
is at most the row's largest contribution w = max_j p_j s_j (s_j the value's scale: the kernels round p_j s_j over a running
maximum of it), so those roundings add up to 2^-25 w sum_j |c_j| over the value's codes c_j; where the keys that carry a row have
the code 0 in a channel, that is what remains of it.  The output's own rounding adds half a step.  fp32 sums add at most
(n + d) 2^-23 to either."""
import numpy as np
import pytest
import torch

from gpu_util import REL_FRO, say
from oracle import paged

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
FMT = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def raw(t):
    return t.view(torch.uint8).cpu().numpy()


def f64(t):
    return t.cpu().double().numpy()


def dev_codes(a, fmt):
    return torch.from_numpy(a.copy()).cuda().view(FMT[fmt])


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


# ---- rotary positions -----------------------------------------------------------------------------------
@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=3.5), dict(scaling="ntk", factor=8.0, base=5e5),
                                dict(scaling="yarn", factor=4.0, orig_len=4096), dict(scaling="yarn", factor=1.0, orig_len=64)])
@pytest.mark.parametrize("n_pos,rot", [(1, 16), (1000, 64), (9001, 96), (70001, 128)])
def test_rope_table(F, n_pos, rot, kw):
    say(f"table n_pos={n_pos} rot={rot} {kw}")
    got = F.rope_table(n_pos, rot, **kw)
    torch.cuda.synchronize()
    want = paged.table(n_pos, rot, **kw)
    m = paged.frequencies(rot, **kw)[1]
    assert got.shape == want.shape
    # 2 ulp of m, and fp64 angles whose frequency is known to 2^-50 of itself
    tol = 2.0 ** -22 * m + n_pos * 2.0 ** -49
    assert np.abs(f64(got) - want).max() <= tol
    assert torch.equal(F.rope_table(n_pos, rot, out=torch.empty_like(got), **kw), got)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,d,rot", [(1, 1, 16, 16), (5, 3, 64, 32), (77, 16, 128, 128), (300, 5, 128, 48), (64, 2, 200, 96),
                                       (1025, 12, 64, 64)])
def test_rope(F, T, H, d, rot, layout, dtype):
    say(f"rope {T} x {H} x {d} rot {rot} {layout} {dtype}")
    dt = DT[dtype]
    g = torch.Generator().manual_seed(T + d)
    x = torch.randn(T, 3 * H * d, generator=g).to(dt)
    cs = paged.table(400, rot).astype(np.float32)
    pos = torch.randint(0, 400, (T,), generator=g, dtype=torch.int32)
    part = x.cuda()[:, H * d:2 * H * d].view(T, H, d)
    xs = f64(x)[:, H * d:2 * H * d].reshape(T, H, d)
    tab = torch.from_numpy(cs).cuda()
    for inverse in (False, True):
        got = F.rope(part, tab, pos.cuda(), layout=layout, inverse=inverse)
        want = paged.rotate(xs, cs[pos.numpy()], layout, inverse)
        mag = paged.rotate(np.abs(xs), np.abs(cs[pos.numpy()]) * [1, -1], layout)
        mag = np.maximum(np.abs(mag), np.abs(paged.rotate(np.abs(xs), np.abs(cs[pos.numpy()]), layout)))
        err = np.abs(f64(got) - want)
        assert np.all(err <= half_step(dt) * np.abs(want) + 2.0 ** -22 * mag + (2.0 ** -24 if dtype == "f16" else 0))
        assert torch.equal(got[..., rot:], part[..., rot:])
    # in place within a fused row, the neighbours untouched
    whole = x.cuda()
    at = whole[:, H * d:2 * H * d].view(T, H, d)
    assert F.rope(at, tab, pos.cuda(), layout=layout, out=at) is at
    assert torch.equal(at, F.rope(part, tab, pos.cuda(), layout=layout))
    assert torch.equal(whole[:, :H * d].cpu(), x[:, :H * d]) and torch.equal(whole[:, 2 * H * d:].cpu(), x[:, 2 * H * d:])
    if T <= 400:                                            # without positions: 0 .. T-1
        assert torch.equal(F.rope(part, tab, layout=layout), F.rope(part, tab, i32(np.arange(T)), layout=layout))


def test_rope_gradient(F):
    """The inverse is the gradient, in 16 bits: <w, rope(x)> and <rope^-1(w), x> agree, and it meets differences."""
    T, H, d, rot = 33, 2, 64, 64
    g = torch.Generator().manual_seed(0)
    x, w = (torch.randn(T, H, d, generator=g).to(torch.float16) for _ in range(2))
    tab = F.rope_table(T, rot, scaling="yarn", factor=2.0, orig_len=16)
    y, grad = F.rope(x.cuda(), tab), F.rope(w.cuda(), tab, inverse=True)
    a, b = (f64(y) * f64(w)).sum(), (f64(grad) * f64(x)).sum()
    # each of the T H d terms is off by half a step of the rotated value, of magnitude at most 1.07 * sqrt(2) * max
    bound = 2 * T * H * d * 2.0 ** -11 * float(x.abs().max()) * float(w.abs().max()) * 1.07 * 2 ** 0.5
    assert abs(a - b) <= bound
    want = paged.rotate(f64(w), f64(tab), "half", inverse=True)
    assert np.all(np.abs(f64(grad) - want) <= 2.0 ** -11 * np.abs(want) + 2.0 ** -19)
    # differences: a step of 1 in one value moves <w, rope(x)> by that value's gradient
    for at in [(0, 0, 0), (7, 1, 5), (32, 0, 63)]:
        up, dn = x.clone(), x.clone()
        up[at] += 0.5
        dn[at] -= 0.5
        step = float(up[at]) - float(dn[at])
        num = (f64(w) * (f64(F.rope(up.cuda(), tab)) - f64(F.rope(dn.cuda(), tab)))).sum() / step
        assert abs(num - want[at]) <= 4 * 2.0 ** -11 * 8 * 1.07 * float(w.abs().max())


def test_rope_positions_out_of_range(F):
    x = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    tab = F.rope_table(8, 32)
    got = F.rope(x, tab, i32([0, 8, -1, 7]))
    bad = torch.isnan(got).cpu()
    assert bad[1:3, :, :32].all() and not bad[[0, 3]].any() and not bad[:, :, 32:].any()
    F.set_index_checks(True)
    try:
        with pytest.raises(F.FlashLoopError, match="pos"):
            F.rope(x, tab, i32([0, 8, -1, 7]))
        F.rope(x, tab, i32([0, 1, 2, 7]))
    finally:
        F.set_index_checks(False)


# ---- appending ---------------------------------------------------------------------------------------------
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
    ([200, 5], [1, 127], 128, 2, 128, 128),
    ([130, 64, 65], [0, 0, 63], 64, 5, 64, 48),
    ([1] * 70, list(range(70)), 64, 1, 128, 128),
    ([1, 0, 2, 0, 0, 0, 0, 50, 1], [5, 3, 31, 0, 1, 2, 3, 9, 100], 64, 2, 64, 32),    # few on average, many for one
    ([23, 1, 1, 1], [8, 127, 128, 1], 128, 3, 128, 64),
]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,layout", [("bf16", "half"), ("f16", "interleaved"), ("bf16", None)])
@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append(F, case, dtype, layout, fmt):
    new, past, page, H, d, rot = APPENDS[case]
    say(f"append case {case} {dtype} {layout} {fmt}")
    rng = np.random.default_rng(case)
    cu, lens, tab, n_pages = batch(rng, new, past, page)
    T = cu[-1] + 3                                         # three rows of no sequence
    dt = DT[dtype]
    size = np.exp(rng.normal(size=(T, H, 1)) * 1.5)        # later positions outgrow earlier ones
    k, v = (torch.from_numpy(rng.normal(size=(T, H, d)) * size).to(dt) for _ in range(2))
    k[cu[-1]:] = float("nan")
    rows = torch.cat((k, v), dim=1).cuda()
    kd, vd = rows[:, :H], rows[:, H:]
    codes = [np.frombuffer(rng.bytes(n_pages * H * page * d), np.uint8).reshape(n_pages, H, page, d).copy() for _ in range(2)]
    if fmt == "e4m3":
        codes = [np.where((c & 127) == 127, 3, c) for c in codes]
    else:
        codes = [np.where(c == 128, 129, c).astype(np.uint8) for c in codes]
    scale = [np.exp2(rng.integers(-9, -4, (n_pages, H))).astype(np.float32) for _ in range(2)]
    if fmt == "int8":
        scale = [(s * rng.uniform(1, 2, s.shape)).astype(np.float32) for s in scale]
    cs = paged.table(tab.shape[1] * page, rot).astype(np.float32)
    gc, gs = [dev_codes(c, fmt) for c in codes], [torch.from_numpy(s.copy()).cuda() for s in scale]
    F.paged_append(kd, vd, i32(cu), i32(lens), i32(tab), *gc, *gs, table=None if layout is None else torch.from_numpy(cs).cuda(),
                   layout=layout or "half")
    torch.cuda.synchronize()
    kx = f64(k)
    if layout:
        pos = np.concatenate([np.arange(lens[b] - new[b], lens[b]) for b in range(len(new))] + [np.zeros(3, int)]).astype(int)
        with np.errstate(invalid="ignore"):
            kx = paged.rotate(kx, cs[pos], layout).astype(np.float32).astype(np.float64)
    for x, c, s, g, h in ((kx, codes[0], scale[0], gc[0], gs[0]), (f64(v), codes[1], scale[1], gc[1], gs[1])):
        paged.append(x, cu, lens, tab, c, s, fmt)
        assert np.array_equal(h.cpu().numpy(), s)
        same = raw(g) == c
        assert same.all(), f"{(~same).sum()} codes differ, first at {np.argwhere(~same)[0]}"


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_edges(F, fmt):
    """Zeros, tiny values, infinities and NaN, an exact border, pages that are not there, negative starts."""
    page, H, d = 16, 2, 64
    say(f"append edges {fmt}")
    tab = np.array([[0, 1, -1], [2, 99, 3], [4, 5, 6]], np.int32)
    codes = [np.full((8, H, page, d), 17, np.uint8) for _ in range(2)]
    scale = [np.full((8, H), 0.25, np.float32) for _ in range(2)]
    scale[0][5] = 0
    scale[1][5] = np.nan
    gc, gs = [dev_codes(c, fmt) for c in codes], [torch.from_numpy(s.copy()).cuda() for s in scale]
    rng = np.random.default_rng(0)

    def step(new, lens, fill):
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T = int(cu[-1]) + 1
        x = torch.from_numpy(rng.normal(size=(T, H, d))).to(torch.bfloat16)
        fill(x)
        F.paged_append(x.cuda(), (-x).cuda(), i32(cu), i32(lens), i32(tab), *gc, *gs)
        torch.cuda.synchronize()
        for y, c, s, g, h in ((f64(x), codes[0], scale[0], gc[0], gs[0]), (-f64(x), codes[1], scale[1], gc[1], gs[1])):
            paged.append(y, cu, lens, tab, c, s, fmt)
            assert np.array_equal(h.cpu().numpy(), s, equal_nan=True)
            assert np.array_equal(raw(g), c)

    def zeros(x):
        x[:] = 0

    def special(x):
        x[0, 0, 3], x[1, 1, 0], x[2, 0, 9] = float("inf"), float("nan"), float("-inf")

    def tiny(x):
        x *= 2.0 ** -105
        x[0, 0, 0] = 2.0 ** -100

    def border(x):
        x[:] = 0
        x[:, :, 5] = 448.0 if fmt == "e4m3" else 127.0

    step([40, 40, 20], [40, 40, 20], lambda x: None)        # sequence 0 runs into a page that is not there; 1 has a hole
    step([3, 1, 2], [3, 18, 22], zeros)
    step([1, 2, 0], [4, 40, 22], special)
    step([1, 1, 1], [5, 41, 23], lambda x: None)            # a NaN scale stays
    step([3, 2, 2], [3, 2, 2], tiny)
    step([2, 3, 1], [5, 5, 3], border)
    step([2, 3, 1], [7, 8, 4], border)                      # the same magnitude again: the scale stays
    step([5, 9, 4], [2, 9, 0], lambda x: None)              # longer than their sequences: the first positions are dropped
    step([7, 0, 30], [60, 0, 60], lambda x: None)           # beyond the block table


def test_index_checks(F):
    page, H, d = 16, 1, 64
    x = torch.zeros(4, H, d, dtype=torch.float16, device="cuda")
    cache = F.paged_cache(4, H, page, d)
    F.set_index_checks(True)
    try:
        def app(cu, lens, tab):
            F.paged_append(x, x, i32(cu), i32(lens), i32(tab), *cache)

        def att(cu, lens, tab):
            F.paged_attn(x, i32(cu), i32(lens), i32(tab), *cache)
        app([0, 2, 4], [2, 18], [[0, 1], [2, 3]])
        att([0, 2, 4], [2, 18], [[0, 1], [0, 3]])                       # sequences may share what they read
        for call in (app, att):
            for cu, lens in (([1, 2, 4], [2, 18]), ([0, 3, 2], [3, 18]), ([0, 2, 5], [2, 18]), ([0, 2, 4], [1, 18]),
                             ([0, 2, 4], [2, 33])):
                with pytest.raises(F.FlashLoopError, match="FL_E_RANGE"):
                    call(cu, lens, [[0, 1], [2, 3]])
        with pytest.raises(F.FlashLoopError, match="appended to twice"):
            app([0, 2, 4], [2, 18], [[3, 1], [2, 3]])
        with pytest.raises(F.FlashLoopError, match="outside"):
            app([0, 2, 4], [2, 18], [[0, 1], [2, -1]])
    finally:
        F.set_index_checks(False)


# ---- attention ---------------------------------------------------------------------------------------------
def make_cache(rng, n_pages, H, page, d, fmt, spread=1.0):
    codes = []
    for _ in range(2):
        x = rng.normal(size=(n_pages, H, page, d)) * (40 if fmt == "int8" else 30)
        codes.append(paged.encode(np.clip(x, -127, 127), fmt))
    scale = [(np.exp(rng.normal(size=(n_pages, H)) * spread) * 0.025).astype(np.float32) for _ in range(2)]
    return codes, scale


def check_attn(F, rng, new, past, page, Hq, Hkv, d, dtype, fmt, layout=None, rot=0, window=0, n_sink=0, hints=((None, 0),),
               holes=(), spoil=False, spread=1.0, amp=1.0, scale_edit=None, lse=True):
    cu, lens, tab, n_pages = batch(rng, new, past, page, holes=holes)
    T = int(cu[-1]) + 2
    dt = DT[dtype]
    codes, scale = make_cache(rng, n_pages, Hkv, page, d, fmt, spread)
    if scale_edit:
        scale_edit(scale, tab)
    if spoil:              # what lies behind a sequence's end, and pages of nobody: NaN codes, NaN and infinite scales
        for b, L in enumerate(lens):
            if L % page and tab[b, L // page] >= 0:
                for c in codes:
                    c[tab[b, L // page], :, L % page:] = 127
        mine = set(tab[tab >= 0].tolist())
        for p in set(range(n_pages)) - mine:
            codes[0][p], codes[1][p] = 255, 127
            scale[0][p], scale[1][p] = np.nan, np.inf
    q = torch.from_numpy(rng.normal(size=(T, 2 * Hq * d)) * amp).to(dt)
    part = q.cuda()[:, Hq * d:].view(T, Hq, d)
    qx = f64(q)[:, Hq * d:].reshape(T, Hq, d)
    cs = None
    if layout:
        cs = paged.table(tab.shape[1] * page, rot).astype(np.float32)
        pos = np.concatenate([np.arange(lens[b] - new[b], lens[b]) for b in range(len(new))] + [np.zeros(2, int)]).astype(int)
        qx = paged.rotate(qx, cs[pos], layout)
    want, wlse, av, aq, aw = paged.attend(qx, cu, lens, tab, *codes, *scale, fmt, d ** -0.5, window, n_sink)
    args = (i32(cu), i32(lens), i32(tab), dev_codes(codes[0], fmt), dev_codes(codes[1], fmt),
            torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda())
    n = int(cu[-1])
    for max_q, max_len in hints:
        out = torch.full((T, 3 * Hq * d), 7.0, dtype=dt, device="cuda")
        o = out[:, Hq * d:2 * Hq * d].view(T, Hq, d)
        L = torch.full((T, Hq), 7.0, device="cuda") if lse else None
        F.paged_attn(part, *args, table=None if cs is None else torch.from_numpy(cs).cuda(), layout=layout or "half",
                     window=window, n_sink=n_sink, max_q=max_q, max_len=max_len, out=o, lse=L)
        torch.cuda.synchronize()
        got = f64(o)
        assert np.all(got[n:] == 7) and torch.all(out[:, :Hq * d] == 7) and torch.all(out[:, 2 * Hq * d:] == 7)
        fin = np.isfinite(want[:n])
        assert np.array_equal(np.isnan(got[:n]), np.isnan(want[:n])), f"NaN where none belongs, hints {max_q} {max_len}"
        keys = int(max(lens))
        e = 2.0 ** -11 * aq[:n]
        acc = (keys + d) * 2.0 ** -23
        tol = (2 * e[..., None] + 2.0 ** -10 + acc) * av[:n] + 2.0 ** -25 * aw[:n] + half_step(dt) * np.abs(want[:n]) + 2.0 ** -24
        err = np.abs(got[:n] - want[:n])[fin]
        den = np.linalg.norm(want[:n][fin])
        rel = np.linalg.norm(err) / den if den else 0.0
        say(f"  new={list(new)[:5]} past={list(past)[:5]} page={page} {Hq}/{Hkv}x{d} {dtype} {fmt} w={window}+{n_sink} "
            f"hint={max_q},{max_len}: rel={rel:.2e} worst={np.max(err / np.maximum(tol[fin], 1e-30)) if err.size else 0:.2f} of tol")
        assert np.all(err <= tol[fin])
        assert rel <= REL_FRO + half_step(dt)
        if lse:
            gl = f64(L)
            assert np.all(gl[n:] == 7)
            none = np.isneginf(wlse[:n])
            assert np.array_equal(np.isneginf(gl[:n]), none)
            ok = np.isfinite(wlse[:n])
            assert np.array_equal(np.isfinite(gl[:n]), ok)
            assert np.all(np.abs(gl[:n] - wlse[:n])[ok] <= (e + acc + 2.0 ** -20 * (1 + np.abs(wlse[:n])))[ok])
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
@pytest.mark.parametrize("dtype,fmt", [("bf16", "int8"), ("f16", "e4m3"), ("bf16", "e4m3"), ("f16", "int8")])
@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(F, case, dtype, fmt, d):
    new, past, page, Hq, Hkv, window, n_sink = ATTN[case]
    rng = np.random.default_rng(100 + case)
    layout, rot = [(None, 0), ("half", d), ("interleaved", d // 2), ("half", 16)][(case + d // 64) % 4]
    check_attn(F, rng, new, past, page, Hq, Hkv, d, dtype, fmt, layout, rot, window, n_sink,
               hints=((None, 0), (1, 5000), (1000, 1), (1000, 5000)), spoil=True)


@pytest.mark.parametrize("dtype,fmt,d,page,window,n_sink", [("bf16", "int8", 128, 64, 0, 0), ("f16", "e4m3", 64, 32, 700, 40),
                                                            ("bf16", "e4m3", 128, 16, 1500, 4), ("f16", "int8", 64, 128, 0, 0)])
def test_attention_of_long_chunks(F, dtype, fmt, d, page, window, n_sink):
    """Many row tiles over long contexts: shares of the work that begin and end inside row tiles, of one sequence and between
    sequences; also with a hint that leaves each tile to a workgroup, and with the kernel for few rows."""
    rng = np.random.default_rng(12)
    check_attn(F, rng, [300, 0, 1, 170], [1200, 50, 2000, 3], page, 4, 2, d, dtype, fmt, "half", d, window, n_sink,
               hints=((300, 2001), (300, 500), (300, 0), (1, 2001)), spoil=True)


@pytest.mark.parametrize("dtype,fmt,d,window,n_sink", [("bf16", "int8", 128, 0, 0), ("f16", "e4m3", 64, 900, 20)])
def test_attention_of_few_row_tiles(F, dtype, fmt, d, window, n_sink):
    """Few row tiles against many workgroups: shares of the least length, a row tile joined from many of them."""
    rng = np.random.default_rng(22)
    check_attn(F, rng, [33, 0, 64, 1], [2500, 0, 1100, 3], 64, 2, 1, d, dtype, fmt, "half", d, window, n_sink,
               hints=((64, 2533),), spoil=True)


def test_thousands_of_sequences(F):
    """More sequences than a search looks at in one or two rounds, many of them without a row."""
    rng = np.random.default_rng(14)
    B, page, d = 5000, 16, 64
    new = (np.arange(B) % 3 > 0).astype(int)
    new[[0, 17, 4097, B - 1]] = [0, 20, 33, 0]
    past = rng.integers(0, 40, B)
    check_attn(F, rng, list(new), list(past), page, 1, 1, d, "bf16", "int8", hints=((1, 0), (33, 0), (33, 2000)))
    cu, lens, tab, n_pages = batch(rng, list(new), list(past), page)
    x = torch.from_numpy(rng.normal(size=(int(cu[-1]), 1, d))).to(torch.float16)
    for few in (True, False):                               # an average of up to eight rows takes the kernel for few
        if not few:
            new = new * 13
            cu, lens, tab, n_pages = batch(rng, list(new), list(past), page)
            x = torch.from_numpy(rng.normal(size=(int(cu[-1]), 1, d))).to(torch.float16)
        codes, scale = make_cache(rng, n_pages, 1, page, d, "int8")
        gc, gs = [dev_codes(c, "int8") for c in codes], [torch.from_numpy(s.copy()).cuda() for s in scale]
        F.paged_append(x.cuda(), (-x).cuda(), i32(cu), i32(lens), i32(tab), *gc, *gs)
        for y, c, s, g, h in ((f64(x), codes[0], scale[0], gc[0], gs[0]), (-f64(x), codes[1], scale[1], gc[1], gs[1])):
            paged.append(y, cu, lens, tab, c, s, "int8")
            assert np.array_equal(h.cpu().numpy(), s) and np.array_equal(raw(g), c)


def test_attention_beyond_4_gib(F):
    """Pages whose offsets in the cache pass 32 bits, written and read."""
    page, Hkv, d = 128, 8, 128
    n_pages = (1 << 32) // (Hkv * page * d) + 600
    cache = F.paged_cache(n_pages, Hkv, page, d)
    assert cache[0].numel() > 1 << 32
    rng = np.random.default_rng(13)
    far = np.sort(rng.choice(np.arange(n_pages - 500, n_pages), 6, replace=False))[::-1].copy()
    tab = np.stack([far[:3], far[3:]]).astype(np.int32)
    for new, lens, max_q in (([300, 257], [300, 257], 300), ([1, 1], [301, 258], 1), ([40, 30], [341, 288], 40)):
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T = int(cu[-1])
        q, k, v = (torch.from_numpy(rng.normal(size=(T, h, d))).to(torch.bfloat16) for h in (16, Hkv, Hkv))
        keep = [c[torch.from_numpy(far).long().cuda()].clone() for c in cache]
        F.paged_append(k.cuda(), v.cuda(), i32(cu), i32(lens), i32(tab), *cache)
        o = F.paged_attn(q.cuda(), i32(cu), i32(lens), i32(tab), *cache, max_q=max_q)
        torch.cuda.synchronize()
        near = np.arange(6, dtype=np.int32).reshape(2, 3)           # the same pages, six of them on the host
        codes = [raw(c) if i < 2 else c.cpu().numpy() for i, c in enumerate(keep)]
        for x, c, s in ((f64(k), codes[0], codes[2]), (f64(v), codes[1], codes[3])):
            paged.append(x, cu, lens, near, c, s, "int8")
        got = [c[torch.from_numpy(far).long().cuda()] for c in cache]
        held = [[p for b in range(2) for p in range(3 * b, 3 * b - (-lens[b] // page))]]
        for i in range(4):
            g = raw(got[i]) if i < 2 else got[i].cpu().numpy()
            assert np.array_equal(g[held[0]], codes[i][held[0]])
        want, _, av, aq, aw = paged.attend(f64(q), cu, lens, near, *codes, "int8", d ** -0.5)
        tol = (2 * 2.0 ** -11 * aq[..., None] + 2.0 ** -10 + 500 * 2.0 ** -23) * av + 2.0 ** -25 * aw + 2.0 ** -8 * np.abs(want) + 2.0 ** -24
        assert np.all(np.abs(f64(o) - want) <= tol)


def test_attention_holes_and_empty_rows(F):
    rng = np.random.default_rng(7)
    # every page of sequence 0 is gone; 1 keeps its first page (sinks) and its window; 2 starts behind a hole
    holes = [(0, p) for p in range(5)] + [(1, p) for p in range(1, 9)] + [(2, 0), (2, 1)]
    for new in ([2, 3, 4], [40, 50, 60]):
        for window, n_sink in ((0, 0), (20, 4)):
            check_attn(F, rng, new, [70, 200, 60], 16, 4, 2, 64, "bf16", "e4m3", window=window, n_sink=n_sink, holes=holes,
                       hints=((None, 0), (1, 0), (500, 4000)), spoil=True)
    # sequences shorter than their rows: the first rows lie before position 0
    cu, lens, tab = i32([0, 5, 45]), i32([2, 0]), i32([[0], [1]])
    cache = F.paged_cache(2, 2, 64, 64)
    for c in cache:
        c.fill_(1)
    q = torch.ones(45, 4, 64, dtype=torch.float16, device="cuda")
    for max_q in (1, 40):
        lse = torch.empty(45, 4, device="cuda")
        o = F.paged_attn(q, cu, lens, tab, *cache, lse=lse, max_q=max_q)
        assert torch.all(o[:3] == 0) and torch.all(o[3:5] == 1) and torch.all(o[5:] == 0)
        assert torch.all(torch.isneginf(lse[:3])) and torch.all(torch.isneginf(lse[5:])) and torch.isfinite(lse[3:5]).all()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("new,past", [([1, 2], [400, 90]), ([80, 50], [300, 0])])
def test_attention_scales(F, new, past, fmt):
    """Pages of zeros, pages far quieter or louder than others, a page with a NaN scale (rows that see it are NaN, those that
    do not are not)."""
    rng = np.random.default_rng(8)

    def quiet(scale, tab):
        scale[0][tab[0, 1]] = 0                # keys of zeros: scores 0
        scale[1][tab[0, 2]] = 0                # values of zeros
        scale[1][tab[0, 3]] = 1e-9
        scale[1][tab[1, 0]] = 0
        scale[1][tab[0, 0]] *= 50
    check_attn(F, rng, new, past, 32, 4, 2, 128, "bf16", fmt, hints=((None, 0), (1, 3000), (400, 3000)), scale_edit=quiet)

    def all_zero(scale, tab):
        scale[1][:] = 0
    check_attn(F, rng, new, past, 32, 4, 2, 64, "f16", fmt, hints=((None, 0), (400, 3000)), scale_edit=all_zero)

    def poison(scale, tab):
        scale[0][tab[0, 2]] = np.nan
        scale[1][tab[0, 5], 1] = np.nan
        scale[1][tab[1, 1], 0] = np.inf
    check_attn(F, rng, new, past, 32, 4, 2, 64, "bf16", fmt, window=70, n_sink=40, hints=((None, 0), (1, 3000), (400, 3000)),
               scale_edit=poison)


@pytest.mark.parametrize("new,past", [([1, 1], [400, 20]), ([80, 25], [300, 0])])
def test_attention_key_scales_that_are_not_finite(F, new, past):
    """The row's normaliser is NaN with its output, also where a wave, a part or the whole row has no other key."""
    rng = np.random.default_rng(15)

    def poison(scale, tab):
        scale[0][tab[0, 5], 0] = np.nan           # one head of keys 160 .. 191
        scale[0][tab[1, 0], 1] = np.inf           # the only page of sequence 1
    check_attn(F, rng, new, past, 32, 4, 2, 64, "bf16", "int8", hints=((None, 0), (1, 3000), (400, 3000)), scale_edit=poison)


def test_attention_peaked_rows(F):
    """Scores of hundreds: the softmax reference moves far and often; one key carries a row."""
    rng = np.random.default_rng(9)
    for new, past in (([2, 1], [700, 33]), ([150], [200])):
        check_attn(F, rng, new, past, 64, 4, 2, 128, "bf16", "int8", "half", 128, amp=30.0, hints=((None, 0), (1, 3000), (400, 0)),
                   spread=0.3)


def test_attention_runs_twice_to_the_same_bits(F):
    rng = np.random.default_rng(10)
    for new, past, hint in (([1] * 5, [3000, 100, 1, 900, 64], 1), ([200, 64], [100, 900], 200)):
        part, args = check_attn(F, rng, new, past, 64, 8, 2, 128, "bf16", "int8", hints=((hint, 4000),))
        one = F.paged_attn(part, *args, max_q=hint, max_len=4000)
        for _ in range(3):
            assert torch.equal(F.paged_attn(part, *args, max_q=hint, max_len=4000)[:sum(new)], one[:sum(new)])


def test_workspace(F):
    rng = np.random.default_rng(11)
    part, args = check_attn(F, rng, [1, 1], [3000, 100], 64, 8, 2, 128, "bf16", "int8", hints=((1, 4000),))
    ws = F.paged_attn_ws(part, args[2], args[3], max_q=1, max_len=4000)
    one = F.paged_attn(part, *args, max_q=1, max_len=4000)
    if ws is not None:
        ws.fill_(255)                                      # (NaN patterns)
        assert torch.equal(F.paged_attn(part, *args, max_q=1, max_len=4000, ws=ws)[:2], one[:2])
        with pytest.raises(F.FlashLoopError, match="FL_E_WORKSPACE"):
            F.paged_attn(part, *args, max_q=1, max_len=4000, ws=ws[:16])
