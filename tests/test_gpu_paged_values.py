"""Attention over the paged cache where values of one row span the range of their scales, against the fp64 oracle.

Tolerances are those of test_gpu_paged.py without their absolute term, so that they bound the error relative to the values, however
small: probabilities off by 2 e + 2^-10 of themselves, e = 2^-11 A with A = max_j sm_scale sum |q_e k_je|; fp16's subnormal
rounding, 2^-25 of the row's largest contribution w = max_j p_j s_j for each code (the reference that the products are rounded
relative to counts a page's scale as 2^-112 at least, so s_j is max(s_j, 2^-112) there: beside a page of zeros, products below
2^-24 * 2^-112 of what that page's keys would contribute are rounded to 0); fp32 sums, (keys + d) 2^-23; logarithms and powers
of scales up to 2^121 in fp32, 2^-17 of themselves twice; half a step of the output."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import paged
from test_gpu_paged import DT, batch, dev_codes, f64, half_step, i32, make_cache

pytestmark = pytest.mark.gpu


def attend(F, rng, new, past, page, Hq, Hkv, d, fmt, edit, hints, dtype="bf16", amp=1.0, sm=None, window=0, n_sink=0):
    """Calls for every hint; (got, lse, want, wanted lse, tolerances) of the rows of sequences."""
    cu, lens, tab, n_pages = batch(rng, new, past, page)
    codes, scale = make_cache(rng, n_pages, Hkv, page, d, fmt, 0.3)
    edit(scale, tab, codes)
    n = int(cu[-1])
    q = torch.from_numpy(rng.normal(size=(n, Hq, d)) * amp).to(DT[dtype])
    sm = d ** -0.5 if sm is None else sm
    want, wlse, av, aq, _ = paged.attend(f64(q), cu, lens, tab, *codes, *scale, fmt, sm, window, n_sink)
    aw = paged.attend(f64(q), cu, lens, tab, *codes, scale[0], np.maximum(scale[1], 2.0 ** -112), fmt, sm, window, n_sink)[4]
    args = (i32(cu), i32(lens), i32(tab), dev_codes(codes[0], fmt), dev_codes(codes[1], fmt),
            torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda())
    e, acc = 2.0 ** -11 * aq, (int(max(lens)) + d) * 2.0 ** -23 + 2.0 ** -16
    tol = (2 * e[..., None] + 2.0 ** -10 + acc) * av + 2.0 ** -25 * aw + half_step(DT[dtype]) * np.abs(want)
    for max_q, max_len in hints:
        lse = torch.empty(n, Hq, device="cuda")
        got = f64(F.paged_attn(q.cuda(), *args, sm_scale=sm, window=window, n_sink=n_sink, max_q=max_q, max_len=max_len, lse=lse))
        say(f"  new={list(new)[:4]} past={list(past)[:4]} {Hq}/{Hkv}x{d} {fmt} hint={max_q},{max_len}: "
            f"worst={np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300)):.2f} of tol")
        yield got, f64(lse), want, wlse, tol
        none = np.isneginf(wlse)
        assert np.array_equal(np.isneginf(f64(lse)), none)
        assert np.all(np.abs(f64(lse) - wlse)[~none] <= (e + acc + 2.0 ** -20 * (1 + np.abs(wlse)))[~none])


SHAPES = [([1, 2], [1500, 90], 32, 4, 2, 64, ((None, 0), (1, 3000))), ([5], [40], 16, 6, 1, 128, ((5, 100),)),
          ([90, 40], [1200, 0], 64, 4, 2, 128, ((None, 0), (90, 5000))), ([300], [0], 16, 1, 1, 64, ((300, 300), (300, 1024), (1, 300)))]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("octave", [-108, -80, -61, 100])
def test_values_of_any_magnitude(F, octave, shape, fmt):
    """All pages around one scale: the smallest that an append stores, between, and large ones."""
    new, past, page, Hq, Hkv, d, hints = SHAPES[shape]

    def edit(scale, tab, codes):
        scale[1][:] = np.ldexp(1 + (scale[1] * 1e4 % 1), octave)
    for got, _, want, _, tol in attend(F, np.random.default_rng(shape), new, past, page, Hq, Hkv, d, fmt, edit, hints):
        assert np.all(np.abs(got - want) <= tol)
        assert np.linalg.norm(got - want) <= 2.0 ** -7 * np.linalg.norm(want)


@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_the_least_scale(F, shape):
    """2^-112 itself, and the next number, beside scales that count as 0."""
    new, past, page, Hq, Hkv, d, hints = SHAPES[shape]
    rng = np.random.default_rng(shape)
    least = np.float32(2.0 ** -112)

    def edit(scale, tab, codes):
        scale[1][:] = rng.choice([least, np.nextafter(least, np.float32(1)), np.nextafter(least, np.float32(0)), 0], scale[1].shape)
    reads = []
    for got, _, _, _, _ in attend(F, rng, new, past, page, Hq, Hkv, d, "int8", edit, hints):
        reads.append(got)
    # (the oracle knows of no least scale: the same with those below it as 0)
    rng = np.random.default_rng(shape)

    def cut(scale, tab, codes):
        edit(scale, tab, codes)
        scale[1][scale[1] < least] = 0
    for was, (got, _, want, _, tol) in zip(reads, attend(F, rng, new, past, page, Hq, Hkv, d, "int8", cut, hints)):
        assert np.array_equal(got, was) and np.all(np.abs(got - want) <= tol) and np.abs(got).max() > 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("amp", [0.3, 12.0])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_pages_of_all_magnitudes(F, shape, amp, fmt):
    """Scales from 2^-108 to 2^110 side by side, and pages of zeros: rows that see small ones alone, rows that a key of a small
    page carries by its score; the normaliser counts every key."""
    new, past, page, Hq, Hkv, d, hints = SHAPES[shape]
    rng = np.random.default_rng(40 + shape)

    def edit(scale, tab, codes):
        scale[1][:] = np.ldexp(1.0, rng.integers(-108, 111, scale[1].shape)).astype(np.float32)
        scale[1][rng.random(scale[1].shape) < 0.2] = 0
        for b, row in enumerate(tab):                       # from small to large, but for the last sequence
            if b + 1 < len(tab) or b == 0:
                mine = row[row >= 0]
                scale[1][mine] = np.sort(scale[1][mine], axis=0)
    for got, _, want, _, tol in attend(F, rng, new, past, page, Hq, Hkv, d, fmt, edit, hints, amp=amp):
        assert np.all(np.abs(got - want) <= tol)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_one_loud_page(F, shape, fmt):
    """One page of values near fp32's limit among ordinary ones: its keys' probabilities, not their contributions, count."""
    new, past, page, Hq, Hkv, d, hints = SHAPES[shape]

    def edit(scale, tab, codes):
        scale[1][tab[:, 1]] = 2.0 ** 117
    for got, _, want, _, tol in attend(F, np.random.default_rng(shape), new, past, page, Hq, Hkv, d, fmt, edit, hints):
        assert np.all(np.abs(got - want) <= tol)


@pytest.mark.parametrize("dtype,fmt", [("f16", "int8"), ("bf16", "e4m3")])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_a_scale_of_zero_reads_zero(F, shape, dtype, fmt):
    """Whatever the codes are: a page's values, or all of them."""
    new, past, page, Hq, Hkv, d, hints = SHAPES[shape]
    rng = np.random.default_rng(shape)

    def some(scale, tab, codes):
        scale[1][rng.random(scale[1].shape) < 0.6] = 0

    def all_of_them(scale, tab, codes):
        scale[1][:] = 0
    for got, _, want, _, tol in attend(F, rng, new, past, page, Hq, Hkv, d, fmt, some, hints, dtype):
        # (fp16 outputs: subnormal ones are off by half of 2^-24)
        assert np.all(np.abs(got - want) <= tol + (2.0 ** -25 if dtype == "f16" else 0))
        assert np.all(got[want == 0] == 0)
    for got, _, _, _, _ in attend(F, rng, new, past, page, Hq, Hkv, d, fmt, all_of_them, hints, dtype):
        assert np.all(got == 0)


def test_small_values_come_back(F):
    """Appended and read: values of 1e-22, one position per sequence and a prompt; with one key the output is the value."""
    g = torch.Generator().manual_seed(3)
    for fmt in (torch.int8, torch.float8_e4m3fn):
        cache = F.paged_cache(40, 2, 16, 64, fmt)
        k, v, q = (torch.randn(40, h, 64, generator=g).to(torch.bfloat16) for h in (2, 2, 4))
        v *= 1e-22
        cu, lens, tab = i32(np.arange(41)), i32(np.ones(40)), i32(np.arange(40).reshape(40, 1))
        F.paged_append(k.cuda(), v.cuda(), cu, lens, tab, *cache)
        got = f64(F.paged_attn(q.cuda(), cu, lens, tab, *cache, max_q=1))
        stored = f64(cache[1].float())[:, :, 0] * f64(cache[3])[..., None]
        want = stored.repeat(2, axis=1)
        assert np.all(np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(want))
        assert np.all(np.abs(stored - f64(v)) <= np.abs(f64(v)).max(axis=2, keepdims=True) * (2.0 ** -4 if fmt != torch.int8 else 2.0 ** -7))


def test_a_negative_scale_reads_nan(F):
    """As one that is not finite: in the rows that see its page alone."""
    rng = np.random.default_rng(5)
    for at in (0, 1):
        cu, lens, tab, n_pages = batch(rng, [3, 40], [20, 0], 16)
        codes, scale = make_cache(rng, n_pages, 1, 16, 64, "int8")
        scale[at][tab[1, 1]] = -0.5
        args = (i32(cu), i32(lens), i32(tab), *(dev_codes(c, "int8") for c in codes), *(torch.from_numpy(s).cuda() for s in scale))
        q = torch.from_numpy(rng.normal(size=(43, 2, 64))).to(torch.bfloat16).cuda()
        for max_q in (1, 40):
            bad = torch.isnan(F.paged_attn(q, *args, max_q=max_q)).flatten(1).all(dim=1).cpu().numpy()
            assert np.array_equal(bad, np.arange(43) >= 3 + 16)


@pytest.mark.parametrize("dtype,layout", [("bf16", None), ("f16", None), ("bf16", "half"), ("f16", "interleaved")])
def test_a_query_that_is_not_finite(F, dtype, layout):
    """NaN in the output and the normaliser of the rows that see a key, also where every score is -inf; other rows as they were."""
    rng = np.random.default_rng(6)
    new, past = [2, 40, 1], [30, 0, 0]
    cu, lens, tab, n_pages = batch(rng, new, past, 16)
    tab[2] = -1                                             # a row that sees nothing
    codes, scale = make_cache(rng, n_pages, 1, 16, 64, "int8")
    codes[0][..., :2] = 256 - 5
    q = torch.from_numpy(rng.normal(size=(43, 2, 64))).to(DT[dtype])
    table = None if layout is None else F.rope_table(100 * 16, 16)
    args = (i32(cu), i32(lens), i32(tab), *(dev_codes(c, "int8") for c in codes), *(torch.from_numpy(s).cuda() for s in scale))
    bad = np.zeros((43, 2), bool)
    for r, h, c, x in ((0, 0, 0, np.inf), (5, 1, 0, np.inf), (6, 0, 1, -np.inf), (20, 1, 63, np.nan), (42, 0, 0, np.inf)):
        bad[r, h] = r != 42
        p = q.clone() if r == 0 else p
        p[r, h, c] = x
    for max_q, max_len in ((1, 0), (40, 0), (40, 3000)):
        lse, was = torch.empty(43, 2, device="cuda"), torch.empty(43, 2, device="cuda")
        kw = dict(table=table, layout=layout or "half", max_q=max_q, max_len=max_len)
        want = F.paged_attn(q.cuda(), *args, **kw, lse=was).cpu()
        got = F.paged_attn(p.cuda(), *args, **kw, lse=lse).cpu()
        nan = torch.from_numpy(bad)
        assert torch.isnan(got[nan]).all() and torch.isnan(lse.cpu()[nan]).all()
        assert torch.equal(got[~nan], want[~nan]) and torch.equal(lse.cpu()[~nan], was.cpu()[~nan])
        assert torch.all(got[42] == 0) and torch.isneginf(lse[42]).all()
