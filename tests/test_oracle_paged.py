"""The oracle of the rotary positions, the paged 8-bit cache and its attention, pinned on the CPU."""
import math

import numpy as np
import pytest
import torch

from oracle import paged


def test_e4m3_against_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(paged.E4M3, want, equal_nan=True)
    rng = np.random.default_rng(0)
    mid = (paged._POS[1:] + paged._POS[:-1]) / 2
    x = np.concatenate([rng.uniform(-448, 448, 4000), rng.normal(size=4000) * 0.01, mid, -mid, paged._POS, [-0.0]])
    got = paged.e4m3_encode(x.astype(np.float32))
    assert np.array_equal(got, torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_table_scalings():
    f, m = paged.frequencies(64)
    assert m == 1 and f[0] == 1 and math.isclose(f[-1], 10000 ** (-62 / 64))
    lin, _ = paged.frequencies(64, scaling="linear", factor=4.0)
    assert np.allclose(lin, f / 4, rtol=1e-15)
    ntk, _ = paged.frequencies(64, scaling="ntk", factor=4.0)
    assert ntk[0] == 1 and math.isclose(ntk[-1], f[-1] / 4, rel_tol=1e-12)     # the lowest frequency is divided by factor
    y, m = paged.frequencies(64, scaling="yarn", factor=4.0, orig_len=4096, low=1.0, high=32.0)
    turns = 4096 * f / (2 * math.pi)
    assert math.isclose(m, 1 + 0.1 * math.log(4))
    assert np.allclose(y[turns >= 32], f[turns >= 32], rtol=1e-15)
    assert np.allclose(y[turns <= 1], f[turns <= 1] / 4, rtol=1e-15)
    between = (turns > 1) & (turns < 32)
    assert between.any() and np.all((y[between] < f[between]) & (y[between] > f[between] / 4))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation(layout):
    rng = np.random.default_rng(1)
    x, y = rng.normal(size=(40, 3, 64)), rng.normal(size=(40, 3, 64))
    cs = paged.table(40, 32)
    rx = paged.rotate(x, cs, layout)
    assert np.allclose((rx ** 2).sum(-1), (x ** 2).sum(-1))                     # a rotation
    assert np.array_equal(rx[..., 32:], x[..., 32:])                            # part of the head
    assert np.allclose(paged.rotate(rx, cs, layout, inverse=True), x)
    # products go by the distance of the positions alone
    one, two = np.repeat(x[:1], 40, 0), np.repeat(y[:1], 40, 0)
    a, b = paged.rotate(one, cs, layout), paged.rotate(two, cs, layout)
    d = np.einsum("thd,shd->ths", a, b)
    for gap in (0, 3, 17):
        v = np.stack([d[t, :, t - gap] for t in range(gap, 40)])
        assert np.allclose(v, v[:1])
    # the inverse is the gradient: against differences of the sum of w * rotate(x)
    w, eps = rng.normal(size=x.shape), 1e-6
    grad = paged.rotate(w, cs, layout, inverse=True)
    for at in [(0, 0, 0), (5, 1, 3), (39, 2, 31), (7, 0, 16), (7, 0, 40)]:
        up, dn = x.copy(), x.copy()
        up[at] += eps
        dn[at] -= eps
        num = ((w * paged.rotate(up, cs, layout)).sum() - (w * paged.rotate(dn, cs, layout)).sum()) / (2 * eps)
        assert abs(num - grad[at]) < 1e-7


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_token_by_token_stays_within_a_step(fmt):
    rng = np.random.default_rng(2)
    page, H, d, n = 16, 2, 64, 40
    x = (rng.normal(size=(n, H, d)) * np.exp(rng.normal(size=(n, 1, 1)))).astype(np.float32).astype(np.float64)
    tab = np.array([[2, 0, 1]], np.int32)

    def fill(steps):
        codes, scale = np.full((3, H, page, d), 77, np.uint8), np.full((3, H), 9.0, np.float32)
        at = 0
        for m in steps:
            paged.append(x[at:at + m], np.array([0, m]), np.array([at + m]), tab, codes, scale, fmt)
            at += m
        v = paged.decode(codes, fmt) * scale.astype(np.float64)[:, :, None, None]
        return np.stack([v[tab[0, i // page], :, i % page] for i in range(n)]), scale

    once, s1 = fill([n])
    grown, s2 = fill([1] * n)
    part, _ = fill([5, 1, 13, 21])
    step = np.stack([s2[tab[0, i // page]] for i in range(n)])[:, :, None].astype(np.float64)
    assert np.all(s2 >= s1) and np.all(s2 < 2 * s1)
    if fmt == "int8":
        assert np.all(np.abs(once - x) <= 0.5 * np.stack([s1[tab[0, i // page]] for i in range(n)])[:, :, None] * (1 + 1e-6))
        assert np.all(np.abs(grown - x) <= step) and np.all(np.abs(part - x) <= step)
    else:                              # halving a scale's codes is exact but for the smallest
        assert np.all(np.abs(grown - x) <= np.maximum(2.0 ** -4 * np.abs(x) * (1 + 2.0 ** -4), 2.0 ** -9 * step))


def test_append_edges():
    tab = np.array([[0, 1]], np.int32)

    def put(vals, past=0, codes=None, scale=None, fmt="int8"):
        codes = np.zeros((2, 1, 16, 64), np.uint8) if codes is None else codes
        scale = np.zeros((2, 1), np.float32) if scale is None else scale
        x = np.zeros((len(vals), 1, 64))
        x[:, 0, 0] = vals
        paged.append(x, np.array([0, len(vals)]), np.array([past + len(vals)]), tab, codes, scale, fmt)
        return codes, scale

    c, s = put([127.0])
    assert s[0, 0] == 1 and c[0, 0, 0, 0] == 127
    c, s = put([254.0], 1, c, s)                        # exactly doubled; 127 / 2 = 63.5 to even
    assert s[0, 0] == 2 and c[0, 0, 0, 0] == 64 and c[0, 0, 1, 0] == 127
    c, s = put([254.0], 2, c, s)                        # the same again: no growth
    assert s[0, 0] == 2
    c, s = put([np.nan], 3, c, s)
    assert np.isnan(s[0, 0]) and c[0, 0, 3, 0] == 0
    c, s = put([1.0], 4, c, s)
    assert np.isnan(s[0, 0])                            # until the page is begun anew
    c, s = put([1.0], 0, c, s)
    assert s[0, 0] == np.float32(1 / 127)
    c, s = put([0.0, 0.0])
    assert s[0, 0] == 0
    c, s = put([3.0], 2, c, s)                          # from zero at once
    assert s[0, 0] == np.float32(3) * np.float32(1 / 127)
    c, s = put([1.0] * 3, 15)                           # over the border of a page
    assert s[0, 0] == s[1, 0] == np.float32(1 / 127) and c[0, 0, 15, 0] == c[1, 0, 1, 0] == 127
    for a, want in ((448.0, 1.0), (448.5, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (1.75, 2.0 ** -8), (1.76, 2.0 ** -7)):
        assert paged.need_of(a, "e4m3") == want
    assert paged.need_of(2.0 ** -101, "int8") == 0


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (7, 0), (7, 3), (1, 0), (100, 4)])
def test_attention_against_sdpa(fmt, window, n_sink):
    rng = np.random.default_rng(3)
    page, Hq, Hkv, d = 16, 6, 2, 64
    new, lens = [5, 1, 0, 20], np.array([37, 1, 9, 20])
    cu = np.concatenate([[0], np.cumsum(new)])
    T = cu[-1] + 2
    n_pages = 10
    tab = np.full((4, 4), -1, np.int32)
    order = rng.permutation(n_pages)
    at = 0
    for b in range(4):
        m = -(-lens[b] // page)
        tab[b, :m] = order[at:at + m]
        at += m
    codes = [rng.integers(0, 127, (n_pages, Hkv, page, d)).astype(np.uint8) ^ rng.choice([0, 128], (n_pages, Hkv, page, d)).astype(np.uint8)
             for _ in range(2)]
    if fmt == "e4m3":
        codes = [np.where((c & 127) == 127, 5, c).astype(np.uint8) for c in codes]
    scale = [rng.uniform(0.001, 0.02, (n_pages, Hkv)).astype(np.float32) for _ in range(2)]
    q = rng.normal(size=(T, Hq, d))
    o, lse, av, aq, aw = paged.attend(q, cu, lens, tab, *codes, *scale, fmt, d ** -0.5, window, n_sink)
    assert np.isnan(o[cu[-1]:]).all()
    for b in range(4):
        n, L = new[b], lens[b]
        if n == 0:
            continue
        kv = [np.concatenate([paged.decode(c[p], fmt) * s[p].astype(np.float64)[:, None, None] for p in tab[b, :-(-L // page)]],
                             axis=1)[:, :L] for c, s in zip(codes, scale)]
        i, j = np.arange(L - n, L)[:, None], np.arange(L)[None]
        mask = (j <= i) & ((j > i - window) | (j < n_sink) if window else True)
        k, v = (torch.from_numpy(np.repeat(x, Hq // Hkv, axis=0)) for x in kv)
        want = torch.nn.functional.scaled_dot_product_attention(
            torch.from_numpy(q[cu[b]:cu[b + 1]].transpose(1, 0, 2).copy()), k, v, attn_mask=torch.from_numpy(mask))
        assert np.allclose(o[cu[b]:cu[b + 1]], want.numpy().transpose(1, 0, 2), rtol=1e-10, atol=1e-12)
    # a page that is not there: its positions are seen by no row; a row that sees nothing is 0
    gone = tab.copy()
    gone[0] = -1
    o2, lse2, *_ = paged.attend(q, cu, lens, gone, *codes, *scale, fmt, d ** -0.5, window, n_sink)
    assert np.all(o2[:5] == 0) and np.all(lse2[:5] == -np.inf) and np.array_equal(o2[5:], o[5:], equal_nan=True)
