"""The oracle of the paged 4-bit cache and of packed attention, pinned on the CPU."""
import numpy as np
import pytest
import torch

from oracle import codec, paged4


def test_e2m1_by_hand():
    x = np.zeros(32)
    x[0] = 6.0                                       # the group's largest: e = 0
    x[1:15] = [0.25, 0.26, 0.75, 0.74, 1.25, 1.26, 1.75, 2.5, 2.51, 3.5, 3.49, 5.0, 5.01, -0.2]
    c, e = paged4.encode_group(x, "e2m1")
    assert e == 127
    assert c[:15].tolist() == [7, 0, 1, 2, 1, 2, 3, 4, 4, 5, 6, 5, 6, 7, 8]
    for a, want in ((6.0, 0), (6.001, 1), (3.0, -1), (1.5, -2), (1.51, -1), (2.0 ** -40, -23), (0.0, -23), (32768.0, 13), (1e30, 13)):
        x = np.zeros(32)
        x[3] = -a
        c, e = paged4.encode_group(x, "e2m1")
        assert e - 127 == want, a
        got = paged4.decode_group(c, e, "e2m1")
        assert abs(got[3] + min(a, 32768.0)) <= max(0.25 * min(a, 32768.0), 2.0 ** -25)


def test_e2m1_properties():
    rng = np.random.default_rng(0)
    for _ in range(50):
        x = (rng.normal(size=32) * np.exp(rng.normal() * 4)).astype(np.float32).astype(np.float64)
        c, e = paged4.encode_group(x, "e2m1")
        y = paged4.decode_group(c, e, "e2m1")
        unit = 2.0 ** (e - 127)
        assert np.abs(x).max() <= 6 * unit and np.abs(x).max() > 3 * unit
        step = np.where(np.abs(x) < 2 * unit, 0.5, np.where(np.abs(x) < 4 * unit, 1.0, 2.0)) * unit
        assert np.all(np.abs(y - x) <= step / 2)
        again, e2 = paged4.encode_group(y, "e2m1")                # what a code stands for is kept
        assert np.array_equal(paged4.decode_group(again, e2, "e2m1"), y)


def test_int4_against_the_codec():
    """The group's numbers are the base codec's (groups of consecutive channels), and so are the codes but where the fp32 quotient
    of that one rounds to a half."""
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(1, 40, 2, 64)) * np.exp(rng.normal(size=(1, 40, 2, 1)) * 2)).astype(np.float32)
    xs = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    enc = codec.encode(xs.astype(np.float32), 4, 32, codec.AXIS_CHANNEL)
    q, scale, zero = enc["q"], enc["scale"], enc["zero"]
    differ = 0
    for n in range(40):
        for h in range(2):
            for g in range(2):
                c, (s, z) = paged4.encode_group(xs[0, n, h, 32 * g:32 * g + 32], "int4")
                y = paged4.decode_group(c, (s, z), "int4")
                v = xs[0, n, h, 32 * g:32 * g + 32]
                assert float(z) <= v.min() and float(z) + 15 * float(s) >= v.max()
                assert np.all(np.abs(y - v) <= float(s) / 2 * (1 + 1e-12))
                assert scale[0, n, h, g] == s and zero[0, n, h, g] == z
                differ += int((q[0, n, h, 32 * g:32 * g + 32] != c).sum())
    assert differ <= 2


def test_int4_edges():
    flat = np.full(32, 0.1)
    c, (s, z) = paged4.encode_group(flat, "int4")
    assert float(z) < 0.1 and np.all(c == c[0])
    c, (s, z) = paged4.encode_group(np.full(32, -3.0), "int4")
    assert s == 0 and z == -3 and np.all(c == 0) and np.all(paged4.decode_group(c, (s, z), "int4") == -3)
    c, (s, z) = paged4.encode_group(np.zeros(32), "int4")
    assert (s, z) == (0, 0) and not np.signbit(s) and not np.signbit(z)
    x = np.linspace(-1e6, 1e6, 32)
    c, (s, z) = paged4.encode_group(x, "int4")
    assert float(z) == -32768 and float(s) == paged4.S_MOST and c[0] == 0 and c[-1] == 15
    for bad in (np.inf, -np.inf, np.nan):
        x = np.ones(32)
        x[5] = bad
        for fmt in ("int4", "e2m1"):
            c, m = paged4.encode_group(x, fmt)
            assert not c.any() and np.all(np.isnan(paged4.decode_group(c, m, fmt)))


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_rows_by_tables(fmt):
    rng = np.random.default_rng(2)
    codes, meta = paged4.empty(3, 2, 16, 64, fmt, rng)
    if fmt == "int4":
        meta[0, 0, 0, 0] = (np.nan, 0)
        meta[0, 0, 1, 1] = (-1, 0)
        meta[0, 0, 2, 1] = (1, np.inf)
        meta[0, 0, 3, 0] = (4376, 0)
    else:
        meta[0, 0, 0, 0], meta[0, 0, 1, 1], meta[0, 0, 2, 0] = 255, 103, 141
    got = paged4.rows_of(codes, meta, fmt)
    want = np.stack([[[paged4.row_of(codes[p, h, i], meta[p, h, i], fmt) for i in range(16)] for h in range(2)] for p in range(3)])
    assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(got[0, 0, :4]).any(axis=1).sum() == (4 if fmt == "int4" else 3)


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_append_then_read(fmt):
    rng = np.random.default_rng(3)
    n_pages, H, page, d = 9, 2, 16, 64
    codes, meta = paged4.empty(n_pages, H, page, d, fmt, rng)
    was = codes.copy(), meta.copy()
    cu, lens = np.array([0, 20, 20, 23]), np.array([20, 5, 36])
    tab = np.array([[3, 1, -1], [4, -1, -1], [0, 99, 7]])
    x = rng.normal(size=(25, H, d)).astype(np.float32).astype(np.float64)
    rows, dropped = paged4.append(x, cu, lens, tab, codes, meta, fmt)
    assert dropped.tolist() == [False] * 23 + [True] * 2             # sequence 2: positions 33 .. 35 lie in page 7
    back, none = paged4.read(cu, lens, tab, codes, meta, 25, fmt)
    assert np.array_equal(back[:23], rows[:23]) and none.tolist() == [False] * 23 + [True] * 2
    assert np.abs(rows[:23] - x[:23]).max() < 1.0
    assert np.array_equal(codes[[2, 5, 6, 8, 4, 0]], was[0][[2, 5, 6, 8, 4, 0]])
    lens2 = np.array([20, 5, 30])                                    # positions 27 .. 29 lie in a page that is not there
    rows, dropped = paged4.append(x, cu, lens2, tab, codes, meta, fmt)
    assert dropped[20:23].all()
    back, _ = paged4.read(cu, lens2, tab, codes, meta, 25, fmt)
    assert np.all(back[20:23] == 0)


@pytest.mark.parametrize("window,n_sink", [(0, 0), (7, 2)])
def test_packed_against_the_library(window, n_sink):
    rng = np.random.default_rng(4)
    cu_q, cu_k = np.array([0, 5, 5, 17, 21]), np.array([0, 9, 12, 24, 26])       # the last has more queries than keys
    Hq, Hkv, d = 4, 2, 16
    q, k, v = rng.normal(size=(22, Hq, d)), rng.normal(size=(26, Hkv, d)), rng.normal(size=(26, Hkv, d))
    o, lse, av, aq, aw = paged4.attend(q, paged4.packed_seqs(k, v, cu_q, cu_k), Hkv, 0.3, window, n_sink)
    assert np.isnan(o[21]).all()
    assert np.all(o[17:19] == 0) and np.all(np.isneginf(lse[17:19]))
    for b in range(4):
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        for t in range(max(0, n - m), n):
            i = m - n + t
            j = np.arange(m)
            seen = (j <= i) & ((j > i - window) | (j < n_sink) if window else True)
            for h in range(Hq):
                kk, vv = torch.from_numpy(k[cu_k[b]:cu_k[b + 1], h // 2]), torch.from_numpy(v[cu_k[b]:cu_k[b + 1], h // 2])
                want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[cu_q[b] + t, h])[None], kk, vv,
                                                                        attn_mask=torch.from_numpy(seen)[None], scale=0.3)
                assert np.allclose(o[cu_q[b] + t, h], want[0].numpy())
                x = 0.3 * kk.numpy()[seen] @ q[cu_q[b] + t, h]
                assert np.isclose(lse[cu_q[b] + t, h], np.logaddexp.reduce(x))
    assert np.all(np.abs(o[:17]) <= av[:17] + 1e-12) and np.all(aw >= av - 1e-12)
