"""Windowed attention over the paged 4-bit cache of rows at and behind the block table's end: a window counts back from the row's own
position, wherever the stored keys end, and the kernel that a hint selects makes no difference.

Tolerances are those of the other tests of this attention: e bounds a score's error (fp16 queries, int4 keys in fp16, an fp32 sum), a
probability is off by 2 e and its own rounding, an int4 value by 2^-11 of itself, sums over n keys by (n + d) 2^-23, the output by half
a step."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import paged, paged4

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def up(a):
    return torch.from_numpy(a.copy()).cuda()


def check(F, rng, new, lens, page, max_pages, Hq, Hkv, d, dtype, fmt, window, n_sink, hints, rotate=False):
    """Pages that no row sees hold numbers that read as NaN."""
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T, B, cap, dt = int(cu[-1]), len(new), max_pages * page, DT[dtype]
    tab = rng.permutation(B * max_pages).reshape(B, max_pages).astype(np.int32)
    sides = [paged4.empty(B * max_pages, Hkv, page, d, fmt, rng) for _ in range(2)]
    pos = np.concatenate([np.arange(L - n, L) for n, L in zip(new, lens)])
    for b in range(B):
        seen = np.zeros(cap, bool)
        for i in range(lens[b] - new[b], lens[b]):
            seen[paged.seen_by(i, cap, window, n_sink)] = True
        for p in np.flatnonzero(~seen.reshape(max_pages, page).any(axis=1)):
            for _, m in sides:
                m[tab[b, p]] = np.nan if fmt == "int4" else 255
    q = torch.from_numpy(rng.normal(size=(T, Hq, d))).to(dt)
    qx, table = q.double().numpy(), None
    if rotate:
        cs = paged.table(cap, d).astype(np.float32)
        qx, table = paged.rotate(qx, cs[np.clip(pos, 0, cap - 1)], "half"), torch.from_numpy(cs).cuda()
    want, wlse, av, aq, aw = paged4.attend(qx, paged4.paged_seqs(cu, np.array(lens), tab, sides, fmt), Hkv, d ** -0.5, window, n_sink)
    assert np.isfinite(want).all()
    wide = 2.0 ** -11 if fmt == "int4" else 0.0
    e, acc = (2.0 ** -11 + wide + (d + 8) * 2.0 ** -23) * aq, (cap + d) * 2.0 ** -23
    tol = (2 * e[..., None] + 2.0 ** -11 + wide + acc) * av + 2.0 ** -25 * aw + torch.finfo(dt).eps / 2 * np.abs(want) + 2.0 ** -24
    cache = [up(sides[0][0]), up(sides[1][0]), up(sides[0][1]), up(sides[1][1])]
    for max_q, shared in hints:
        lse = torch.zeros(T, Hq, device="cuda")
        ws = F.paged4_attn_ws(q.cuda(), i32(tab), cache[0], window=window, n_sink=n_sink, max_q=max_q)
        assert shared is None or (ws is not None) == shared
        got = F.paged4_attn(q.cuda(), i32(cu), i32(lens), i32(tab), *cache, table=table, window=window, n_sink=n_sink, max_q=max_q, lse=lse,
                            ws=ws).cpu().double().numpy()
        err = np.abs(got - want)
        what = f"{new} of {lens}, {cap} places, {Hq}/{Hkv}x{d} {dtype} {fmt} w={window}+{n_sink} hint {max_q}"
        say(f"  {what}: worst={np.max(err / tol):.2f} of tol, {int((err > tol).any(axis=(1, 2)).sum())} rows beyond it")
        assert bool((err <= tol).all()), what
        assert np.all(np.abs(lse.cpu().double().numpy() - wlse) <= e + acc + 2.0 ** -20 * (1 + np.abs(wlse))), what


@pytest.mark.parametrize("n_sink", [0, 4, 70])
@pytest.mark.parametrize("dtype,fmt,d", [("bf16", "int4", 128), ("f16", "e2m1", 64), ("f16", "int4", 64), ("bf16", "e2m1", 128)])
def test_windows_of_rows_beyond_the_block_table(F, dtype, fmt, d, n_sink):
    rng = np.random.default_rng(31)
    hints = ((1, None), (20, None), (128, None))
    check(F, rng, [128, 5, 60], [400, 257, 300], 16, 16, 1, 1, d, dtype, fmt, 200, n_sink, hints)
    check(F, rng, [128, 5, 60], [400, 257, 300], 16, 16, 4, 2, d, dtype, fmt, 200, n_sink, hints, rotate=True)
    check(F, rng, [100, 1], [500, 481], 32, 15, 2, 1, d, dtype, fmt, 65, n_sink, hints)          # (the last pages are half a stage)


@pytest.mark.parametrize("dtype,fmt,d,n_sink", [("bf16", "int4", 128, 0), ("f16", "e2m1", 64, 130), ("f16", "int4", 128, 4)])
def test_windows_beyond_the_block_table_in_shares(F, dtype, fmt, d, n_sink):
    """The same where the work is cut into shares."""
    check(F, np.random.default_rng(32), [300, 40], [4300, 4200], 128, 32, 2, 1, d, dtype, fmt, 3000, n_sink, ((300, True),))


def test_lengths_next_to_the_largest(F):
    """Positions so far behind the block table that no row sees a key of it, or the leading ones alone."""
    most = 2 ** 31 - 1
    for n_sink, seen in ((0, 0), (3, 3)):
        rng = np.random.default_rng(33)
        d, tab = 64, i32(np.arange(8).reshape(1, 8))
        sides = [paged4.empty(8, 1, 16, d, "int4", rng) for _ in range(2)]
        cache = [up(sides[0][0]), up(sides[1][0]), up(sides[0][1]), up(sides[1][1])]
        v = paged4.rows_of(*sides[1], "int4").reshape(-1, d)
        q = torch.zeros(130, 1, d, dtype=torch.bfloat16, device="cuda")
        for window in (1, 2, 64, 100):
            for max_q in (1, 130):
                got = F.paged4_attn(q, i32([0, 130]), i32([most]), tab, *cache, window=window, n_sink=n_sink, max_q=max_q)
                want = v[:seen].mean(axis=0) if seen else np.zeros(d)
                # equal probabilities of 1, fp16 values, fp32 sums, half a step of the output
                tol = (2.0 ** -11 + 2.0 ** -8) * np.abs(v[:3]).mean(axis=0) + 2.0 ** -20
                assert np.all(np.abs(got.cpu().double().numpy() - want) <= tol), (window, n_sink, max_q)
