"""Windowed attention over the paged 8-bit cache of rows at and behind the block table's end: a window counts back from the row's own
position, wherever the stored keys end, and the kernel that a hint selects makes no difference.

Tolerances are those of the other tests of this attention: fp16 queries move a score by e = 2^-11 A, a probability is off by 2 e and its
own rounding (2^-10 with that of its product with the value's scale), sums over n keys by (n + d) 2^-23, the output by half a step."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import paged

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def dev_codes(a, fmt):
    t = torch.from_numpy(np.ascontiguousarray(a).view(np.uint8)).cuda()
    return t.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn)


def check(F, rng, new, lens, page, max_pages, Hq, Hkv, d, dtype, fmt, window, n_sink, hints, rotate=False):
    """Pages that no row sees have scales that read as NaN."""
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T, B, cap, dt = int(cu[-1]), len(new), max_pages * page, DT[dtype]
    tab = rng.permutation(B * max_pages).reshape(B, max_pages).astype(np.int32)
    codes = [paged.encode(np.clip(rng.normal(size=(B * max_pages, Hkv, page, d)) * 30, -127, 127), fmt) for _ in range(2)]
    scale = [(np.exp(rng.normal(size=(B * max_pages, Hkv))) * 0.025).astype(np.float32) for _ in range(2)]
    pos = np.concatenate([np.arange(L - n, L) for n, L in zip(new, lens)])
    for b in range(B):
        seen = np.zeros(cap, bool)
        for i in range(lens[b] - new[b], lens[b]):
            seen[paged.seen_by(i, cap, window, n_sink)] = True
        for p in np.flatnonzero(~seen.reshape(max_pages, page).any(axis=1)):
            scale[0][tab[b, p]], scale[1][tab[b, p]] = np.nan, np.inf
    q = torch.from_numpy(rng.normal(size=(T, Hq, d))).to(dt)
    qx, table = q.double().numpy(), None
    if rotate:
        cs = paged.table(cap, d).astype(np.float32)
        qx, table = paged.rotate(qx, cs[np.clip(pos, 0, cap - 1)], "half"), torch.from_numpy(cs).cuda()
    want, wlse, av, aq, aw = paged.attend(qx, cu, np.array(lens), tab, *codes, *scale, fmt, d ** -0.5, window, n_sink)
    assert np.isfinite(want).all()
    e, acc = 2.0 ** -11 * aq, (cap + d) * 2.0 ** -23
    tol = (2 * e[..., None] + 2.0 ** -10 + acc) * av + 2.0 ** -25 * aw + torch.finfo(dt).eps / 2 * np.abs(want) + 2.0 ** -24
    cache = [dev_codes(codes[0], fmt), dev_codes(codes[1], fmt), torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda()]
    for max_q, split in hints:
        lse = torch.zeros(T, Hq, device="cuda")
        ws = F.paged_attn_ws(q.cuda(), i32(tab), cache[0], window=window, n_sink=n_sink, max_q=max_q)
        assert split is None or (ws is not None) == split
        got = F.paged_attn(q.cuda(), i32(cu), i32(lens), i32(tab), *cache, table=table, window=window, n_sink=n_sink, max_q=max_q, lse=lse,
                           ws=ws).cpu().double().numpy()
        err = np.abs(got - want)
        what = f"{new} of {lens}, {cap} places, {Hq}/{Hkv}x{d} {dtype} {fmt} w={window}+{n_sink} hint {max_q}"
        say(f"  {what}: worst={np.max(err / tol):.2f} of tol, {int((err > tol).any(axis=(1, 2)).sum())} rows beyond it")
        assert bool((err <= tol).all()), what
        assert bool((np.abs(lse.cpu().double().numpy() - wlse) <= e + acc + 2.0 ** -20 * (1 + np.abs(wlse))).all()), what


@pytest.mark.parametrize("n_sink", [0, 4, 70])
@pytest.mark.parametrize("dtype,fmt,d", [("bf16", "int8", 128), ("f16", "e4m3", 64), ("f16", "int8", 64), ("bf16", "e4m3", 128)])
def test_windows_of_rows_beyond_the_block_table(F, dtype, fmt, d, n_sink):
    rng = np.random.default_rng(31)
    hints = ((1, None), (20, None), (128, None))
    check(F, rng, [128, 5, 60], [400, 257, 300], 16, 16, 1, 1, d, dtype, fmt, 200, n_sink, hints)
    check(F, rng, [128, 5, 60], [400, 257, 300], 16, 16, 4, 2, d, dtype, fmt, 200, n_sink, hints, rotate=True)
    check(F, rng, [100, 1], [500, 481], 32, 15, 2, 1, d, dtype, fmt, 65, n_sink, hints)          # (the last pages are half a stage)


@pytest.mark.parametrize("dtype,fmt,d,n_sink", [("bf16", "int8", 128, 0), ("f16", "e4m3", 64, 130)])
def test_windows_beyond_the_block_table_in_shares(F, dtype, fmt, d, n_sink):
    """The same where the work is cut into shares."""
    check(F, np.random.default_rng(32), [150, 40], [2300, 2200], 128, 16, 2, 1, d, dtype, fmt, 1500, n_sink, ((150, True),))
