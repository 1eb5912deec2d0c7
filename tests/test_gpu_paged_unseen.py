"""Attention over the paged cache beside what no row sees: freed pages between the leading positions and the window that still
have an entry in the block table, whatever they hold; lengths beyond the block table."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import paged
from test_gpu_paged import DT, batch, check_attn, dev_codes, f64, i32, make_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("e4m3", "f16"), ("int8", "bf16")])
@pytest.mark.parametrize("new,past,page,window,n_sink,d", [([1, 1, 1], [1000, 200, 40], 16, 50, 5, 64),
                                                           ([3, 2], [2100, 130], 16, 70, 17, 128),
                                                           ([6, 1], [500, 300], 32, 33, 0, 64),
                                                           ([150, 40], [1300, 90], 16, 60, 20, 128),
                                                           ([70, 200], [400, 0], 32, 37, 3, 64),
                                                           ([300], [1500], 128, 200, 1, 128)])
def test_freed_pages_that_hold_anything(F, new, past, page, window, n_sink, d, fmt, dtype):
    """Entries of freed pages name a spare page of NaN codes and scales that are not finite: the bits of a table without them."""
    rng = np.random.default_rng(len(new) + page)
    cu, lens, tab, n_pages = batch(rng, new, past, page)
    codes, scale = make_cache(rng, n_pages + 2, 2, page, d, fmt)
    gone = tab.copy()
    for b, n in enumerate(new):
        first = max(0, lens[b] - n - window + 1) // page
        gone[b, -(-n_sink // page):first] = -1
    spare = np.where((gone < 0) & (tab >= 0), n_pages + np.arange(tab.shape[1]) % 2, tab)
    assert (spare != tab).any()
    codes[0][n_pages:], codes[1][n_pages:] = 255, 127
    scale[0][n_pages:], scale[1][n_pages], scale[1][n_pages + 1] = np.nan, np.inf, 1.0
    args = (dev_codes(codes[0], fmt), dev_codes(codes[1], fmt), torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda())
    q = torch.from_numpy(rng.normal(size=(int(cu[-1]), 6, d))).to(DT[dtype]).cuda()
    for max_q, max_len in ((None, 0), (1, 0), (max(new), 4000), (200, 500)):
        say(f"  new={new} past={past} page={page} {fmt} {dtype} w={window}+{n_sink} hint={max_q},{max_len}")
        one, two = (F.paged_attn(q, i32(cu), i32(lens), i32(t), *args, window=window, n_sink=n_sink, max_q=max_q, max_len=max_len)
                    for t in (gone, spare))
        assert torch.isfinite(one).all() and torch.equal(one, two)


def test_the_same_against_the_oracle(F):
    """Pages of nobody and positions behind the end hold NaN; the block table is whole."""
    rng = np.random.default_rng(3)
    for new, past in (([1, 2], [300, 70]), ([90, 40], [250, 0])):
        check_attn(F, rng, new, past, 16, 4, 2, 64, "bf16", "e4m3", window=45, n_sink=6, hints=((None, 0), (1, 1000), (90, 2000)),
                   spoil=True)


@pytest.mark.parametrize("window,n_sink", [(30, 20), (30, 2 ** 31 - 1), (1500, 2 ** 30), (2 ** 31 - 1, 0), (0, 7)])
def test_lengths_beyond_the_block_table(F, window, n_sink):
    """Positions behind the last page see what the window and the leading positions leave of the stored ones."""
    rng = np.random.default_rng(4)
    for new, lens in (([1, 2], [2 ** 31 - 1, 100000]), ([300, 40], [2 ** 31 - 1, 1700])):
        max_pages, page = 100, 16
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        tab = rng.permutation(2 * max_pages).reshape(2, max_pages).astype(np.int32)
        codes, scale = make_cache(rng, 2 * max_pages, 1, page, 64, "int8")
        q = torch.from_numpy(rng.normal(size=(int(cu[-1]), 2, 64))).to(torch.bfloat16)
        want, wlse, av, aq, aw = paged.attend(f64(q), cu, np.array(lens), tab, *codes, *scale, "int8", 0.125, window, n_sink)
        args = (i32(cu), i32(lens), i32(tab), dev_codes(codes[0], "int8"), dev_codes(codes[1], "int8"),
                torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda())
        tol = (2 * 2.0 ** -11 * aq[..., None] + 2.0 ** -10 + 1700 * 2.0 ** -23) * av + 2.0 ** -25 * aw + 2.0 ** -8 * np.abs(want)
        for max_q, max_len in ((1, 0), (300, 0), (300, 100)):
            say(f"  new={new} w={window}+{n_sink} hint={max_q},{max_len}")
            lse = torch.empty(q.shape[:2], device="cuda")
            got = F.paged_attn(q.cuda(), *args, window=window, n_sink=n_sink, max_q=max_q, max_len=max_len, lse=lse)
            assert np.all(np.abs(f64(got) - want) <= tol)
            assert np.array_equal(np.isneginf(f64(lse)), np.isneginf(wlse))


@pytest.mark.parametrize("new,past,Hq,Hkv,max_q", [([1] * 7, [3000, 1, 900, 40, 5000, 64, 0], 8, 2, 1), ([2, 0, 1], [9000, 10, 700], 12, 1, 2),
                                                   ([1] * 150, [37 * i % 1500 for i in range(150)], 4, 2, 1),
                                                   ([200, 0, 30], [1300, 5, 10], 4, 2, 200), ([3, 5], [2000, 4000], 16, 4, 1)])
def test_the_workspace_is_enough(F, new, past, Hq, Hkv, max_q):
    """A workspace of exactly the size asked for, between guards that stay as they are, whatever it held before."""
    rng = np.random.default_rng(6)
    cu, lens, tab, n_pages = batch(rng, new, past, 64)
    codes, scale = make_cache(rng, n_pages, Hkv, 64, 64, "int8")
    args = (i32(cu), i32(lens), i32(tab), dev_codes(codes[0], "int8"), dev_codes(codes[1], "int8"),
            torch.from_numpy(scale[0]).cuda(), torch.from_numpy(scale[1]).cuda())
    q = torch.from_numpy(rng.normal(size=(int(cu[-1]), Hq, 64))).to(torch.bfloat16).cuda()
    one = F.paged_attn(q, *args, max_q=max_q)
    need = F.paged_attn_ws(q, args[2], args[3], max_q=max_q).numel()
    for fill in (0, 255):
        room = torch.full((need + 2048,), fill, dtype=torch.uint8, device="cuda")
        room[:1024], room[1024 + need:] = 85, 85
        assert torch.equal(F.paged_attn(q, *args, max_q=max_q, ws=room[1024:1024 + need]), one)
        assert torch.all(room[:1024] == 85) and torch.all(room[1024 + need:] == 85)
