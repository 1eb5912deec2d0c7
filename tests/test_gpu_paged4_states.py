"""Contexts kept in 4 bits between the loops of a model whose later loops are sparse: a loop's states are appended to a cache of its own,
read back as bf16 [B, N, H, d], and the sparse loops and the decode step run over what came back."""
import numpy as np
import pytest
import torch

from gpu_util import assert_close, down, down_bits16
from oracle import decode as dec
from oracle import paged4
from oracle.numerics import bf16_to_f64
from paper_2609_29812_amd import driver

pytestmark = pytest.mark.gpu

PAGE = 64


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def stored(F, k, v, fmt, seed):
    """(states read back, rows that append gave, the oracle's bf16 rows) of k, v [B, N, H, d]."""
    B, N, H, d = k.shape
    per = -(-N // PAGE)
    tab = np.random.default_rng(seed).permutation(B * per).reshape(B, per).astype(np.int32)
    cu, lens = np.arange(B + 1) * N, np.full(B, N)
    cache = F.paged4_cache(B * per, H, PAGE, d, fmt)
    rows = [torch.empty(B * N, H, d, dtype=k.dtype, device="cuda") for _ in range(2)]
    flat = [x.view(B * N, H, d) for x in (k, v)]
    F.paged4_append(*flat, i32(cu), i32(lens), i32(tab), *cache, k_rows=rows[0], v_rows=rows[1])
    states = [torch.full_like(k, 7.0) for _ in range(2)]
    F.paged4_read(i32(cu), i32(lens), i32(tab), *cache, B * N, k_out=states[0].view(B * N, H, d), v_out=states[1].view(B * N, H, d))
    want = []
    for x in flat:
        c, m = paged4.empty(B * per, H, PAGE, d, fmt)
        y, _ = paged4.append(x.cpu().double().numpy(), cu, lens, tab, c, m, fmt)
        want.append(torch.from_numpy(y).float().to(torch.bfloat16).view(B, N, H, d))
    return states, [r.view(B, N, H, d) for r in rows], want


def loops(B, N, H, d, n, seed):
    """States of n loops: a fifth of the positions moves from one to the next."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    out = [[rand(B, N, H, d).to(torch.bfloat16) for _ in range(3)]]
    for _ in range(n - 1):
        move = (torch.rand(B, N, 1, 1, generator=g, device="cuda") < 0.2).float()
        out.append([(x.float() + 0.3 * move * rand(B, N, H, d)).to(torch.bfloat16) for x in out[-1]])
    return out


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_sparse_loops_over_states_read_back(F, fmt):
    """The same bits as over the rows that append gave, which are the oracle's."""
    B, N, H, d = 2, 256, 2, 128
    qs, back, given = [], [], []
    for i, (q, k, v) in enumerate(loops(B, N, H, d, 3, 1)):
        states, rows, want = stored(F, k, v, fmt, i)
        assert all(torch.equal(s.cpu(), w) for s, w in zip(states, want))
        qs.append(q)
        back.append(states)
        given.append(rows)

    def chain(s):
        st = driver.setup(qs[0], s[0][0], s[0][1], 4, 64, 4, 48, 64)
        for r in (1, 2):
            driver.sparse_step(st, qs[r], qs[r - 1], s[r][0], s[r - 1][0], s[r][1], s[r - 1][1], [0, 96, 48][r], 4)
        return [st.o, st.lse, st.cols, st.cand, st.k_hat, st.v_hat]
    got, want = chain(back), chain(given)
    torch.cuda.synchronize()
    assert torch.isfinite(got[0]).all() and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_decode_over_states_read_back(F, fmt):
    """A decode position's loops against the oracle of the decode step over the oracle's rows."""
    B, N, H, d, n_sink, window = 2, 200, 2, 128, 4, 16
    o, prev = torch.zeros(B, H, d, device="cuda"), (None, None, None)
    host = {(b, h): dict(S=None, m=None, sub=None, o=None) for b in range(B) for h in range(H)}
    for i, ((q, k, v), budget) in enumerate(zip(loops(B, N, H, d, 3, 2), (60, 40, 0)), start=1):
        (ks, vs), _, want = stored(F, k, v, fmt, i)
        x = q[:, -1].contiguous()
        lse = torch.zeros(B, H, device="cuda")
        prev = F.decode_step(x, ks, vs, *prev, o, budget, n_sink=n_sink, window=window, lse=lse)
        torch.cuda.synchronize()
        qx, kx, vx = (bf16_to_f64(down_bits16(t)) for t in (x, *want))
        outs, ls = [], []
        for (b, h), st in host.items():
            oo, S, m, sub, L = dec.decode_step(qx[b, h], kx[b, :, h], vx[b, :, h], st["S"], st["m"], st["sub"], st["o"], d ** -0.5, n_sink,
                                               window, budget)
            st.update(S=S, m=m, sub=sub, o=oo)
            outs.append(oo)
            ls.append(L)
            if budget:
                assert np.array_equal(down(prev[0])[b, h], S), f"loop {i} selection b={b} h={h}"
        assert_close(down(o).reshape(B * H, d), np.array(outs), f"loop {i} output")
        assert_close(down(lse).reshape(-1), np.array(ls), f"loop {i} log-normaliser")
