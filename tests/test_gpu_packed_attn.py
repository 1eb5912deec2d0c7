"""Attention of packed prompts: the HIP path against the fp64 oracle.

Tolerances.  Products are exact in fp32 and sums of n of them off by at most n 2^-23 of the sum of their magnitudes, so a score by
e = (d + 8) 2^-23 A, A = max_j sm_scale sum |q_e k_je| (its argument's own rounding and the exponential's included), a probability by
2 e of itself, and it is rounded to the type: half a step of itself, or in fp16 2^-25 of the unit below its normal range, the unit
being at most the row's largest probability.  fp32 sums over the keys add (n + d) 2^-23, the output's own rounding half a step.
Rotated queries are rounded to the type from fp32 sums that may be off by 2^-22 of their products' magnitudes: a value that lies so
near to the middle between two of the type's may be either of them, which moves a score by sm_scale sum (step_e |k_je|) over those."""
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


def offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def compare(got, L, oracle, n, keys, d, dt, what, either=0.0):
    want, wlse, av, aq, aw = oracle
    fin = np.isfinite(want[:n])
    assert np.array_equal(np.isfinite(got[:n]), fin), f"{what}: finite where it should not be, or the other way round"
    e = (d + 8) * 2.0 ** -23 * aq[:n] + either
    acc = (keys + d) * 2.0 ** -23
    with np.errstate(invalid="ignore", over="ignore"):
        tol = (half_step(dt) + 2 * e[..., None] + acc + 2.0 ** -21) * av[:n] + 2.0 ** -25 * aw[:n] + half_step(dt) * np.abs(want[:n]) + 2.0 ** -24
        err = np.abs(got[:n] - want[:n])[fin]
    den = np.linalg.norm(want[:n][fin])
    rel = np.linalg.norm(err) / den if den else 0.0
    say(f"  {what}: rel={rel:.2e} worst={np.max(err / tol[fin]) if err.size else 0:.2f} of tol")
    assert np.all(err <= tol[fin]), what
    assert rel <= REL_FRO + half_step(dt), what
    if L is not None:
        gl, wl = f64(L)[:n], wlse[:n]
        assert np.array_equal(np.isneginf(gl), np.isneginf(wl)) and np.array_equal(np.isfinite(gl), np.isfinite(wl)), what
        ok = np.isfinite(wl)
        assert np.all(np.abs(gl[ok] - wl[ok]) <= (e + acc + 2.0 ** -20 * (1 + np.abs(wl)))[ok]), what


def check(F, rng, nq, nk, Hq, Hkv, d, dtype, window=0, n_sink=0, hints=(0,), layout=None, rot=0, amp=1.0, edit=None, fused=True, lse=True):
    dt = DT[dtype]
    cu_q, cu_k = offsets(nq), offsets(nk if nk is not None else nq)
    Tq, Tk = int(cu_q[-1]) + 2, int(cu_k[-1]) + (2 if nk is None else 1)
    q = torch.from_numpy(rng.normal(size=(Tq, Hq, d)) * amp).to(dt)
    k, v = (torch.from_numpy(rng.normal(size=(Tk, Hkv, d))).to(dt) for _ in range(2))
    if edit:
        edit(q, k, v, cu_q, cu_k)
    q[cu_q[-1]:] = float("nan")                            # rows of no sequence
    k[cu_k[-1]:], v[cu_k[-1]:] = float("nan"), float("inf")
    if fused and nk is None:                               # as a fused projection leaves them
        whole = torch.cat((q, k, v), dim=1).cuda()
        qd, kd, vd = whole[:, :Hq], whole[:, Hq:Hq + Hkv], whole[:, Hq + Hkv:]
    else:
        qd, kd, vd = q.cuda(), k.cuda(), v.cuda()
    qx, table = f64(q), None
    if layout:
        cs = paged.table(int(max(nk if nk is not None else nq)) + 1, rot).astype(np.float32)
        table = torch.from_numpy(cs).cuda()
        pos = np.concatenate([np.arange(m - n, m) for n, m in zip(nq, nk if nk is not None else nq)] + [np.zeros(2, int)]).astype(int)
        at = cs[np.maximum(pos, 0)]
        exact, most = paged.rotate(qx, at, layout), paged.rotate(np.abs(qx), np.abs(at), layout)
        most = np.maximum(np.abs(most), np.abs(paged.rotate(np.abs(qx), np.abs(at) * [1, -1], layout)))
        exact[:int(cu_q[-1])] = np.nan_to_num(exact[:int(cu_q[-1])])
        near = torch.from_numpy(exact).to(dt).double().numpy()
        lo, hi = (torch.from_numpy(exact + s * 2.0 ** -22 * most).to(dt).double().numpy() for s in (-1, 1))
        qx, either = near, np.where(lo != hi, hi - lo, 0.0)
    seqs = lambda: paged4.packed_seqs(f64(k), f64(v), cu_q, cu_k)  # noqa: E731
    either = paged4.attend(either, seqs(), Hkv, d ** -0.5, window, n_sink)[3][:int(cu_q[-1])] if layout else 0.0
    want = paged4.attend(qx, paged4.packed_seqs(f64(k), f64(v), cu_q, cu_k), Hkv, d ** -0.5, window, n_sink)
    n, keys = int(cu_q[-1]), int(np.diff(cu_k).max())
    for hint in hints:
        out = torch.full((Tq, 3 * Hq * d), 7.0, dtype=dt, device="cuda")
        o = out[:, Hq * d:2 * Hq * d].view(Tq, Hq, d)
        L = torch.full((Tq, Hq), 7.0, device="cuda") if lse else None
        F.packed_attn(qd, kd, vd, i32(cu_q), None if nk is None else i32(cu_k), table=table, layout=layout or "half", window=window,
                      n_sink=n_sink, max_k=hint, out=o, lse=L)
        torch.cuda.synchronize()
        got = f64(o)
        assert np.all(got[n:] == 7) and torch.all(out[:, :Hq * d] == 7) and torch.all(out[:, 2 * Hq * d:] == 7)
        assert L is None or torch.all(L[n:] == 7)
        compare(got, L, want, n, keys, d, dt, f"{list(nq)[:5]} of {list(nk)[:5] if nk is not None else 'the same'} {Hq}/{Hkv}x{d} {dtype} "
                f"w={window}+{n_sink} hint {hint}", either)


CASES = [
    # queries, keys (None: the same), Hq, Hkv, window, n_sink
    ([1], None, 1, 1, 0, 0),
    ([2, 1, 0, 3], None, 6, 2, 0, 0),
    ([300], None, 4, 4, 0, 0),
    ([31, 33, 64, 65], None, 3, 1, 0, 0),
    ([127, 1, 129, 0, 0, 63], None, 8, 2, 0, 0),
    ([200, 90], None, 2, 2, 64, 4),
    ([257, 30], None, 4, 1, 1, 0),
    ([300], None, 5, 5, 33, 70),
    ([1, 1, 1], [1, 700, 64], 4, 2, 0, 0),                    # single positions after others
    ([40, 5, 0, 1], [513, 5, 12, 130], 6, 3, 0, 0),
    ([20, 7, 3], [4, 0, 900], 2, 1, 0, 0),                    # more queries than keys, and no keys at all
    ([100, 33], [400, 65], 4, 2, 50, 5),
    ([1] * 100 + [0] * 20 + [3] * 10, None, 2, 1, 0, 0),      # more than 64 sequences
    ([64] * 9, None, 16, 2, 0, 0),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(F, case, dtype, d):
    nq, nk, Hq, Hkv, window, n_sink = CASES[case]
    layout, rot = [(None, 0), ("half", d), ("interleaved", d // 2), ("half", 16)][(case + d // 64) % 4]
    check(F, np.random.default_rng(case), nq, nk, Hq, Hkv, d, dtype, window, n_sink, hints=(0, 1, 5000), layout=layout, rot=rot,
          fused=case % 2 == 0)


@pytest.mark.parametrize("dtype,d,window,n_sink", [("bf16", 128, 0, 0), ("f16", 64, 700, 40), ("bf16", 64, 1500, 4), ("f16", 128, 0, 0)])
def test_long_chunks(F, dtype, d, window, n_sink):
    """Many row tiles over long sequences: work that is cut inside row tiles, of one sequence and between sequences."""
    check(F, np.random.default_rng(12), [300, 0, 1, 170], [1500, 50, 2001, 173], 4, 2, d, dtype, window, n_sink, hints=(0, 500, 2001))
    check(F, np.random.default_rng(13), [33, 0, 64, 1], [2533, 0, 1164, 4], 2, 1, d, dtype, window, n_sink, hints=(0,))


@pytest.mark.parametrize("dtype,d,window,n_sink", [("bf16", 128, 0, 0), ("f16", 64, 2600, 40), ("bf16", 64, 0, 0), ("f16", 128, 3000, 130)])
def test_chunks_after_long_contexts(F, dtype, d, window, n_sink):
    """Few row tiles over thousands of keys, cut into shares, which begin and end inside row tiles and between sequences."""
    check(F, np.random.default_rng(15), [300, 0, 1, 170], [4500, 50, 5001, 173], 4, 2, d, dtype, window, n_sink, hints=(0, 500, 5001))
    check(F, np.random.default_rng(16), [33, 0, 64, 1], [3033, 0, 2564, 4], 2, 1, d, dtype, window, n_sink, hints=(3033,), layout="half", rot=64)


def test_long_prompt(F):
    check(F, np.random.default_rng(14), [2100, 5], None, 2, 1, 128, "bf16", hints=(0, 100))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_large_and_small_scores(F, dtype):
    """Scores that leave a row to one key, or that grow along it (the running reference moves at every tile), or underflow."""
    def grow(q, k, v, cu_q, cu_k):
        q[:] = torch.sign(q.float()).to(q.dtype)
        k[:] = (torch.linspace(0.0, 6.0, k.shape[0])[:, None, None] * torch.sign(k.float())).to(k.dtype)

    def fall(q, k, v, cu_q, cu_k):
        q[:] = 1.0
        k[:] = torch.linspace(20.0, -20.0, k.shape[0])[:, None, None].to(k.dtype)
    for edit in (grow, fall):
        check(F, np.random.default_rng(3), [200, 64], None, 2, 1, 64, dtype, edit=edit)
    check(F, np.random.default_rng(4), [200], None, 2, 2, 128, dtype, amp=30.0)
    check(F, np.random.default_rng(5), [200], None, 2, 2, 128, dtype, amp=0.0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_what_a_row_does_not_see(F, dtype, d):
    """Infinities and NaN at later positions, in other sequences and outside the window leave a row alone; what sees them is not
    finite, in the value's channel or, for a key, altogether."""
    def edit(q, k, v, cu_q, cu_k):
        v[cu_k[0] + 90, 0, 3] = float("inf")
        v[cu_k[0] + 140, 1, d - 1] = float("nan")
        v[cu_k[0] + 141, 1, 0] = float("-inf")
        k[cu_k[0] + 170, 0, 5] = float("nan")
        k[cu_k[1] + 20, 0, :] = float("nan")
        v[cu_k[2], :, :] = float("nan")
        v[cu_k[2] + 5, :, 9] = float("inf")
    for window, n_sink in ((0, 0), (40, 3)):
        check(F, np.random.default_rng(6), [200, 70, 66], None, 4, 2, d, dtype, window, n_sink, edit=edit)
        check(F, np.random.default_rng(7), [30, 70, 66], [200, 70, 66], 4, 2, d, dtype, window, n_sink, edit=edit)
    check(F, np.random.default_rng(8), [1300, 70, 66], None, 1, 1, d, dtype, edit=lambda q, k, v, a, b: v[1100, 0, 7:9].fill_(float("nan")))
    check(F, np.random.default_rng(9), [4, 1, 3], [1300, 70, 66], 1, 1, d, dtype, edit=lambda q, k, v, a, b: v[1298, 0, 7:9].fill_(float("nan")))


def test_offsets_that_do_not_ascend_or_run_over(F):
    """Row numbers outside the tensors are taken as their ends (and refused with the index checks on)."""
    q, k, v = (torch.randn(8, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(3))
    want = F.packed_attn(q, k, v, i32([0, 8]))
    assert torch.equal(F.packed_attn(q, k, v, i32([-5, 99])), want)
    F.set_index_checks(True)
    try:
        F.packed_attn(q, k, v, i32([0, 3, 8]), i32([0, 3, 7]))
        for cu_q, cu_k in (([0, 5, 4], None), ([1, 5, 8], None), ([0, 5, 9], None), ([0, 4, 8], [0, 9, 9]), ([0, 4, 8], [0, 5, 3])):
            with pytest.raises(F.FlashLoopError, match="FL_E_RANGE"):
                F.packed_attn(q, k, v, i32(cu_q), None if cu_k is None else i32(cu_k))
    finally:
        F.set_index_checks(False)


def test_positions_outside_the_table(F):
    q, k, v = (torch.randn(40, 2, 64, device="cuda").to(torch.float16) for _ in range(3))
    got = F.packed_attn(q, k, v, i32([0, 40]), table=F.rope_table(32, 64))
    assert torch.isnan(got[32:]).all() and not torch.isnan(got[:32]).any()


def test_rows_far_apart(F):
    """Rows whose offsets pass 32 bits: a view with a row stride of 2^23 elements over 600 rows."""
    n, row = 600, 1 << 23
    whole = torch.empty(n * row, dtype=torch.bfloat16, device="cuda")
    parts = []
    for i in range(3):
        x = whole.as_strided((n, 1, 64), (row, 64, 1), 64 * i)
        x.copy_(torch.randn(n, 1, 64, device="cuda"))
        parts.append(x)
    out = whole.as_strided((n, 1, 64), (row, 64, 1), 64 * 3)
    cu = i32([0, 200, 600])
    F.packed_attn(*parts, cu, out=out)
    assert torch.equal(out, F.packed_attn(*(x.contiguous() for x in parts), cu))


def test_a_batch_is_its_sequences(F):
    """Each sequence alone gives the bits that it has in the batch where the work is cut the same way, and its numbers everywhere."""
    nq = [130, 64, 1, 77]
    cu = offsets(nq)
    q, k, v = (torch.randn(cu[-1], h, 128, device="cuda").to(torch.bfloat16) for h in (4, 2, 2))
    whole = F.packed_attn(q, k, v, i32(cu))
    for a, b in zip(cu, cu[1:]):
        one = F.packed_attn(q[a:b], k[a:b], v[a:b], i32([0, b - a]))
        assert torch.allclose(one.float(), whole[a:b].float(), atol=2e-2, rtol=2 ** -7)
    assert torch.equal(F.packed_attn(q, k, v, i32(cu)), whole)         # the same bits again


def test_graphs_that_share_a_workspace_and_streams(F):
    """Two captured calls with one workspace, replayed in turn with other offsets and eager work between; then both at once on
    streams of their own."""
    g = torch.Generator(device="cuda").manual_seed(0)
    q, k, v = (torch.randn(2500, h, 128, generator=g, device="cuda").to(torch.bfloat16) for h in (4, 2, 2))
    calls = [(q[:600], k, v, i32([0, 400, 600]), i32([0, 1800, 2500])), (q, k, v, i32([0, 2000, 2500]), None)]
    ws = max((w for w in (F.packed_attn_ws(c[0], k, 2) for c in calls) if w is not None), key=lambda t: t.numel(), default=None)
    outs = [torch.empty_like(c[0]) for c in calls]
    eager = [F.packed_attn(*c) for c in calls]
    graphs = []
    for c, o in zip(calls, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            F.packed_attn(*c, out=o, ws=ws)
        graphs.append(graph)
    for i in range(4):
        for graph, o, want in zip(graphs, outs, eager):
            o.fill_(0)
            graph.replay()
            assert torch.equal(o, want), f"replay {i}"
        torch.cuda.synchronize()
    calls[1][3].copy_(i32([0, 777, 2400]))                          # the graph reads the present offsets
    want = F.packed_attn(q, k, v, i32([0, 777, 2400]))
    for i in range(2):
        outs[1].fill_(5)
        graphs[1].replay()
        assert torch.equal(outs[1][:2400], want[:2400]) and torch.all(outs[1][2400:] == 5)
    want = [F.packed_attn(*c) for c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in calls], [[], []]
    for _ in range(4):
        for i, (c, s) in enumerate(zip(calls, streams)):
            with torch.cuda.stream(s):
                got[i].append(F.packed_attn(*c))
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        assert all(torch.equal(x[:2400], w[:2400]) for x in many)


def test_far_positions(F):
    """Few rows after hundreds of thousands of keys, and a chunk after many."""
    rng = np.random.default_rng(30)
    for window, n_sink in ((0, 0), (5000, 70)):
        check(F, rng, [1, 3], [5, 300000], 2, 1, 64, "bf16", window=window, n_sink=n_sink, hints=(0, 100))
        check(F, rng, [130, 1], [100000, 77], 1, 1, 128, "f16", window=window, n_sink=n_sink, layout="half", rot=64)
