"""The 4-bit paged calls as a server makes them: whole prompts, chunks and single positions of sequences that come and go; captured
into graphs that share a workspace, on other streams, in caches beyond 4 GiB; and a cache read back into the states of the sparse
loops."""
import numpy as np
import pytest
import torch

from gpu_util import REL_FRO, say
from oracle import paged, paged4
from paper_2609_29812_amd import driver

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def bits(t):
    return t.view(torch.int16) if t.dtype == torch.float16 else t


class Server:
    """Pages, lengths and block tables of sequences on the host, one layer's cache on the GPU and the oracle's beside it."""

    def __init__(self, F, B, n_pages, max_pages, Hq, Hkv, page, d, fmt, dtype, window=0, n_sink=0):
        self.F, self.fmt, self.dtype, self.page, self.d, self.Hq, self.Hkv = F, fmt, dtype, page, d, Hq, Hkv
        self.window, self.n_sink = window, n_sink
        self.cache = F.paged4_cache(n_pages, Hkv, page, d, fmt)
        self.sides = [paged4.empty(n_pages, Hkv, page, d, fmt) for _ in range(2)]
        for c, m, (hc, hm) in zip(self.cache[:2], self.cache[2:], self.sides):
            c.fill_(0)
            m.view(torch.uint8).fill_(255)                       # (both formats: numbers that read as NaN)
            hm.view(np.uint8)[:] = 255
        self.free = list(range(n_pages))
        self.lens = np.zeros(B, np.int32)
        self.tab = np.full((B, max_pages), -1, np.int32)
        self.cs = paged.table(max_pages * page, d).astype(np.float32)
        self.table = torch.from_numpy(self.cs).cuda()

    def place(self, new, whole):
        """Pages for the new positions; pages between the leading positions and the window go back."""
        for b, n in enumerate(new):
            for p in range(-(-self.lens[b] // self.page), -(-(self.lens[b] + n) // self.page)):
                self.tab[b, p] = self.free.pop(0)
            self.lens[b] += n
            if self.window and n and not whole:
                first = max(0, self.lens[b] - n - self.window + 1) // self.page
                for p in range(-(-self.n_sink // self.page), first):
                    if self.tab[b, p] >= 0:
                        self.free.append(int(self.tab[b, p]))
                        self.tab[b, p] = -1

    def end(self, b):
        self.free += [int(p) for p in self.tab[b] if p >= 0]
        self.tab[b], self.lens[b] = -1, 0

    def step(self, rng, new, what, whole=False):
        self.place(new, whole)
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T = int(cu[-1])
        lens = np.asarray(new, np.int32) if whole else self.lens
        q, k, v = (torch.from_numpy(rng.normal(size=(T, h, self.d)) * amp).to(self.dtype)
                   for h, amp in ((self.Hq, 1.0), (self.Hkv, rng.uniform(0.5, 2.0)), (self.Hkv, rng.uniform(0.5, 2.0))))
        kd, vd = k.cuda(), v.cuda()
        o = driver.paged4_step(self.cache, q.cuda(), kd, vd, i32(cu), i32(lens), i32(self.tab), table=self.table,
                               window=self.window, n_sink=self.n_sink, max_q=max(new), max_len=int(lens.max()), whole=whole)
        torch.cuda.synchronize()
        assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v), what
        pos = np.concatenate([np.arange(lens[b] - n, lens[b]) for b, n in enumerate(new)]).astype(int)
        kx = paged.rotate(k.double().numpy(), self.cs[pos]).astype(np.float32).astype(np.float64)
        rows = []
        for x, (c, m), gc, gm in zip((kx, v.double().numpy()), self.sides, self.cache[:2], self.cache[2:]):
            rows.append(paged4.append(x, cu, lens, self.tab, c, m, self.fmt)[0])
            assert np.array_equal(gm.cpu().numpy().view(np.uint8), m.view(np.uint8)), what
            assert np.array_equal(gc.cpu().numpy(), c), what
        qx = paged.rotate(q.double().numpy(), self.cs[pos])
        near = lambda x: torch.from_numpy(x).to(self.dtype).double().numpy()  # noqa: E731
        seqs = (paged4.packed_seqs(near(rows[0]), near(rows[1]), cu, cu) if whole
                else paged4.paged_seqs(cu, lens, self.tab, self.sides, self.fmt))
        want, *_ = paged4.attend(near(qx) if whole else qx, seqs, self.Hkv, self.d ** -0.5, self.window, self.n_sink)
        err = np.linalg.norm(o.cpu().double().numpy() - want) / np.linalg.norm(want)
        say(f"  {what}: {list(new)} of {lens.tolist()}: rel={err:.2e}")
        assert err <= REL_FRO + torch.finfo(self.dtype).eps / 2, what


@pytest.mark.parametrize("fmt,dtype,d,page,window,n_sink", [("int4", torch.bfloat16, 128, 64, 0, 0),
                                                            ("e2m1", torch.float16, 64, 16, 50, 5),
                                                            ("int4", torch.float16, 64, 32, 0, 0)])
def test_prompts_chunks_and_single_positions(F, fmt, dtype, d, page, window, n_sink):
    rng = np.random.default_rng(1)
    s = Server(F, 4, {16: 60, 32: 36, 64: 20}[page], {16: 30, 32: 16, 64: 8}[page], 8, 2, page, d, fmt, dtype, window, n_sink)
    s.step(rng, [100, 37, 0, 1], "whole prompts", whole=True)
    s.step(rng, [150, 0, 64, 1], "a chunk, a new prompt, a single position")
    for i in range(3):
        s.step(rng, [1, 1, 1, 1], f"decode {i}")
    s.end(1)
    s.step(rng, [1, 90, 1, 3], "a sequence replaced, three positions checked at once")
    for i in range(20):
        s.step(rng, [1, 1, 0, 2], f"decode over a page's border {i}")


def _batch(seed, T):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(T, h, 128, generator=g, device="cuda").to(torch.bfloat16) for h in (8, 2, 2)]


def _filled(F, fmt, page, max_pages, lens, seed=1, spare=0):
    """A cache with len(lens) sequences of these lengths, and its block table."""
    B = len(lens)
    cache = F.paged4_cache(B * max_pages + spare, 2, page, 128, fmt)
    for c in cache:
        c.view(torch.uint8).fill_(0)
    tab = i32(np.random.default_rng(seed).permutation(B * max_pages).reshape(B, max_pages))
    _, k, v = _batch(seed, int(sum(lens)))
    F.paged4_append(k, v, i32(np.concatenate([[0], np.cumsum(lens)])), i32(lens), tab, *cache)
    return cache, tab


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_graph_replays_match_eager_steps(F, fmt):
    """A step captured once and replayed with other lengths and values in the same buffers, eager steps between."""
    B, page, max_pages = 5, 16, 40
    table = F.rope_table(page * max_pages, 128)
    past = np.array([3, 0, 200, 77, 610 - 12])
    one, tab = _filled(F, fmt, page, max_pages, past)
    two = [c.clone() for c in one]
    q, k, v = _batch(0, B)
    cu, lens, t = i32(np.arange(B + 1)), i32(past + 1), tab.clone()
    kw = dict(table=table, max_q=1, max_len=page * max_pages)
    ws = F.paged4_attn_ws(q, t, one[0], max_q=1, max_len=page * max_pages)
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        driver.paged4_step(one, q, k, v, cu, lens, t, out=out, ws=ws, **kw)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        driver.paged4_step(one, q, k, v, cu, lens, t, out=out, ws=ws, **kw)
    for i in range(6):
        for x, y in zip((q, k, v), _batch(i, B)):
            x.copy_(y)
        lens.copy_(i32(past + 1 + i))
        out.fill_(float("nan"))
        graph.replay()
        got = out.clone()
        want = driver.paged4_step(two, *_batch(i, B), cu, i32(past + 1 + i), tab, **kw)
        torch.cuda.synchronize()
        assert torch.equal(got, want), f"replay {i}"
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(one, two)), f"replay {i}"


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_graphs_that_share_a_workspace(F, fmt):
    """Captured calls with one workspace - two of many rows, two of few, packed chunks - replayed in turn with eager work between."""
    page, max_pages = 64, 60
    cache, tab = _filled(F, fmt, page, max_pages, [3600, 3200])
    calls = []
    for new, lens in (([700, 300], [3600, 3200]), ([1, 1], [3600, 3200]), ([300, 290], [2900, 3100]), ([2, 0], [1999, 7])):
        q = _batch(len(calls), sum(new))[0]
        args = (q, i32([0, new[0], sum(new)]), i32(lens), tab, *cache)
        calls.append((F.paged4_attn, args, dict(max_q=max(new), max_len=3600), torch.empty_like(q)))
    q, k, v = _batch(9, 6000)
    calls.append((F.packed_attn, (q[:500], k, v, i32([0, 300, 500]), i32([0, 3100, 6000])), {}, torch.empty_like(q[:500])))
    wss = [F.paged4_attn_ws(a[0], tab, cache[0], **kw) for f, a, kw, _ in calls[:-1]] + [F.packed_attn_ws(q[:500], k, 2)]
    ws = max((w for w in wss if w is not None), key=lambda t: t.numel())
    assert sum(w is not None for w in wss) >= 3
    eager = [f(*a, **kw) for f, a, kw, _ in calls]
    graphs = []
    for f, a, kw, out in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f(*a, **kw, out=out, ws=ws)
        graphs.append(graph)
    for i in range(4):
        for j, ((*_, out), graph, want) in enumerate(zip(calls, graphs, eager)):
            out.fill_(0)
            graph.replay()
            assert torch.equal(out, want), f"replay {i} of call {j}"
        ws.fill_(255)
        torch.cuda.synchronize()


def test_two_streams_at_once(F):
    """Calls on streams of their own, with workspaces of their own: the bits of the calls one after the other."""
    page, max_pages = 64, 40
    cache, tab = _filled(F, "int4", page, max_pages, [2200, 1800], seed=2)
    few, many = _batch(3, 2)[0], _batch(4, 600)[0]
    calls = [((few, i32([0, 1, 2]), i32([2200, 1800]), tab, *cache), dict(max_q=1, max_len=2200)),
             ((many, i32([0, 400, 600]), i32([2200, 1800]), tab, *cache), dict(max_q=400, max_len=2200))]
    want = [F.paged4_attn(*a, **kw) for a, kw in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in calls], [[], []]
    for _ in range(5):
        for i, ((a, kw), s) in enumerate(zip(calls, streams)):
            with torch.cuda.stream(s):
                got[i].append(F.paged4_attn(*a, **kw))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(x, w) for x in g)


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_a_cache_beyond_4_gib(F, fmt):
    """Pages whose codes lie behind 2^32 bytes of a side: the bits of the same calls over a small cache."""
    page, per = 128, 64 * 2 * 128                                # bytes of a page's codes: two heads of 128 channels
    n_pages = (9 << 29) // per + 64
    B, max_pages = 3, 10
    lens, past = np.array([1200, 1, 700]), np.array([1100, 0, 699])
    tab = np.random.default_rng(3).permutation(B * max_pages).reshape(B, max_pages)
    big, small = F.paged4_cache(n_pages, 2, page, 128, fmt), F.paged4_cache(B * max_pages, 2, page, 128, fmt)
    high = i32(tab + n_pages - B * max_pages)
    cu = i32(np.concatenate([[0], np.cumsum(lens)]))
    q, k, v = _batch(5, int(lens.sum()))
    got, want = [], []
    for cache, t, res in ((big, high, got), (small, i32(tab), want)):
        F.paged4_append(k, v, cu, i32(lens), t, *cache)
        res += F.paged4_read(cu, i32(lens), t, *cache, int(lens.sum()))
        res.append(F.paged4_attn(q, cu, i32(lens), t, *cache))
        new = i32(np.concatenate([[0], np.cumsum(lens - past)]))
        res.append(F.paged4_attn(q[:int((lens - past).sum())], new, i32(lens), t, *cache, max_len=1200))
        res.append(F.paged4_attn(q[:B], i32(np.arange(B + 1)), i32(lens), t, *cache, max_q=1, max_len=1200))
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        assert not torch.isnan(b).any() and torch.equal(a, b), f"result {i}"


def test_read_back_into_the_sparse_loops_states(F):
    """A decoded position of a sparse loop whose states come out of a 4-bit cache: the call over the rows that append gave."""
    B, N, H, d, page = 2, 192, 2, 128, 64
    g = torch.Generator(device="cuda").manual_seed(7)
    k, v = (torch.randn(B * N, H, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    cu, lens, tab = i32([0, N, 2 * N]), i32([N, N]), i32([[3, 0, 5], [1, 4, 2]])
    cache = F.paged4_cache(6, H, page, d, "int4")
    kr, vr = torch.empty_like(k), torch.empty_like(v)
    F.paged4_append(k, v, cu, lens, tab, *cache, k_rows=kr, v_rows=vr)
    k_state, v_state = (torch.full((B, N, H, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    F.paged4_read(cu, lens, tab, *cache, B * N, k_out=k_state.view(B * N, H, d), v_out=v_state.view(B * N, H, d))
    assert torch.equal(k_state.view_as(kr), kr) and torch.equal(v_state.view_as(vr), vr)
    q = torch.randn(B, N, H, d, generator=g, device="cuda").to(torch.bfloat16)
    o, lse = F.dense_attn(q, k_state, v_state)
    packed = F.packed_attn(q.view(B * N, H, d), kr, vr, cu)
    assert torch.linalg.norm(packed.float() - o.view_as(packed)) <= 2 * (REL_FRO + 2.0 ** -8) * torch.linalg.norm(o)
