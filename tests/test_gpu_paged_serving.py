"""The paged calls as a server makes them: prompts in chunks, then single positions, for a batch whose sequences come and go;
captured into graphs, on other streams, two at once."""
import numpy as np
import pytest
import torch

from gpu_util import REL_FRO, say
from oracle import paged
from paper_2609_29812_amd import driver

pytestmark = pytest.mark.gpu

FMT = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def raw(t):
    return t.view(torch.uint8).cpu().numpy()


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


class Server:
    """Pages, lengths and block tables of sequences on the host, one layer's cache on the GPU and the oracle's beside it."""

    def __init__(self, F, B, n_pages, max_pages, Hq, Hkv, page, d, fmt, dtype, window=0, n_sink=0):
        self.F, self.fmt, self.dtype, self.page, self.d, self.Hq, self.Hkv = F, fmt, dtype, page, d, Hq, Hkv
        self.window, self.n_sink = window, n_sink
        self.cache = F.paged_cache(n_pages, Hkv, page, d, FMT[fmt])
        for c in self.cache[:2]:
            c.view(torch.uint8).fill_(127)                       # (e4m3: NaN)
        self.codes = [np.full((n_pages, Hkv, page, d), 127, np.uint8) for _ in range(2)]
        self.scale = [np.zeros((n_pages, Hkv), np.float32) for _ in range(2)]
        self.free = list(range(n_pages))
        self.lens = np.zeros(B, np.int32)
        self.tab = np.full((B, max_pages), -1, np.int32)
        self.cs = paged.table(max_pages * page, d).astype(np.float32)
        self.table = torch.from_numpy(self.cs).cuda()

    def place(self, new):
        """Pages for the new positions; pages between the leading positions and the window go back."""
        for b, n in enumerate(new):
            for p in range(-(-self.lens[b] // self.page), -(-(self.lens[b] + n) // self.page)):
                self.tab[b, p] = self.free.pop(0)
            self.lens[b] += n
            if self.window and n:
                first = max(0, self.lens[b] - n - self.window + 1) // self.page
                for p in range(-(-self.n_sink // self.page), first):
                    if self.tab[b, p] >= 0:
                        self.free.append(int(self.tab[b, p]))
                        self.tab[b, p] = -1

    def end(self, b):
        self.free += [int(p) for p in self.tab[b] if p >= 0]
        self.tab[b], self.lens[b] = -1, 0

    def step(self, rng, new, what):
        self.place(new)
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        T = int(cu[-1])
        q, k, v = (torch.from_numpy(rng.normal(size=(T, h, self.d)) * amp).to(self.dtype)
                   for h, amp in ((self.Hq, 1.0), (self.Hkv, rng.uniform(0.5, 3.0)), (self.Hkv, rng.uniform(0.5, 3.0))))
        o = driver.paged_step(self.cache, q.cuda(), k.cuda(), v.cuda(), i32(cu), i32(self.lens), i32(self.tab), table=self.table,
                              window=self.window, n_sink=self.n_sink, max_q=max(new), max_len=int(self.lens.max()))
        torch.cuda.synchronize()
        pos = np.concatenate([np.arange(self.lens[b] - n, self.lens[b]) for b, n in enumerate(new)]).astype(int)
        kx = paged.rotate(k.double().numpy(), self.cs[pos]).astype(np.float32).astype(np.float64)
        for x, c, s, gc, gs in ((kx, self.codes[0], self.scale[0], self.cache[0], self.cache[2]),
                                (v.double().numpy(), self.codes[1], self.scale[1], self.cache[1], self.cache[3])):
            paged.append(x, cu, self.lens, self.tab, c, s, self.fmt)
            assert np.array_equal(gs.cpu().numpy(), s), what
            same = raw(gc) == c
            if self.fmt == "e4m3":                               # (what no sequence holds: a NaN of either sign)
                same |= ((raw(gc) & 127) == 127) & ((c & 127) == 127)
            at = np.argwhere(~same)[:1]
            assert same.all(), (what, at, raw(gc)[tuple(at[0])], c[tuple(at[0])])
        want, *_ = paged.attend(paged.rotate(q.double().numpy(), self.cs[pos]), cu, self.lens, self.tab, *self.codes,
                                     *self.scale, self.fmt, self.d ** -0.5, self.window, self.n_sink)
        err = np.linalg.norm(o.cpu().double().numpy() - want) / np.linalg.norm(want)
        say(f"  {what}: {list(new)} of {self.lens.tolist()}: rel={err:.2e}")
        assert err <= REL_FRO + torch.finfo(self.dtype).eps / 2, what
        return o


@pytest.mark.parametrize("fmt,dtype,d,page,window,n_sink", [("int8", torch.bfloat16, 128, 64, 0, 0),
                                                            ("e4m3", torch.float16, 64, 16, 50, 5)])
def test_prompts_chunks_and_single_positions(F, fmt, dtype, d, page, window, n_sink):
    rng = np.random.default_rng(1)
    s = Server(F, 4, 60 if page == 16 else 20, 30 if page == 16 else 8, 8, 2, page, d, fmt, dtype, window, n_sink)
    s.step(rng, [100, 37, 0, 1], "prompts")
    s.step(rng, [150, 0, 64, 1], "a chunk, a new prompt, a single position")
    for i in range(3):
        s.step(rng, [1, 1, 1, 1], f"decode {i}")
    s.end(1)
    s.step(rng, [1, 90, 1, 3], "a sequence replaced, three positions checked at once")
    for i in range(20):
        s.step(rng, [1, 1, 0, 2], f"decode over a page's border {i}")


def _batch(seed, B=5, T=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(B if T is None else T, h, 128, generator=g, device="cuda").to(torch.bfloat16) for h in (8, 2, 2)]


def test_graph_replays_match_eager_steps(F):
    """A step captured once and replayed with other lengths, tables and values in the same buffers, eager steps between."""
    B, page, max_pages = 5, 16, 40
    table = F.rope_table(page * max_pages, 128)
    tab = i32(np.arange(B * max_pages).reshape(B, max_pages))
    past = np.array([3, 0, 200, 77, 610 - 12])
    one, two = (F.paged_cache(B * max_pages, 2, page, 128) for _ in range(2))
    for c in one:
        c.view(torch.uint8).fill_(0)
    fill = torch.randn(int(past.sum()), 4, 128, device="cuda").to(torch.bfloat16)
    cu0 = i32(np.concatenate([[0], np.cumsum(past)]))
    F.paged_append(fill[:, :2], fill[:, 2:], cu0, i32(past), tab, *one)
    for a, b in zip(one, two):
        b.copy_(a)
    q, k, v = _batch(0)
    cu, lens, t = i32(np.arange(B + 1)), i32(past + 1), tab.clone()
    ws = F.paged_attn_ws(q, t, one[0], max_q=1, max_len=page * max_pages)
    out = torch.empty_like(q)
    run = lambda: driver.paged_step(one, q, k, v, cu, lens, t, table=table, max_q=1, max_len=page * max_pages, out=out, ws=ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()                                                    # (the same positions: the replay's first step repeats it)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(6):
        for x, y in zip((q, k, v), _batch(i)):
            x.copy_(y)
        lens.copy_(i32(past + 1 + i))
        out.fill_(float("nan"))
        graph.replay()
        got = out.clone()
        want = driver.paged_step(two, *_batch(i), cu, i32(past + 1 + i), tab, table=table, max_q=1, max_len=page * max_pages)
        torch.cuda.synchronize()
        assert torch.equal(got, want), f"replay {i}"
        if i > 0:                                                # (the first token was stored twice on one side)
            for a, b in zip(one, two):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), f"replay {i}"


def test_prompt_graphs_that_share_a_workspace(F):
    """Two captured prompt calls with one workspace, replayed in turn with eager work between."""
    page, max_pages = 64, 40
    cache = F.paged_cache(2 * max_pages, 2, page, 128)
    tab = i32(np.random.default_rng(0).permutation(2 * max_pages).reshape(2, max_pages))
    _, k, v = _batch(1, T=4000)
    F.paged_append(k, v, i32([0, 2200, 4000]), i32([2200, 1800]), tab, *cache)
    calls = []
    for new, lens in (([700, 300], [2200, 1800]), ([300, 290], [1500, 1700])):
        q = _batch(len(calls), T=sum(new))[0]
        args = (q, i32([0, new[0], sum(new)]), i32(lens), tab, *cache)
        calls.append((args, dict(max_q=max(new), max_len=2200), torch.empty_like(q)))
    need = max((F.paged_attn_ws(a[0], tab, cache[0], **kw) for a, kw, _ in calls), key=lambda t: t.numel())
    eager = [F.paged_attn(*a, **kw) for a, kw, _ in calls]
    graphs = []
    for a, kw, out in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            F.paged_attn(*a, **kw, out=out, ws=need)
        graphs.append(g)
    for i in range(4):
        for (a, kw, out), g, want in zip(calls, graphs, eager):
            out.fill_(0)
            g.replay()
            assert torch.equal(out, want), f"replay {i}"
        torch.cuda.synchronize()


def test_two_streams_at_once(F):
    """Calls on two streams of their own, with workspaces of their own: the bits of the calls one after the other."""
    page, max_pages = 64, 40
    cache = F.paged_cache(2 * max_pages, 2, page, 128)
    tab = i32(np.arange(2 * max_pages).reshape(2, max_pages))
    _, k, v = _batch(2, T=4000)
    F.paged_append(k, v, i32([0, 2200, 4000]), i32([2200, 1800]), tab, *cache)
    few, many = _batch(3, T=2)[0], _batch(4, T=600)[0]
    calls = [((few, i32([0, 1, 2]), i32([2200, 1800]), tab, *cache), dict(max_q=1, max_len=2200)),
             ((many, i32([0, 400, 600]), i32([2200, 1800]), tab, *cache), dict(max_q=400, max_len=2200))]
    want = [F.paged_attn(*a, **kw) for a, kw in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = [[], []]
    for _ in range(5):
        for i, ((a, kw), s) in enumerate(zip(calls, streams)):
            with torch.cuda.stream(s):
                got[i].append(F.paged_attn(*a, **kw))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(x, w) for x in g)
