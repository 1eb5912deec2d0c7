"""Packed attention whose work is cut into shares: captured calls with one workspace, and calls on streams of their own."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def calls_of(dtype, d):
    """Chunks after long contexts: each call is cut, and needs a workspace."""
    g = torch.Generator(device="cuda").manual_seed(d)
    q, k, v = (torch.randn(n, h, d, generator=g, device="cuda").to(dtype) for n, h in ((700, 4), (9000, 2), (9000, 2)))
    return [(q[:500], k, v, i32([0, 300, 500]), i32([0, 4400, 9000])), (q, k[:5000], v[:5000], i32([0, 700]), i32([0, 5000])),
            (q[:130], k, v, i32([0, 130, 130]), i32([0, 6000, 9000]))]


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float16, 64)])
def test_graphs_that_share_a_workspace(F, dtype, d):
    calls = calls_of(dtype, d)
    wss = [F.packed_attn_ws(c[0], c[1], c[3].numel() - 1) for c in calls]
    assert all(w is not None for w in wss)
    ws = max(wss, key=lambda t: t.numel())
    eager = [F.packed_attn(*c) for c in calls]
    outs, graphs = [torch.empty_like(c[0]) for c in calls], []
    for c, o in zip(calls, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            F.packed_attn(*c, out=o, ws=ws)
        graphs.append(graph)
    for i in range(4):
        for j, (graph, o, want) in enumerate(zip(graphs, outs, eager)):
            o.fill_(0)
            graph.replay()
            assert torch.equal(o, want), f"replay {i} of call {j}"
        assert torch.equal(F.packed_attn(*calls[i % 3], ws=ws), eager[i % 3])
        ws.fill_(255)
        torch.cuda.synchronize()
    calls[0][3].copy_(i32([0, 77, 440]))                            # the graph reads the present offsets
    want = F.packed_attn(*calls[0])
    for i in range(2):
        outs[0].fill_(5)
        graphs[0].replay()
        assert torch.equal(outs[0][:440], want[:440]) and torch.all(outs[0][440:] == 5), f"replay {i}"


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float16, 64)])
def test_streams_at_once(F, dtype, d):
    calls = calls_of(dtype, d)
    want = [F.packed_attn(*c) for c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in calls], [[] for _ in calls]
    wss = [F.packed_attn_ws(c[0], c[1], c[3].numel() - 1) for c in calls]
    for _ in range(5):
        for c, s, ws, many in zip(calls, streams, wss, got):
            with torch.cuda.stream(s):
                many.append(F.packed_attn(*c, ws=ws))               # its own workspace, given
                many.append(F.packed_attn(*c))                      # and made in the call
    torch.cuda.synchronize()
    for w, many in zip(want, got):
        assert all(torch.equal(x, w) for x in many)
