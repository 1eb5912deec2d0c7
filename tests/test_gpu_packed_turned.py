"""Packed attention that turns its queries itself gives the bits of the call over queries that rope has turned."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 48), (64, 64), (64, 16)])
def test_turned_queries_are_those_of_rope(F, d, rot, dtype, layout):
    g = torch.Generator(device="cuda").manual_seed(rot)
    nq, nk = [1500, 1, 0, 700], [1500, 4000, 30, 2500]
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(n)]) for n in (nq, nk))
    q = torch.randn(sum(nq), 8, d, generator=g, device="cuda").to(dtype)
    k, v = (torch.randn(sum(nk), 2, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    table = F.rope_table(max(nk), rot)
    pos = i32(np.concatenate([np.arange(b - a, b) for a, b in zip(nq, nk)]))
    for qs in (q, q * 1000):
        got = F.packed_attn(qs, k, v, i32(cu_q), i32(cu_k), table=table, layout=layout)
        want = F.packed_attn(F.rope(qs, table, pos=pos, layout=layout), k, v, i32(cu_q), i32(cu_k))
        assert torch.equal(got, want), f"{int((got != want).any(-1).sum())} rows differ"
