"""Offsets that do not ascend, in calls whose work is cut into shares: they end, write the rows of the call alone, and leave the calls
after them what they were.  (What they write is of no meaning; with the index checks on they are refused.)"""
import numpy as np
import pytest
import torch

from gpu_util import say
from test_prompt_shares import OTHERS

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def check(call, q, cu, B):
    """call(q, offsets, out, ws) of one sequence after others, before and after the same with odd offsets."""
    T, Hq, d = q.shape
    plain = [0] + [T] * B
    want = call(q, i32(plain), torch.empty_like(q))
    out = torch.full((T + 2, Hq, d), 7.0, dtype=q.dtype, device="cuda")
    call(q, i32(cu), out[1:T + 1])
    torch.cuda.synchronize()
    assert torch.all(out[0] == 7) and torch.all(out[-1] == 7)
    assert torch.equal(call(q, i32(plain), torch.empty_like(q)), want)


@pytest.mark.parametrize("case", range(len(OTHERS)))
def test_packed_offsets_that_do_not_ascend(F, case):
    cu, T, G = OTHERS[case]
    B, Tk = len(cu) - 1, 6000
    q = torch.randn(T, G, 64, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(Tk, 1, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    cu_k, ws = i32([0] + [Tk] * B), F.packed_attn_ws(q, k, B, max_k=Tk)
    assert ws is not None
    say(f"  packed {cu}")
    check(lambda q, c, out: F.packed_attn(q, k, v, c, cu_k, max_k=Tk, out=out, ws=ws), q, cu, B)


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
@pytest.mark.parametrize("case", range(len(OTHERS)))
def test_4_bit_offsets_that_do_not_ascend(F, case, fmt):
    cu, T, G = OTHERS[case]
    B, page, n_pages, L = len(cu) - 1, 64, 128, 6000
    cache = F.paged4_cache(n_pages, 1, page, 64, fmt)
    k = torch.randn(L, 1, 64, device="cuda").to(torch.bfloat16)
    tab = i32(np.stack([np.random.default_rng(b).permutation(n_pages) for b in range(B)]))
    F.paged4_append(k, k, i32([0, L]), i32([L]), tab[:1].contiguous(), *cache)
    q = torch.randn(T, G, 64, device="cuda").to(torch.bfloat16)
    lens, ws = i32([L] * B), F.paged4_attn_ws(q, tab, cache[0], max_q=T)
    assert ws is not None
    say(f"  4 bits {cu}")
    check(lambda q, c, out: F.paged4_attn(q, c, lens, tab, *cache, max_q=T, out=out, ws=ws), q, cu, B)


@pytest.mark.parametrize("fmt", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("case", range(len(OTHERS)))
def test_8_bit_offsets_that_do_not_ascend(F, case, fmt):
    cu, T, G = OTHERS[case]
    B, page, n_pages, L = len(cu) - 1, 64, 128, 6000
    cache = F.paged_cache(n_pages, 1, page, 64, fmt)
    k = torch.randn(L, 1, 64, device="cuda").to(torch.bfloat16)
    tab = i32(np.stack([np.random.default_rng(b).permutation(n_pages) for b in range(B)]))
    F.paged_append(k, k, i32([0, L]), i32([L]), tab[:1].contiguous(), *cache)
    q = torch.randn(T, G, 64, device="cuda").to(torch.bfloat16)
    lens, ws = i32([L] * B), F.paged_attn_ws(q, tab, cache[0], max_q=T)
    assert ws is not None
    say(f"  8 bits {cu}")
    check(lambda q, c, out: F.paged_attn(q, c, lens, tab, *cache, max_q=T, out=out, ws=ws), q, cu, B)
