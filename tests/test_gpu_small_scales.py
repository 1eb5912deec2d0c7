"""Scores that are 0 to fp32: queries at or near 0 under any sm_scale, the smallest included.  A row's output is the mean of the values
that it sees, its log-normaliser the logarithm of their number, and what it does not see stays out."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SCALES = [1.0, 1e-6, 1e-8, 1e-20, 1e-38, 1e-44]


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32).cuda()


def check(got, lse, v, lens, cu, step, window, what):
    """Equal probabilities are exact powers of two or near 1; sums of n values in fp32, one rounding of `step` of the output, and for
    values in fp16 one of 2^-11 of them."""
    got, lse = got.cpu().double().numpy(), lse.cpu().double().numpy()
    for b, L in enumerate(lens):
        n = cu[b + 1] - cu[b]
        for t in range(n):
            i = L - n + t
            x = v[b][max(0, i - window + 1) if window else 0:i + 1]
            tol = step * np.abs(x.mean(axis=0)) + (2.0 ** -11 + 2.0 ** -16) * np.abs(x).mean(axis=0) + 2.0 ** -24
            assert bool((np.abs(got[cu[b] + t] - x.mean(axis=0)[:, None]).transpose(0, 2, 1) <= tol[:, :, None]).all()), (what, b, t)
            assert bool((np.abs(lse[cu[b] + t] - math.log(len(x))) <= 2.0 ** -20 * 8).all()), (what, b, t)


@pytest.mark.parametrize("size", [0.0, 1e-38, 1e-30])
@pytest.mark.parametrize("fmt,dtype", [("int4", torch.bfloat16), ("e2m1", torch.bfloat16), ("int4", torch.float16)])
def test_attention_over_the_4_bit_cache(F, fmt, dtype, size):
    page, d, new, lens = 16, 64, [100, 1, 30], [100, 77, 130]
    cu, at = [0, 100, 101, 131], [0, 100, 177, 307]
    tab = i32(np.random.default_rng(1).permutation(30).reshape(3, 10))
    cache = F.paged4_cache(30, 1, page, d, fmt)
    k, v = (torch.randn(307, 1, d, device="cuda").to(dtype) for _ in range(2))
    F.paged4_append(k, v, i32(at), i32(lens), tab, *cache)
    rows = F.paged4_read(i32(at), i32(lens), tab, *cache, 307, dtype=torch.float16)[1].cpu().double().numpy()
    seqs = [rows[a:b] for a, b in zip(at, at[1:])]
    q = torch.randn(131, 2, d, device="cuda").mul(size).to(dtype)
    for scale in SCALES:
        for window in (0, 20):
            for max_q in (1, 16, 100):
                lse = torch.zeros(131, 2, device="cuda")
                got = F.paged4_attn(q, i32(cu), i32(lens), tab, *cache, sm_scale=scale, window=window, max_q=max_q, lse=lse)
                check(got, lse, seqs, lens, cu, torch.finfo(dtype).eps / 2, window, f"scale {scale} window {window} max_q {max_q}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_packed_attention(F, dtype):
    lens, cu = [100, 1, 70], [0, 100, 101, 171]
    k, v = (torch.randn(171, 1, 64, device="cuda").to(dtype) for _ in range(2))
    q = torch.zeros(171, 2, 64, dtype=dtype, device="cuda")
    seqs = [v.cpu().double().numpy()[a:b] for a, b in zip(cu, cu[1:])]
    for scale in SCALES:
        for window in (0, 20):
            lse = torch.zeros(171, 2, device="cuda")
            got = F.packed_attn(q, k, v, i32(cu), sm_scale=scale, window=window, lse=lse)
            check(got, lse, seqs, lens, cu, torch.finfo(dtype).eps / 2, window, f"scale {scale} window {window}")
