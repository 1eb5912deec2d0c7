"""Appending to pages whose held scale is smaller than any that an append writes (a cache that a caller filled)."""
import numpy as np
import pytest
import torch

from gpu_util import say

from test_gpu_paged import i32, raw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [torch.int8, torch.float8_e4m3fn])
@pytest.mark.parametrize("held", [2.0 ** -149, 1e-40, 2.0 ** -126, 2.0 ** -115, 2.0 ** -108.5])
@pytest.mark.parametrize("new", [2, 60])
def test_values_that_count_as_zero(F, new, held, fmt):
    """Values below 2^-100 are codes of 0 there, and the scale stays; larger ones set it."""
    page, H, d = 128, 2, 64
    cache = F.paged_cache(2, H, page, d, fmt)
    for size, grows in ((0.0, False), (2.0 ** -101, False), (2.0 ** -100, True)):
        say(f"  {fmt} held {held:.2e} new values {size:.2e}")
        for c in cache[:2]:
            c.view(torch.uint8).fill_(17)
        for c in cache[2:]:
            c.fill_(held)
        was = cache[2].clone()
        g = torch.Generator().manual_seed(new)
        x = (torch.rand(new, H, d, generator=g) - 0.5) * 2 * size
        x[0, :, 0] = -size
        x = x.to(torch.bfloat16)
        F.paged_append(x.cuda(), (-x).cuda(), i32([0, new]), i32([5 + new]), i32([[1]]), *cache)
        for c, s, y in ((cache[0], cache[2], x), (cache[1], cache[3], -x)):
            at = c[1, :, 5:5 + new]
            assert torch.equal(s[0], was[0])
            if not grows:
                assert torch.equal(s, was) and np.all(raw(at) == 0)
                assert np.all(raw(c[1, :, :5]) == 17)
            else:
                got = at.float().cpu().double() * s[1].cpu().double()[:, None, None]
                want = y.double().transpose(0, 1)
                assert torch.all(s[1] >= 2.0 ** -108)
                # (int8: half a step of the scale, at most size / 64; e4m3: 2^-4 of the value, or half of its least step)
                assert torch.all((got - want).abs() <= torch.maximum(want.abs() * 2.0 ** -4, s[1].cpu().double()[:, None, None] * 0.5))
