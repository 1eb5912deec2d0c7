"""Rotary positions at the ends of their range."""
import numpy as np
import pytest
import torch

from gpu_util import say
from oracle import paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pos", [2 ** 31 - 1, 2 ** 31 - 33])
def test_the_longest_tables(F, n_pos):
    """All positions that an int32 names (137 GB): the last rows, some between, the first."""
    need = n_pos * 8 * 8
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < need + (8 << 30):
        pytest.skip("not enough free memory")
    say(f"table of {n_pos} positions")
    out = torch.empty(n_pos, 8, 2, dtype=torch.float32, device="cuda")
    out[-64:] = 7.0
    F.rope_table(n_pos, 16, base=5e5, out=out)
    f, _ = paged.frequencies(16, base=5e5)
    for lo, hi in ((0, 300), (2 ** 20 - 9, 2 ** 20 + 9), (2 ** 30 - 40, 2 ** 30 + 40), (n_pos - 300, n_pos)):
        got = out[lo:hi].cpu().double().numpy()
        angle = np.arange(lo, hi)[:, None] * f
        want = np.stack([np.cos(angle), np.sin(angle)], axis=-1)
        # 2 ulp, the frequency's rounding on either side (2^-51 and 2^-52 of an angle), the reference's product
        assert np.all(np.abs(got - want) <= 2.0 ** -22 + angle[..., None] * 2.0 ** -50)
    del out, got
    torch.cuda.empty_cache()
