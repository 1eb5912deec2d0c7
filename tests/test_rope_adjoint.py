"""The rotation's inverse as its gradient: <w, rope(x)> = <inverse(w), x>, with w near rope(x), so that what is not the adjoint
misses by a good part of the product itself; the wrong ones are planted on the CPU.

Both sides are rounded once to the type (half a step of each value) after fp32 sums of two rounded products (2^-22 of the
magnitudes), so they differ by at most sum |w| (u |y| + 2^-22 m_y) + sum |x| (u |g| + 2^-22 m_g), m the rotation of magnitudes with
magnitudes."""
import numpy as np
import pytest
import torch

from oracle import paged

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
CASES = [(33, 2, 64, 64, "half", "f16", dict(scaling="yarn", factor=2.0, orig_len=16)), (1, 1, 16, 16, "interleaved", "f16", {}),
         (130, 3, 128, 96, "interleaved", "bf16", {}), (257, 1, 128, 128, "half", "bf16", dict(scaling="ntk", factor=4.0)),
         (9, 5, 200, 48, "half", "f16", dict(scaling="linear", factor=3.0))]


def case(T, H, d, rot, layout, dtype, kw):
    """Values of the type in fp64 and the table in fp32, at positions from 3 on."""
    rng = np.random.default_rng(T + d)
    def to(a): return torch.from_numpy(a).to(DT[dtype]).double().numpy()  # noqa: E704
    cs = paged.table(T + 3, rot, **kw).astype(np.float32)
    x = to(rng.normal(size=(T, H, d)))
    w = to(paged.rotate(x, cs[3:], layout) + 0.3 * rng.normal(size=x.shape))
    return x, w, cs


def bound(x, w, y, g, cs, layout, dtype):
    c = np.abs(cs.astype(np.float64))
    def mag(v): return np.maximum(*(np.abs(paged.rotate(np.abs(v), c * [1, s], layout)) for s in (1, -1)))  # noqa: E704
    u = torch.finfo(DT[dtype]).eps / 2
    return (np.abs(w) * (u * np.abs(y) + 2.0 ** -22 * mag(x))).sum() + (np.abs(x) * (u * np.abs(g) + 2.0 ** -22 * mag(w))).sum()


@pytest.mark.parametrize("args", CASES)
def test_what_is_not_the_adjoint_fails(args):
    T, H, d, rot, layout, dtype, kw = args
    x, w, cs = case(*args)
    cs = cs[3:]
    y, g = paged.rotate(x, cs, layout), paged.rotate(w, cs, layout, inverse=True)
    limit, want = bound(x, w, y, g, cs, layout, dtype), (w * y).sum()
    assert abs((g * x).sum() - want) <= 1e-9 * want
    other = "interleaved" if layout == "half" else "half"
    for name, wrong in (("zeros", 0 * w), ("unrotated", w), ("forward", paged.rotate(w, cs, layout)),
                        ("other pairs", paged.rotate(w, cs, other, inverse=True)), ("a scale", g * 1.02)):
        assert abs((wrong * x).sum() - want) > limit, name


@pytest.mark.gpu
@pytest.mark.parametrize("args", CASES)
def test_the_inverse_is_the_adjoint(F, args):
    T, H, d, rot, layout, dtype, kw = args
    x, w, cs = case(*args)
    dev = lambda a: torch.from_numpy(a).to(DT[dtype]).cuda()  # noqa: E731
    pos = torch.arange(3, T + 3, dtype=torch.int32, device="cuda")
    table = torch.from_numpy(cs).cuda()
    y = F.rope(dev(x), table, pos, layout=layout).double().cpu().numpy()
    g = F.rope(dev(w), table, pos, layout=layout, inverse=True).double().cpu().numpy()
    assert abs((g * x).sum() - (w * y).sum()) <= bound(x, w, y, g, cs[3:], layout, dtype)
