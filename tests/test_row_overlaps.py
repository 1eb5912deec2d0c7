"""Which rows of different numbers and widths overlap, by what fl_packed_attn answers on the host: a call that needs a workspace and has
none is refused for that (FL_E_WORKSPACE) once its tensors have passed, and for its tensors (FL_E_SHAPE) otherwise."""
import ctypes
import os
import random

import numpy as np
import pytest

from paper_2609_29812_amd import flashloop as fl

FL_E_SHAPE, FL_E_WORKSPACE = 2, 5
TQ, TK, HQ, HKV, D = 512, 8192, 4, 2, 128
WQ, WK = 2 * HQ * D, 2 * HKV * D                       # bytes of a row


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fl.LIB_PATH):
        from paper_2609_29812_amd import build
        build.build(verbose=False)
    return fl.load()


def call(lib, q, qs, k, ks, v, vs, o, os_):
    """Addresses and strides in bytes."""
    P = ctypes.c_void_p
    return lib.fl_packed_attn(P(q), qs // 2, P(k), ks // 2, P(v), vs // 2, 0, P(1 << 20), P(2 << 20), 1, TQ, TK, HQ, HKV, D, None, 0, 0, 0,
                              0.1, 0, 0, TK, P(o), os_ // 2, None, None, ctypes.c_size_t(0), None)


def test_the_call_needs_a_workspace(lib):
    assert lib.fl_packed_attn_ws(1, TQ, TK, HQ, HKV, D, 0, 0, TK) > 0


@pytest.mark.parametrize("order", ["okv", "kov", "kvo"])
def test_an_output_between_the_rows_of_a_projection(lib, order):
    """In front of the keys, between them and the values, behind both: 16 bytes to either side it overlaps one of them."""
    base, row, far = 1 << 30, WQ + 2 * WK, 1 << 36
    at, places = base, {}
    for name in order:
        places[name] = at
        at += WQ if name == "o" else WK
    k, v, o = places["k"], places["v"], places["o"]
    for rows in (0, 3, -3, TK - TQ, -TQ + 1, TK, -TQ):                # begun that many rows on
        assert call(lib, far, WQ, k, row, v, row, o + rows * row, row) == FL_E_WORKSPACE, rows
    for off in (-16, 16, WK, -WK, row // 2):
        assert call(lib, far, WQ, k, row, v, row, o + off, row) == FL_E_SHAPE, off
    assert call(lib, far, WQ, k, row, v, row, o, row + 16) == FL_E_SHAPE                # other strides: its rows drift into them


def test_the_four_of_a_projection(lib):
    base, row = 1 << 30, 2 * WQ + 2 * WK
    assert call(lib, base, row, base + WQ, row, base + WQ + WK, row, base + WQ + 2 * WK, row) == FL_E_WORKSPACE
    assert call(lib, base, row, base + WQ, row, base + WQ + WK, row, base + WQ + 2 * WK + 16, row) == FL_E_SHAPE      # into the next q
    assert call(lib, base, row, base + WQ, row, base + WQ + WK, row, base, row) == FL_E_SHAPE


def units(x, stride, n, width):
    return (x // 16 + np.arange(n)[:, None] * (stride // 16) + np.arange(width // 16)).reshape(-1)


@pytest.mark.parametrize("seed", range(60))
def test_what_is_accepted_overlaps_nothing(lib, seed):
    """And with one stride what overlaps nothing is accepted."""
    rng = random.Random(seed)
    row = WQ + 2 * WK + 16 * rng.choice([0, 1, 40])
    stride = row if seed % 3 else row + 16 * rng.randrange(1, 9)
    k, far = 1 << 30, 1 << 36
    o = k + rng.choice([0, row * rng.randrange(-TQ - 2, TK + 2)]) + 16 * rng.randrange(-row // 16, row // 16)
    rc = call(lib, far, WQ, k, row, far + (1 << 34), row, o, stride)
    both = np.intersect1d(units(k, row, TK, WK), units(o, stride, TQ, WQ)).size > 0
    assert rc in (FL_E_SHAPE, FL_E_WORKSPACE)
    if both:
        assert rc == FL_E_SHAPE
    elif stride == row:
        assert rc == FL_E_WORKSPACE
