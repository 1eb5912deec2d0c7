"""Refusals of the rotary and paged calls on the host (no GPU: every call fails before anything is enqueued)."""
import ctypes
import os

import pytest
import torch

from paper_2609_29812_amd import flashloop as fl

FL_OK, FL_E_NULL, FL_E_SHAPE, FL_E_RANGE, FL_E_UNSUPPORTED, FL_E_WORKSPACE = 0, 1, 2, 3, 4, 5


def P(n):
    return ctypes.c_void_p(0x100000 * n)     # stand-ins, never dereferenced on the host


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fl.LIB_PATH):
        from paper_2609_29812_amd import build
        build.build(verbose=False)
    return fl.load()


def test_rope_table_refusals(lib):
    def call(n_pos=8, rot=64, base=1e4, scaling=0, factor=1.0, orig=0.0, low=1.0, high=32.0, table=P(1)):
        return lib.fl_rope_table(n_pos, rot, base, scaling, factor, orig, low, high, table, None)
    assert call(table=None) == FL_E_NULL
    assert call(table=ctypes.c_void_p(0x1004)) == FL_E_SHAPE
    assert call(n_pos=0) == FL_E_SHAPE
    assert call(rot=24) == FL_E_SHAPE and call(rot=0) == FL_E_SHAPE and call(rot=1040) == FL_E_SHAPE
    assert call(scaling=4) == FL_E_UNSUPPORTED and call(scaling=-1) == FL_E_UNSUPPORTED
    assert call(base=1.0) == FL_E_RANGE and call(base=float("nan")) == FL_E_RANGE
    assert call(scaling=1, factor=0.5) == FL_E_RANGE and call(scaling=2, factor=float("inf")) == FL_E_RANGE
    assert call(scaling=3, factor=2.0) == FL_E_RANGE                         # no original length
    assert call(scaling=3, factor=2.0, orig=4096, low=32.0, high=1.0) == FL_E_RANGE
    assert b"fl_rope_table" in lib.fl_last_error()


def test_rope_refusals(lib):
    def call(x=P(1), xs=256, pos=P(2), table=P(3), n_pos=64, rot=64, layout=0, dtype=0, T=4, H=2, d=128, y=P(9), ys=256):
        return lib.fl_rope(x, xs, pos, table, n_pos, rot, layout, 0, dtype, T, H, d, y, ys, None)
    assert call(x=None) == FL_E_NULL and call(y=None) == FL_E_NULL and call(table=None) == FL_E_NULL
    assert call(dtype=2) == FL_E_UNSUPPORTED and call(layout=2) == FL_E_UNSUPPORTED
    assert call(rot=144) == FL_E_SHAPE and call(rot=8) == FL_E_SHAPE
    assert call(d=100) == FL_E_SHAPE and call(d=2048, xs=4096, ys=4096) == FL_E_SHAPE
    assert call(xs=248) == FL_E_SHAPE and call(ys=260) == FL_E_SHAPE
    assert call(x=ctypes.c_void_p(0x100008)) == FL_E_SHAPE
    assert call(T=-1) == FL_E_SHAPE and call(H=0) == FL_E_SHAPE
    assert call(pos=None, T=65) == FL_E_RANGE                                # more rows than the table has positions
    assert call(y=ctypes.c_void_p(0x100000 + 512)) == FL_E_SHAPE             # the second row of x
    assert call(xs=512, ys=512, y=ctypes.c_void_p(0x100000 + 256)) == FL_E_SHAPE     # half of its own row
    assert call(y=P(1), ys=512) == FL_E_SHAPE                                # in place with another stride
    assert call(T=0, x=None, y=None) == FL_OK
    assert b"fl_rope" in lib.fl_last_error()


def _append(lib, k=P(1), ks=256, v=P(2), vs=256, dtype=0, cu=P(3), lens=P(4), B=2, T=4, Hkv=2, d=128, table=P(5), n_pos=1024,
            rot=64, layout=0, bt=P(6), max_pages=16, num_pages=40, page=64, fmt=0, kc=P(7), vc=P(8), ksc=P(10), vsc=P(11)):
    return lib.fl_paged_append(k, ks, v, vs, dtype, cu, lens, B, T, Hkv, d, table, n_pos, rot, layout, bt, max_pages, num_pages,
                               page, fmt, kc, vc, ksc, vsc, None)


def _attn(lib, q=P(1), qs=512, dtype=0, cu=P(3), lens=P(4), B=2, T=4, Hq=4, Hkv=2, d=128, table=P(5), n_pos=1024, rot=64,
          layout=0, bt=P(6), max_pages=16, num_pages=40, page=64, fmt=0, kc=P(7), vc=P(8), ksc=P(10), vsc=P(11), scale=0.1,
          window=0, n_sink=0, max_q=2, max_len=0, o=P(12), os=512, lse=None, ws=P(13), ws_bytes=1 << 40):
    return lib.fl_paged_attn(q, qs, dtype, cu, lens, B, T, Hq, Hkv, d, table, n_pos, rot, layout, bt, max_pages, num_pages, page,
                             fmt, kc, vc, ksc, vsc, scale, window, n_sink, max_q, max_len, o, os, lse, ws,
                             ctypes.c_size_t(ws_bytes), None)


@pytest.mark.parametrize("call", [_append, _attn])
def test_refusals_of_a_paged_batch(lib, call):
    for name in ("cu", "lens", "bt", "kc", "vc", "ksc", "vsc"):
        assert call(lib, **{name: None}) == FL_E_NULL, name
    assert call(lib, dtype=2) == FL_E_UNSUPPORTED and call(lib, fmt=2) == FL_E_UNSUPPORTED
    assert call(lib, layout=3) == FL_E_UNSUPPORTED
    assert call(lib, d=96) == FL_E_SHAPE and call(lib, d=256) == FL_E_SHAPE
    for page in (0, 8, 24, 48, 256):
        assert call(lib, page=page) == FL_E_SHAPE
    assert call(lib, B=0) == FL_E_SHAPE and call(lib, B=65537) == FL_E_SHAPE and call(lib, T=-1) == FL_E_SHAPE
    assert call(lib, Hkv=0) == FL_E_SHAPE
    assert call(lib, max_pages=0) == FL_E_SHAPE and call(lib, max_pages=1 << 26) == FL_E_SHAPE
    assert call(lib, num_pages=0) == FL_E_SHAPE
    assert call(lib, vc=P(7)) == FL_E_SHAPE and call(lib, vsc=P(10)) == FL_E_SHAPE       # keys and values in one cache
    assert call(lib, kc=ctypes.c_void_p(0x700004)) == FL_E_SHAPE
    assert call(lib, rot=144) == FL_E_SHAPE and call(lib, rot=24) == FL_E_SHAPE
    assert call(lib, n_pos=1023) == FL_E_RANGE                                           # 16 pages of 64
    assert call(lib, T=0) == FL_OK                                                       # nothing to do


def test_append_refusals(lib):
    assert _append(lib, k=None) == FL_E_NULL and _append(lib, v=None) == FL_E_NULL
    assert _append(lib, ks=248) == FL_E_SHAPE and _append(lib, vs=257) == FL_E_SHAPE
    assert _append(lib, k=ctypes.c_void_p(0x100002)) == FL_E_SHAPE
    assert b"fl_paged_append" in lib.fl_last_error()


def test_attn_refusals(lib):
    assert _attn(lib, q=None) == FL_E_NULL and _attn(lib, o=None) == FL_E_NULL
    assert _attn(lib, Hq=5) == FL_E_SHAPE and _attn(lib, Hq=1) == FL_E_SHAPE
    assert _attn(lib, qs=504) == FL_E_SHAPE and _attn(lib, os=520 + 4) == FL_E_SHAPE
    assert _attn(lib, o=P(1)) == FL_E_SHAPE                                              # o over q
    assert _attn(lib, o=ctypes.c_void_p(0x100000 + 1024)) == FL_E_SHAPE
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert _attn(lib, scale=scale) == FL_E_RANGE
    assert _attn(lib, window=-1) == FL_E_RANGE and _attn(lib, n_sink=-1) == FL_E_RANGE
    assert _attn(lib, max_q=-1) == FL_E_RANGE and _attn(lib, max_len=-1) == FL_E_RANGE
    assert b"fl_paged_attn" in lib.fl_last_error()


def test_workspace_of_few_rows(lib):
    """It holds a place for each row of the work items, which the chip's size bounds: not one for every part of every row, nor
    more of them for longer contexts."""
    def ws(B, T, Hq, Hkv, d=128, page=64, max_pages=2048, max_q=1, max_len=0):
        return lib.fl_paged_attn_ws(B, T, Hq, Hkv, d, page, max_pages, 0, 0, max_q, max_len)
    for B, T, Hq, Hkv, max_q in ((48, 48, 64, 8, 1), (32, 32, 32, 8, 1), (48, 192, 32, 8, 4), (95, 95, 128, 8, 1), (1, 1, 8, 1, 1)):
        rows = 16 if max_q * Hq // Hkv <= 16 else 32
        items = (T * (Hq // Hkv) // rows + B + 768 // Hkv + 1) * Hkv
        need = ws(B, T, Hq, Hkv, max_q=max_q)
        assert 0 < need <= items * rows * (128 + 4) * 4
        assert ws(B, T, Hq, Hkv, max_q=max_q, max_pages=1 << 17) == need
    assert ws(1, 1, 16, 16, max_len=300) == 0                    # one part: nothing to join


def test_binding_refuses_tensors_of_another_place(monkeypatch):
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(fl.FlashLoopError, match="device"):
        fl.rope(x, torch.zeros(4, 8, 2))
    with pytest.raises(fl.FlashLoopError, match="device"):
        fl.paged_append(x, x, None, None, None, None, None, None, None)
    with pytest.raises(fl.FlashLoopError, match="device"):
        fl.paged_attn(x, None, None, None, None, None, None, None)
    # a tensor of another GPU than the current one, or than the call's first tensor
    class Elsewhere:
        is_cuda, dtype, device, shape = True, torch.float32, torch.device("cuda", 1), (4,)
        def get_device(self): return 1
        def is_contiguous(self): return True
    monkeypatch.setattr(fl, "_current", lambda: 0)
    with pytest.raises(fl.FlashLoopError, match="current device"):
        fl._here(Elsewhere(), "x")
    monkeypatch.setattr(fl, "_current", lambda: 1)
    assert fl._here(Elsewhere(), "x") == 1
    with pytest.raises(fl.FlashLoopError, match="other tensors"):
        fl._on(Elsewhere(), 0, torch.float32, "table", (4,))
    fl._on(Elsewhere(), 1, torch.float32, "table", (4,))
    with pytest.raises(fl.FlashLoopError, match="scaling must be one of"):
        fl.rope_table(4, 64, scaling="other")
    with pytest.raises(fl.FlashLoopError, match="int8 or float8"):
        fl.paged_cache(4, 1, 16, 64, dtype=torch.uint8, device="cpu")


def test_counts_beyond_an_int(lib, monkeypatch):
    """Sizes, windows and hints that a C int does not hold are refused, and not passed modulo 2^32."""
    class Fake(torch.Tensor):                                     # a CPU tensor that says it is on the current device
        is_cuda = True
        def get_device(self): return 0
    monkeypatch.setattr(fl, "_current", lambda: 0)
    monkeypatch.setattr(fl, "_stream", lambda: 0)
    def fake(*shape, dtype): return torch.zeros(*shape, dtype=dtype).as_subclass(Fake)
    q = fake(4, 4, 64, dtype=torch.bfloat16)
    cu, lens, tab = (fake(*s, dtype=torch.int32) for s in ((3,), (2,), (2, 8)))
    cache = [fake(4, 2, 16, 64, dtype=torch.int8) for _ in range(2)] + [fake(4, 2, dtype=torch.float32) for _ in range(2)]
    for name in ("window", "n_sink", "max_q", "max_len"):
        for n in (2 ** 32 + 5, 2 ** 31, -1):
            with pytest.raises(fl.FlashLoopError, match=name):
                fl.paged_attn(q, cu, lens, tab, *cache, **{name: n})
            with pytest.raises(fl.FlashLoopError, match=name):
                fl.paged_attn_ws(q, tab, cache[0], **{name: n})
    for kw in (dict(n_pos=2 ** 32 + 8, rot=64), dict(n_pos=8, rot=2 ** 32 + 64), dict(n_pos=-1, rot=64)):
        with pytest.raises(fl.FlashLoopError, match="must be in"):
            fl.rope_table(**kw, device="meta")
    # views of one row, as many as a C int does not hold: the strides are refused only afterwards
    many = torch.zeros(1, 1, 64, dtype=torch.bfloat16).expand(2 ** 32 + 5, 1, 64).as_subclass(Fake)
    with pytest.raises(fl.FlashLoopError, match="T must be in"):
        fl.rope(many, fake(8, 8, 2, dtype=torch.float32))
    with pytest.raises(fl.FlashLoopError, match="T must be in"):
        fl.paged_append(many, many, cu, lens, tab, *(fake(4, 1, 16, 64, dtype=torch.int8) for _ in range(2)), *cache[2:])


def test_rows_of_the_binding():
    cpu = torch.zeros(1).get_device()
    x = torch.zeros(6, 3 * 128, dtype=torch.float16)[:, 128:256].view(6, 2, 64)
    assert fl._rows(x, cpu, torch.float16, "x") == 384
    assert fl._rows(x[:1], cpu, torch.float16, "x") == 128           # one row has no stride
    for bad, what in ((x.transpose(0, 1), "dense"), (x[:, :, ::2], "dense"), (x[:, 0], "shape"), (x.float(), "bfloat16"),
                      (x.view(6, 2, 64)[:, ::2], None)):
        if what is None:
            assert fl._rows(bad, cpu, torch.float16, "x") == 384     # a single head of each row
        else:
            with pytest.raises(fl.FlashLoopError, match=what):
                fl._rows(bad, cpu, bad.dtype, "x")
