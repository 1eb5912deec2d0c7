"""Refusals of packed attention and of the 4-bit cache's calls on the host (no GPU: every call fails before anything is enqueued)."""
import ctypes
import os

import pytest
import torch

from paper_2609_29812_amd import flashloop as fl

FL_OK, FL_E_NULL, FL_E_SHAPE, FL_E_RANGE, FL_E_UNSUPPORTED, FL_E_WORKSPACE = 0, 1, 2, 3, 4, 5


def P(n):
    return ctypes.c_void_p(0x100000 * n)     # stand-ins, never dereferenced on the host


def at(x):
    return ctypes.c_void_p(x)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fl.LIB_PATH):
        from paper_2609_29812_amd import build
        build.build(verbose=False)
    return fl.load()


def _packed(lib, q=P(1), qs=512, k=P(2), ks=256, v=P(3), vs=256, dtype=0, cu_q=P(4), cu_k=P(5), B=2, Tq=4, Tk=6, Hq=4, Hkv=2, d=128,
            table=None, n_pos=0, rot=0, layout=0, scale=0.1, window=0, n_sink=0, max_k=0, o=P(6), os=512, lse=None, ws=P(7),
            ws_bytes=1 << 40):
    return lib.fl_packed_attn(q, qs, k, ks, v, vs, dtype, cu_q, cu_k, B, Tq, Tk, Hq, Hkv, d, table, n_pos, rot, layout, scale, window,
                              n_sink, max_k, o, os, lse, ws, ctypes.c_size_t(ws_bytes), None)


def test_packed_attn_refusals(lib):
    for name in ("q", "k", "v", "cu_q", "cu_k", "o"):
        assert _packed(lib, **{name: None}) == FL_E_NULL, name
    assert _packed(lib, dtype=2) == FL_E_UNSUPPORTED and _packed(lib, dtype=-1) == FL_E_UNSUPPORTED
    assert _packed(lib, d=96) == FL_E_SHAPE and _packed(lib, d=256) == FL_E_SHAPE
    assert _packed(lib, B=0) == FL_E_SHAPE and _packed(lib, B=65537) == FL_E_SHAPE
    assert _packed(lib, Tq=-1) == FL_E_SHAPE and _packed(lib, Tk=-1) == FL_E_SHAPE
    assert _packed(lib, Hq=5) == FL_E_SHAPE and _packed(lib, Hq=1) == FL_E_SHAPE and _packed(lib, Hkv=0) == FL_E_SHAPE
    assert _packed(lib, Tq=1 << 30) == FL_E_SHAPE                                       # Tq * Hq
    for name, bad in (("qs", 504), ("ks", 248), ("vs", 252), ("os", 516), ("qs", (1 << 24) + 8), ("ks", (1 << 24) + 8)):
        assert _packed(lib, **{name: bad}) == FL_E_SHAPE, (name, bad)
    for name in ("q", "k", "v", "o"):
        assert _packed(lib, **{name: at(0x1000008)}) == FL_E_SHAPE, name
    assert _packed(lib, o=P(1)) == FL_E_SHAPE and _packed(lib, o=P(2)) == FL_E_SHAPE      # over q, over k
    assert _packed(lib, o=at(0x300000 + 5 * 512)) == FL_E_SHAPE                           # over the last row of v
    assert _packed(lib, o=at(0x300000 - 4 * 1024 + 16)) == FL_E_SHAPE
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert _packed(lib, scale=scale) == FL_E_RANGE
    assert _packed(lib, window=-1) == FL_E_RANGE and _packed(lib, n_sink=-1) == FL_E_RANGE and _packed(lib, max_k=-1) == FL_E_RANGE
    assert _packed(lib, table=P(9), rot=24, n_pos=9) == FL_E_SHAPE and _packed(lib, table=P(9), rot=64) == FL_E_RANGE
    assert _packed(lib, table=P(9), rot=64, n_pos=9, layout=2) == FL_E_UNSUPPORTED
    assert _packed(lib, Tq=0, q=None, o=None) == FL_OK                                    # nothing to do
    assert b"fl_packed_attn" in lib.fl_last_error()


def test_packed_attn_interleaved_rows(lib):
    """An output between the rows of a fused projection overlaps nothing: refused for another reason (no workspace) or not at all."""
    need = lib.fl_packed_attn_ws(1, 1 << 20, 1 << 20, 4, 2, 128, 0, 0, 0)
    base, row = 0x10000000, 512 + 256 + 256 + 512
    args = dict(q=at(base), k=at(base + 1024), v=at(base + 1536), o=at(base + 2048), qs=row, ks=row, vs=row, os=row)
    assert _packed(lib, **dict(args, o=at(base + 2048 - 16))) == FL_E_SHAPE               # into v
    assert _packed(lib, **dict(args, o=at(base + 2048 + 16))) == FL_E_SHAPE               # into the next row of q
    assert need >= 0


def _append(lib, k=P(1), ks=256, v=P(2), vs=256, dtype=0, cu=P(3), lens=P(4), B=2, T=4, Hkv=2, d=128, table=P(5), n_pos=1024,
            rot=64, layout=0, bt=P(6), max_pages=16, num_pages=40, page=64, fmt=0, kc=P(7), vc=P(8), km=P(10), vm=P(11), kr=None,
            krs=0, vr=None, vrs=0):
    return lib.fl_paged4_append(k, ks, v, vs, dtype, cu, lens, B, T, Hkv, d, table, n_pos, rot, layout, bt, max_pages, num_pages,
                                page, fmt, kc, vc, km, vm, kr, krs, vr, vrs, None)


def _read(lib, dtype=0, cu=P(3), lens=P(4), B=2, T=4, Hkv=2, d=128, bt=P(6), max_pages=16, num_pages=40, page=64, fmt=0, kc=P(7),
          vc=P(8), km=P(10), vm=P(11), ko=P(12), kos=256, vo=P(13), vos=256):
    return lib.fl_paged4_read(cu, lens, B, T, Hkv, d, bt, max_pages, num_pages, page, fmt, kc, vc, km, vm, dtype, ko, kos, vo, vos, None)


def _attn(lib, q=P(1), qs=512, dtype=0, cu=P(3), lens=P(4), B=2, T=4, Hq=4, Hkv=2, d=128, table=P(5), n_pos=1024, rot=64,
          layout=0, bt=P(6), max_pages=16, num_pages=40, page=64, fmt=0, kc=P(7), vc=P(8), km=P(10), vm=P(11), scale=0.1,
          window=0, n_sink=0, max_q=2, max_len=0, o=P(12), os=512, lse=None, ws=P(13), ws_bytes=1 << 40):
    return lib.fl_paged4_attn(q, qs, dtype, cu, lens, B, T, Hq, Hkv, d, table, n_pos, rot, layout, bt, max_pages, num_pages, page,
                              fmt, kc, vc, km, vm, scale, window, n_sink, max_q, max_len, o, os, lse, ws,
                              ctypes.c_size_t(ws_bytes), None)


@pytest.mark.parametrize("call", [_append, _read, _attn])
def test_refusals_of_a_4_bit_batch(lib, call):
    for name in ("cu", "lens", "bt", "kc", "vc", "km", "vm"):
        assert call(lib, **{name: None}) == FL_E_NULL, name
    assert call(lib, dtype=2) == FL_E_UNSUPPORTED and call(lib, fmt=2) == FL_E_UNSUPPORTED and call(lib, fmt=-1) == FL_E_UNSUPPORTED
    assert call(lib, d=96) == FL_E_SHAPE and call(lib, d=256) == FL_E_SHAPE
    for page in (0, 8, 24, 48, 256):
        assert call(lib, page=page) == FL_E_SHAPE
    assert call(lib, B=0) == FL_E_SHAPE and call(lib, B=65537) == FL_E_SHAPE and call(lib, T=-1) == FL_E_SHAPE
    assert call(lib, Hkv=0) == FL_E_SHAPE
    assert call(lib, max_pages=0) == FL_E_SHAPE and call(lib, max_pages=1 << 26) == FL_E_SHAPE
    assert call(lib, num_pages=0) == FL_E_SHAPE
    assert call(lib, vc=P(7)) == FL_E_SHAPE and call(lib, vm=P(10)) == FL_E_SHAPE         # keys and values in one cache
    for name in ("kc", "vc", "km", "vm"):
        assert call(lib, **{name: at(0x2000004)}) == FL_E_SHAPE, name
    if call is not _read:
        assert call(lib, layout=3) == FL_E_UNSUPPORTED
        assert call(lib, rot=144) == FL_E_SHAPE and call(lib, rot=24) == FL_E_SHAPE
        assert call(lib, n_pos=1023) == FL_E_RANGE                                        # 16 pages of 64
    assert call(lib, T=0) == FL_OK                                                        # nothing to do


def test_append_refusals(lib):
    assert _append(lib, k=None) == FL_E_NULL and _append(lib, v=None) == FL_E_NULL
    assert _append(lib, ks=248) == FL_E_SHAPE and _append(lib, vs=257) == FL_E_SHAPE
    assert _append(lib, k=at(0x100002)) == FL_E_SHAPE
    assert _append(lib, kr=P(20), krs=248) == FL_E_SHAPE and _append(lib, vr=at(0x2000008), vrs=256) == FL_E_SHAPE
    assert _append(lib, kr=P(2), krs=256) == FL_E_SHAPE                                   # the keys' rows over v
    assert _append(lib, vr=P(1), vrs=256) == FL_E_SHAPE                                   # the values' rows over k
    assert _append(lib, kr=P(1), krs=264) == FL_E_SHAPE                                   # in place with another stride
    assert _append(lib, kr=at(0x100000 + 16), krs=256) == FL_E_SHAPE
    assert _append(lib, kr=P(20), krs=256, vr=P(20), vrs=256) == FL_E_SHAPE
    assert b"fl_paged4_append" in lib.fl_last_error()


def test_read_refusals(lib):
    assert _read(lib, ko=None, vo=None) == FL_E_NULL
    assert _read(lib, ko=P(12), vo=P(12)) == FL_E_SHAPE
    assert _read(lib, kos=248) == FL_E_SHAPE and _read(lib, vo=at(0x2000008)) == FL_E_SHAPE
    assert b"fl_paged4_read" in lib.fl_last_error()


def test_attn_refusals(lib):
    assert _attn(lib, q=None) == FL_E_NULL and _attn(lib, o=None) == FL_E_NULL
    assert _attn(lib, Hq=5) == FL_E_SHAPE and _attn(lib, Hq=1) == FL_E_SHAPE
    assert _attn(lib, qs=504) == FL_E_SHAPE and _attn(lib, os=520 + 4) == FL_E_SHAPE
    assert _attn(lib, o=P(1)) == FL_E_SHAPE                                               # o over q
    assert _attn(lib, o=at(0x100000 + 1024)) == FL_E_SHAPE
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert _attn(lib, scale=scale) == FL_E_RANGE
    assert _attn(lib, window=-1) == FL_E_RANGE and _attn(lib, n_sink=-1) == FL_E_RANGE
    assert _attn(lib, max_q=-1) == FL_E_RANGE and _attn(lib, max_len=-1) == FL_E_RANGE
    assert b"fl_paged4_attn" in lib.fl_last_error()


def test_workspaces(lib):
    """None where the work is not cut; else what 512 workgroups leave in two row tiles each, or a place for every part of a row, however
    long the contexts are.  Calls with less, or with an address that is no multiple of 16, are refused."""
    most = 65536 * 2 * 130 * 4
    for n in (1, 300, 4096, 16384):                                                       # whole prompts of 16 heads
        assert lib.fl_packed_attn_ws(1, n, n, 16, 16, 128, 0, 0, 0) == 0
    for n in (8192, 1 << 20, 1 << 30):
        assert 0 < lib.fl_packed_attn_ws(1, 512, n, 16, 16, 128, 0, 0, 0) <= most + 4 * 1024
        assert 0 < lib.fl_paged4_attn_ws(1, 512, 16, 16, 128, 64, n // 64, 0, 0, 512, n) <= most + 4 * 1024
        assert 0 < lib.fl_paged4_attn_ws(8, 8, 16, 16, 128, 64, n // 64, 0, 0, 1, n) <= 2 * 768 * 16 * 130 * 4
    assert lib.fl_paged4_attn_ws(1, 512, 16, 16, 128, 64, 128, 300, 4, 512, 8192) == 0    # a short window
    assert lib.fl_paged4_attn_ws(1, 1, 16, 16, 128, 64, 128, 0, 0, 1, 64) == 0
    call = dict(B=1, Tq=512, Tk=8192, Hq=16, Hkv=16, q=at(1 << 30), k=at(2 << 30), v=at(3 << 30), o=at(4 << 30), qs=2048, ks=2048, vs=2048,
                os=2048, max_k=8192)
    need = lib.fl_packed_attn_ws(1, 512, 8192, 16, 16, 128, 0, 0, 8192)
    assert _packed(lib, **call, ws=None) == FL_E_WORKSPACE and _packed(lib, **call, ws_bytes=need - 1) == FL_E_WORKSPACE
    assert _packed(lib, **call, ws=at(0x1000008)) == FL_E_SHAPE
    for T, max_q in ((512, 512), (1, 1)):
        call = dict(B=1, T=T, Hq=16, Hkv=16, q=at(1 << 30), o=at(4 << 30), qs=2048, os=2048, table=None, max_pages=128, max_q=max_q)
        need = lib.fl_paged4_attn_ws(1, T, 16, 16, 128, 64, 128, 0, 0, max_q, 0)
        assert need > 0
        assert _attn(lib, **call, ws=None) == FL_E_WORKSPACE and _attn(lib, **call, ws_bytes=need - 1) == FL_E_WORKSPACE
        assert _attn(lib, **call, ws=at(0x1000008)) == FL_E_SHAPE


def test_binding_refuses_tensors_of_another_place():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: fl.packed_attn(x, x, x, None), lambda: fl.paged4_append(x, x, None, None, None, None, None, None, None),
                 lambda: fl.paged4_read(None, None, None, x, None, None, None, 4),
                 lambda: fl.paged4_attn(x, None, None, None, None, None, None, None)):
        with pytest.raises(fl.FlashLoopError, match="device"):
            call()
    with pytest.raises(fl.FlashLoopError, match="fmt must be one of"):
        fl.paged4_cache(4, 1, 16, 64, fmt="int8", device="cpu")


class Fake(torch.Tensor):                                          # a CPU tensor that says it is on the current device
    is_cuda = True
    def get_device(self): return 0


def fake(*shape, dtype):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Fake)


@pytest.fixture
def here(lib, monkeypatch):
    monkeypatch.setattr(fl, "_current", lambda: 0)
    monkeypatch.setattr(fl, "_stream", lambda: 0)


def _cache(fmt, pages=4, H=2, page=16, d=64):
    meta = ((pages, H, page, d // 32, 2), torch.float16) if fmt == "int4" else ((pages, H, page, d // 32), torch.uint8)
    return [fake(pages, H, page, d // 2, dtype=torch.uint8) for _ in range(2)] + [fake(*meta[0], dtype=meta[1]) for _ in range(2)]


def test_shapes_of_a_cache():
    for fmt in ("int4", "e2m1"):
        got = fl.paged4_cache(4, 2, 16, 64, fmt, device="cpu")
        assert [(t.shape, t.dtype) for t in got] == [(t.shape, t.dtype) for t in _cache(fmt)]


@pytest.mark.parametrize("fmt", ["int4", "e2m1"])
def test_binding_checks_caches_and_batches(here, fmt):
    q, x = fake(4, 4, 64, dtype=torch.bfloat16), fake(4, 2, 64, dtype=torch.bfloat16)
    cu, lens, tab = (fake(*s, dtype=torch.int32) for s in ((3,), (2,), (2, 8)))
    good = _cache(fmt)
    other = _cache("e2m1" if fmt == "int4" else "int4")

    def calls(cu, lens, tab, cache):
        return (lambda: fl.paged4_attn(q, cu, lens, tab, *cache), lambda: fl.paged4_append(x, x, cu, lens, tab, *cache),
                lambda: fl.paged4_read(cu, lens, tab, *cache, 4))
    bad = [(cu.long(), lens, tab, good, "int32"), (cu, fake(3, dtype=torch.int32), tab, good, "lens"),
           (fake(4, dtype=torch.int32), lens, tab, good, "cu"), (cu, lens, tab[0], good, "block_table"),
           (cu, lens, tab, [good[0], good[1], good[2], other[3]], "v_meta"), (cu, lens, tab, [good[0], good[1][:3], *good[2:]], "v_cache"),
           (cu, lens, tab, [*good[:2], good[2][:, :1], good[3]], "k_meta"), (cu, lens, tab, [good[0].to(torch.int8).as_subclass(Fake), *good[1:]], "k_cache"),
           (cu, lens, tab, [*good[:2], good[2].float().as_subclass(Fake), good[3]], "float16 .int4. or uint8"),
           (cu, lens, tab[:0], good, "at least one sequence")]
    for *args, what in bad:
        for call in calls(*args):
            with pytest.raises(fl.FlashLoopError, match=what):
                call()
    wide = _cache(fmt, d=128)
    for call in calls(cu, lens, tab, wide)[:2]:
        with pytest.raises(fl.FlashLoopError):
            call()


def test_counts_beyond_an_int(here):
    """Sizes, windows and hints that a C int does not hold are refused, and not passed modulo 2^32."""
    q, k = fake(4, 4, 64, dtype=torch.bfloat16), fake(4, 2, 64, dtype=torch.bfloat16)
    cu, lens, tab = (fake(*s, dtype=torch.int32) for s in ((3,), (2,), (2, 8)))
    cache = _cache("int4")
    for n in (2 ** 32 + 5, 2 ** 31, -1):
        for name in ("window", "n_sink", "max_q", "max_len"):
            with pytest.raises(fl.FlashLoopError, match=name):
                fl.paged4_attn(q, cu, lens, tab, *cache, **{name: n})
            with pytest.raises(fl.FlashLoopError, match=name):
                fl.paged4_attn_ws(q, tab, cache[0], **{name: n})
        for name in ("window", "n_sink", "max_k"):
            with pytest.raises(fl.FlashLoopError, match=name):
                fl.packed_attn(q, k, k, cu, **{name: n})
            with pytest.raises(fl.FlashLoopError, match=name):
                fl.packed_attn_ws(q, k, 2, **{name: n})
        with pytest.raises(fl.FlashLoopError, match="T must be in"):
            fl.paged4_read(cu, lens, tab, *cache, n)


def test_packed_binding_checks(here):
    q, k = fake(4, 4, 64, dtype=torch.bfloat16), fake(6, 2, 64, dtype=torch.bfloat16)
    cu = fake(3, dtype=torch.int32)
    for args, what in (((q, k.half().as_subclass(Fake), k, cu), "k must be"), ((q, k, k[:5], cu), "v must have shape"),
                       ((q, fake(6, 2, 128, dtype=torch.bfloat16), k, cu), "v must have shape"),
                       ((q, fake(6, 2, 128, dtype=torch.bfloat16), fake(6, 2, 128, dtype=torch.bfloat16), cu), "heads of 64"),
                       ((q, k, k, cu.long()), "int32"), ((q, k, k, cu[:1]), "at least one"), ((q, k, k, cu, cu[:2]), "cu_k")):
        with pytest.raises(fl.FlashLoopError, match=what):
            fl.packed_attn(*args)
