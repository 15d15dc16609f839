"""Refusals of the cache operators' C entry points, checked without a GPU: every one is decided on the host before
anything is queued."""

from __future__ import annotations

import ctypes
import math

import pytest

from paper_2607_21848_amd import _lib

NULL = None
FAKE = ctypes.c_void_p(0x10000)   # never dereferenced: validation fails first, or there is nothing to do
FAR = ctypes.c_void_p(0x900000000)
ODD = ctypes.c_void_p(0x10008)    # 8-byte aligned only


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def _rotary(L, **kw):
    a = dict(q=FAKE, q_row=1536, k=FAKE, k_row=1536, qo=FAR, qo_row=1536, ko=FAR, ko_row=1536, dtype=1, n=10, Hq=12, Hk=12, D=128,
             pos=NULL, t0=0, h=30, w=52, nt=22, ny=21, nx=21, theta=10000.0, inv=0, qs=1.0, ks=1.0)
    a.update(kw)
    return L.rotary_embed(*[a[n] for n in ("q", "q_row", "k", "k_row", "qo", "qo_row", "ko", "ko_row", "dtype", "n", "Hq", "Hk", "D",
                                           "pos", "t0", "h", "w", "nt", "ny", "nx", "theta", "inv", "qs", "ks")], NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=9), 3), (dict(D=4), 3), (dict(D=12), 3), (dict(D=520), 3), (dict(n=-1), 2), (dict(Hq=0), 2), (dict(Hk=0), 2),
    (dict(Hq=65536), 2), (dict(nt=23), 4), (dict(ny=-1), 4), (dict(nt=2**31 - 1, ny=2**31 - 1), 4), (dict(theta=0.0), 4),
    (dict(theta=float("nan")), 4), (dict(inv=2), 4), (dict(h=0), 2), (dict(w=0), 2), (dict(h=1 << 16, w=1 << 16), 2),
    (dict(q_row=1535), 2), (dict(qo_row=1528), 2), (dict(q_row=1540), 2), (dict(k_row=1 << 41), 2), (dict(q=NULL), 1),
    (dict(qo=NULL), 1), (dict(ko=NULL), 1), (dict(q=ODD), 2), (dict(ko=ODD), 2), (dict(pos=ctypes.c_void_p(0x10002)), 2),
    (dict(dtype=3, qs=0.0), 4), (dict(dtype=3, ks=float("inf")), 4), (dict(dtype=3, qo=ctypes.c_void_p(0x10004)), 2),
    (dict(qo=FAKE, qo_row=4608), 2), (dict(dtype=3, qo=FAKE), 2), (dict(n=2**31 - 1, Hq=65535), 2),
])
def test_rotary_rejects(L, kw, status):
    assert _rotary(L, **kw) == status
    assert "rotary_embed" in _lib.last_error()


def test_rotary_nothing_to_do(L):
    assert _rotary(L, n=0, q=NULL, k=NULL, qo=NULL, ko=NULL) == 0
    assert _rotary(L, n=0, nt=0, ny=0, nx=0) == 0


def _weight(L, **kw):
    a = dict(q=FAKE, k=FAKE, lse=FAKE, dtype=1, Lq=100, Lk=4680, H=12, D=128, h=30, w=52, slot=FAKE, uv=FAKE, idx=FAKE, S=2,
             scale=1 / math.sqrt(128), lam=1.0, sigma=2.0, prev=NULL, decay=1.0, out=FAKE, parts=1, ws=NULL, ws_bytes=0)
    a.update(kw)
    return L.attention_key_weight(*[a[n] for n in ("q", "k", "lse", "dtype", "Lq", "Lk", "H", "D", "h", "w", "slot", "uv", "idx", "S",
                                                   "scale", "lam", "sigma", "prev", "decay", "out", "parts", "ws", "ws_bytes")], NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), 3), (dict(D=64), 3), (dict(dtype=2, D=96), 3), (dict(Lq=-1), 2), (dict(Lk=0), 2), (dict(H=0), 2), (dict(h=0), 2),
    (dict(S=-1), 2), (dict(Lk=4681), 2), (dict(Lk=1025 * 1560), 2), (dict(h=300, w=1, Lk=3000), 2), (dict(scale=0.0), 4),
    (dict(scale=float("nan")), 4), (dict(sigma=0.0), 4), (dict(lam=float("inf")), 4), (dict(decay=float("nan")), 4),
    (dict(lam=3e38, sigma=1e-3), 4), (dict(parts=-1), 4), (dict(parts=65), 4), (dict(q=NULL), 1), (dict(k=NULL), 1),
    (dict(lse=NULL), 1), (dict(out=NULL), 1), (dict(slot=NULL), 1), (dict(uv=NULL), 1), (dict(idx=NULL), 1), (dict(q=ODD), 2),
    (dict(k=ODD), 2), (dict(out=ctypes.c_void_p(0x10002)), 2), (dict(uv=ctypes.c_void_p(0x10004)), 2),
    # three parts of 12 x 4680 sums: no workspace, too small, NULL, misaligned
    (dict(parts=3), 2), (dict(parts=3, ws=FAKE, ws_bytes=3 * 12 * 4680 * 4 - 1), 2), (dict(parts=3, ws_bytes=1 << 30), 1),
    (dict(parts=3, ws=ODD, ws_bytes=1 << 30), 2),
])
def test_weight_rejects(L, kw, status):
    assert _weight(L, **kw) == status
    assert "attention_key_weight" in _lib.last_error()


def test_weight_workspace(L):
    n = ctypes.c_size_t(7)
    size = lambda *a: (L.rc_key_weight_workspace_size(*a, ctypes.byref(n)), n.value)  # noqa: E731
    assert size(1, 100, 4680, 12, 128, 30, 52, 2, 3) == (0, 3 * 12 * 4680 * 4)
    assert size(1, 100, 4680, 12, 128, 30, 52, 2, 64) == (0, 4 * 12 * 4680 * 4)  # 100 queries are four tiles
    assert size(1, 0, 4680, 12, 128, 30, 52, 0, 5) == (0, 0)
    assert size(1, 100, 4680, 12, 128, 30, 52, 2, 1) == (0, 0)
    assert size(1, 100, 4681, 12, 128, 30, 52, 2, 1) == (2, 0)
    assert L.rc_key_weight_workspace_size(1, 100, 4680, 12, 128, 30, 52, 2, 1, None) == 1


def _select(L, **kw):
    a = dict(weight=FAKE, sets=4, heads=1, n=100, unit=1, keep=50, first=3, last=6, idx=FAKE, score=NULL, ws=NULL, ws_bytes=0)
    a.update(kw)
    return L.select_kept(*[a[n] for n in ("weight", "sets", "heads", "n", "unit", "keep", "first", "last", "idx", "score", "ws",
                                          "ws_bytes")], NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(sets=-1), 2), (dict(heads=0), 2), (dict(n=-1), 2), (dict(unit=0), 2), (dict(n=(1 << 30) + 1), 2), (dict(sets=(1 << 21) + 1), 2),
    (dict(n=1 << 20, unit=1 << 12), 2), (dict(keep=101), 4), (dict(keep=-1), 4), (dict(keep=8), 4), (dict(first=-1), 4),
    (dict(last=-1), 4), (dict(first=2**31 - 1, last=2**31 - 1), 4), (dict(weight=NULL), 1), (dict(idx=NULL), 1),
    (dict(weight=ctypes.c_void_p(0x10002)), 2),
    # sums of 12 x 10000 weights a set go through the workspace: none, too small, NULL, misaligned
    (dict(heads=12, n=10000), 2), (dict(heads=12, n=10000, ws=FAKE, ws_bytes=4 * 10000 * 8 - 1), 2),
    (dict(heads=12, n=10000, ws_bytes=1 << 20), 1), (dict(n=30000, unit=3, ws=ODD, ws_bytes=1 << 30), 2),
])
def test_select_rejects(L, kw, status):
    assert _select(L, **kw) == status
    assert "select_kept" in _lib.last_error()


def test_select_workspace(L):
    n = ctypes.c_size_t(7)
    size = lambda *a: (L.rc_select_workspace_size(*a, ctypes.byref(n)), n.value)  # noqa: E731
    assert size(96, 1, 37440, 1) == (0, 0)            # the weights are the scores
    assert size(4, 12, 100, 1) == (0, 0)              # few weights a set: summed where they are chosen from
    assert size(4, 12, 10000, 1) == (0, 4 * 10000 * 8)
    assert size(30, 12, 18, 1560) == (0, 30 * 18 * 8)
    assert size(1, 12, 18, 1560) == (0, 12 * 18 * 8)  # every head a part
    assert size(-1, 1, 1, 1) == (2, 0)
    # long sets that leave compute units idle: histograms of 4096 + 64 bins and a range per share, a list per set
    assert size(1, 1, 37440, 1) == (0, 4 * (10 * (4096 + 64 + 2) + 37440))
    assert size(2, 12, 65536, 1) == (0, 2 * (65536 * 8 + 4 * (16 * (4096 + 64 + 2) + 65536)))
    assert size(1, 1, 1 << 30, 1) == (0, 4 * (256 * (4096 + 64 + 2) + (1 << 30)))
    assert L.rc_select_workspace_size(1, 1, 1, 1, None) == 1


def test_select_shares(L):
    """Which long sets are shared out over workgroups, as the workspace shows: from n (1 - 1 / shares) = 31000 units on, where
    there are two shares from 50000 on."""
    n = ctypes.c_size_t(7)

    def size(sets, units):
        assert L.rc_select_workspace_size(sets, 1, units, 1, ctypes.byref(n)) == 0
        return n.value

    for sets, shares, least in ((1, 9, 34875), (32, 8, 35428), (51, 5, 38750), (64, 4, 41333), (85, 3, 46500), (100, 2, 100000), (128, 2, 100000)):
        assert size(sets, least) == 0, (sets, least)
        assert size(sets, least + 1) == 4 * (sets * shares * (4096 + 64 + 2) + sets * (least + 1)), (sets, least + 1)
    assert size(129, 1 << 23) == 0


def test_select_nothing_to_do(L):
    assert _select(L, sets=0, weight=NULL, idx=NULL) == 0
    assert _select(L, keep=0, first=0, last=0, weight=NULL, idx=NULL) == 0
    assert _select(L, n=0, keep=0, first=0, last=0) == 0


def _compact(L, **kw):
    a = dict(sk=FAKE, sv=FAKE, rows=120, sel=FAKE, sel_heads=1, keep=5, unit=10, n=12, dk=FAR, dv=FAR, drows=60, row0=5, sw=NULL,
             swc=0, dw=NULL, dwc=0, layers=2, dtype=1, H=3, D=128, pos=NULL, dpos=0, fpu=1, nt=22, theta=10000.0)
    a.update(kw)
    return L.compact_kv(*[a[n] for n in ("sk", "sv", "rows", "sel", "sel_heads", "keep", "unit", "n", "dk", "dv", "drows", "row0", "sw",
                                         "swc", "dw", "dwc", "layers", "dtype", "H", "D", "pos", "dpos", "fpu", "nt", "theta")], NULL)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), 3), (dict(D=4), 3), (dict(D=100), 3), (dict(D=520), 3), (dict(dtype=3, D=8, nt=0), 3), (dict(dtype=3), 3),
    (dict(keep=-1), 2), (dict(unit=0), 2), (dict(H=0), 2), (dict(layers=-1), 2), (dict(row0=-1), 2), (dict(sel_heads=2), 2),
    (dict(n=13), 2), (dict(row0=11), 2), (dict(keep=6), 2), (dict(nt=65), 4), (dict(nt=-1), 4), (dict(theta=0.0), 4), (dict(fpu=-1), 4),
    (dict(sw=FAKE), 1), (dict(dw=FAR), 1), (dict(sw=FAKE, dw=FAR, swc=119, dwc=60), 2), (dict(sw=FAKE, dw=FAR, swc=120, dwc=54), 2),
    (dict(sk=NULL), 1), (dict(sel=NULL), 1), (dict(dv=NULL), 1), (dict(sk=ODD), 2), (dict(dv=ODD), 2),
    (dict(dk=FAKE), 2), (dict(dv=ctypes.c_void_p(0x10000 + 2 * 120 * 3 * 128 * 2 - 16)), 2),
    (dict(sw=FAKE, dw=ctypes.c_void_p(0x10004), swc=120, dwc=60), 2), (dict(layers=1 << 30, H=60000), 2),
])
def test_compact_rejects(L, kw, status):
    assert _compact(L, **kw) == status
    assert "compact_kv" in _lib.last_error()


# bytes of _compact's arrays: src_k and src_v 184320 each, dst_k and dst_v 92160, sel 40, weights 2 x 3 x 120 and x 60 words
_APART = dict(sv=ctypes.c_void_p(0x100000), dv=ctypes.c_void_p(0x900100000), sel=ctypes.c_void_p(0x200000))
_WEIGHTS = dict(sw=ctypes.c_void_p(0x300000), dw=ctypes.c_void_p(0x900300000), swc=120, dwc=60)


@pytest.mark.parametrize("kw", [
    dict(dv=FAKE), dict(dv=ctypes.c_void_p(0x10000 + 184320 - 16)), dict(sk=ctypes.c_void_p(0x500000), dv=ctypes.c_void_p(0x500000 - 92160 + 16)),  # dst_v in src_k
    dict(dk=ctypes.c_void_p(0x100000 + 184320 - 16)), dict(dk=ctypes.c_void_p(0x100000)),                            # dst_k in src_v
    dict(dv=FAR), dict(dv=ctypes.c_void_p(0x900000000 + 92160 - 16)), dict(dk=ctypes.c_void_p(0x900100000 + 16)),    # dst_k with dst_v
    dict(sel=FAR), dict(sel=ctypes.c_void_p(0x900100000 + 92160 - 4)), dict(sel=ctypes.c_void_p(0x900000000 - 36)),  # over the selection
    dict(pos=ctypes.c_void_p(0x900000000 + 400)), dict(pos=ctypes.c_void_p(0x900100000 - 44)),                       # over the positions
    dict(_WEIGHTS, dw=ctypes.c_void_p(0x10000)), dict(_WEIGHTS, dw=ctypes.c_void_p(0x100000 + 4)),                   # weights over the caches
    dict(_WEIGHTS, dw=ctypes.c_void_p(0x900000000 + 8)), dict(_WEIGHTS, dw=ctypes.c_void_p(0x900100000 - 4)),
    dict(_WEIGHTS, dw=ctypes.c_void_p(0x200000 - 1436)), dict(_WEIGHTS, dw=ctypes.c_void_p(0x300000 + 2876)),
    dict(_WEIGHTS, sw=ctypes.c_void_p(0x900000000 + 92160 - 4)), dict(_WEIGHTS, sw=ctypes.c_void_p(0x900100000 - 4)),
])
def test_compact_rejects_overlap(L, kw):
    """Every destination against every source and every other destination: blocks would race. (Layers 2 x rows x 3 x 128 bf16.)"""
    assert _compact(L, **dict(_APART, **kw)) == 2
    assert "overlap" in _lib.last_error()


def test_compact_nothing_to_do(L):
    assert _compact(L, layers=0, sk=NULL, sel=NULL, dk=NULL) == 0
    assert _compact(L, keep=0, row0=60, sk=NULL, sel=NULL, dk=NULL) == 0


def test_binding_refuses_host_tensors():
    import torch

    import paper_2607_21848_amd as rv
    x = torch.zeros(4, 2, 128)
    with pytest.raises(ValueError, match="GPU tensor"):
        rv.rotary_embed(x, x, pairs=(22, 21, 21), theta=1e4, h=2, w=2)
    with pytest.raises(ValueError, match="GPU tensor"):
        rv.attention_key_weight(x, x, torch.zeros(2, 4), None, None, None, h=1, w=4, softmax_scale=1.0, lam=0.0, sigma=1.0)
    with pytest.raises(ValueError, match="GPU tensor"):
        rv.select_kept(torch.zeros(2, 1, 8), unit=1, keep=3)
    with pytest.raises(ValueError, match="GPU tensor"):
        rv.compact_kv(torch.zeros(1, 8, 2, 128), torch.zeros(1, 8, 2, 128), torch.zeros(1, 1, 2, dtype=torch.int32),
                      torch.zeros(1, 8, 2, 128), torch.zeros(1, 8, 2, 128), unit=4)
    with pytest.raises(TypeError, match="float8"):
        rv.rotary_embed(x, pairs=(22, 21, 21), theta=1e4, h=2, w=2, out_dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="heads"):
        rv.rotary_embed(x[0], pairs=(1, 1, 1), theta=1e4, h=2, w=2)
