"""Refusals of the paged cache's C entry points, checked without a GPU: every one is decided on the host before
anything is queued."""

from __future__ import annotations

import ctypes
import math

import pytest

from paper_2607_21848_amd import _lib

NULL = None


def at(gib, plus=0):
    """An address that is never dereferenced: validation fails first, or there is nothing to do."""
    return ctypes.c_void_p((gib << 30) + plus)


@pytest.fixture(scope="module")
def L():
    return _lib.lib()


def _append(L, **kw):
    a = dict(k=at(1), k_row=1536, v=at(2), v_row=1536, dtype=4, n=10, cu=NULL, B=2, len=at(3), out=at(3, 4096), ck=at(4), cv=at(8), sk=at(12),
             sv=at(13), table=at(14), pages=100, page=64, most=40, H=12, D=128, pos=NULL, t0=0, h=30, w=52, nt=22, ny=21, nx=21, theta=10000.0)
    a.update(kw)
    return L.append_paged_kv(*[a[x] for x in ("k", "k_row", "v", "v_row", "dtype", "n", "cu", "B", "len", "out", "ck", "cv", "sk", "sv", "table",
                                              "pages", "page", "most", "H", "D", "pos", "t0", "h", "w", "nt", "ny", "nx", "theta")], NULL)


SHARED = [
    (dict(dtype=0), 3), (dict(dtype=3), 3), (dict(dtype=5), 3), (dict(D=96), 3), (dict(D=256), 3), (dict(n=-1), 2), (dict(n=(1 << 30) + 2), 2),
    (dict(B=-1), 2), (dict(B=(1 << 20) + 1, cu=at(20)), 2), (dict(pages=-1), 2), (dict(most=-1), 2), (dict(page=16), 2), (dict(page=48), 2),
    (dict(page=8192), 2), (dict(page=0), 2), (dict(page=-64), 2), (dict(most=1 << 25), 2), (dict(pages=2**31 - 1, page=4096), 2),
    (dict(n=11), 2), (dict(B=0), 2), (dict(cu=at(20, 2)), 2), (dict(len=at(3, 1)), 2), (dict(table=at(14, 2)), 2), (dict(len=NULL), 1),
    (dict(table=NULL), 1), (dict(ck=NULL), 1), (dict(cv=NULL), 1), (dict(sk=NULL), 1), (dict(sv=NULL), 1), (dict(ck=at(4, 8)), 2), (dict(cv=at(8, 8)), 2),
]


@pytest.mark.parametrize("kw,status", SHARED + [
    (dict(H=0), 2), (dict(H=65536), 2), (dict(nt=23), 4), (dict(ny=-1), 4), (dict(nt=2**31 - 1, ny=2**31 - 1), 4), (dict(theta=0.0), 4),
    (dict(theta=float("inf")), 4), (dict(h=0), 2), (dict(w=0), 2), (dict(h=1 << 16, w=1 << 16), 2), (dict(k_row=1535), 2), (dict(v_row=1528), 2),
    (dict(k_row=1540), 2), (dict(v_row=1 << 41), 2), (dict(k=NULL), 1), (dict(v=NULL), 1), (dict(k=at(1, 8)), 2), (dict(v=at(2, 8)), 2),
    (dict(out=at(3, 4097)), 2), (dict(pos=at(20, 2)), 2),
    # overlaps: of the caches with each other, with inputs, and of the lengths with themselves (100 pages of 12 heads: 9.8 MB a cache)
    (dict(cv=at(4, 4096)), 2), (dict(k=at(4, 9830400 - 16)), 2), (dict(v=at(8, 16)), 2), (dict(k=at(4, -(9 * 1536 + 1536) * 2 + 16)), 2),
    (dict(sk=at(4, 16)), 2), (dict(sv=at(12, 2399)), 2), (dict(out=at(3)), 2), (dict(out=at(3, 4)), 2), (dict(out=at(14, 8)), 2),
    (dict(table=at(4, 32)), 2), (dict(cu=at(12, 4)), 2), (dict(pos=at(8, 64)), 2), (dict(sv=at(4, 9830399)), 2),
])
def test_append_rejects(L, kw, status):
    assert _append(L, **kw) == status
    assert "append_paged_kv" in _lib.last_error()


def test_append_nothing_to_do(L):
    assert _append(L, n=0, B=0, k=NULL, v=NULL, ck=NULL, cv=NULL, sk=NULL, sv=NULL, table=NULL, len=NULL, out=NULL) == 0
    assert _append(L, n=0, out=NULL, len=NULL, k=NULL, v=NULL) == 0
    assert _append(L, n=5, B=0, cu=at(20)) == 0  # nobody's tokens


def _attend(L, **kw):
    a = dict(q=at(1), q_row=1536, ck=at(4), cv=at(8), sk=at(12), sv=at(13), o=at(2), lse=at(2, 1 << 20), dtype=4, n=10, cu=NULL, B=2, len=at(3),
             vis=NULL, table=at(14), pages=100, page=64, most=40, Hq=12, Hk=12, D=128, h=30, w=52, slot=at(15), frames=2, uv=at(16), idx=at(17),
             S=2, scale=1 / math.sqrt(128), lam=1.0, sigma=2.0, max_keys=0, parts=1, ws=NULL, ws_bytes=0)
    a.update(kw)
    return L.paged_chunk_attention(*[a[x] for x in (
        "q", "q_row", "ck", "cv", "sk", "sv", "o", "lse", "dtype", "n", "cu", "B", "len", "vis", "table", "pages", "page", "most", "Hq", "Hk", "D",
        "h", "w", "slot", "frames", "uv", "idx", "S", "scale", "lam", "sigma", "max_keys", "parts", "ws", "ws_bytes")], NULL)


@pytest.mark.parametrize("kw,status", SHARED + [
    (dict(Hk=0), 2), (dict(Hk=65536), 2), (dict(Hq=0), 2), (dict(Hq=13), 2), (dict(Hq=65544, Hk=8), 2), (dict(Hq=6), 2), (dict(max_keys=-1), 4),
    (dict(n=1 << 30, B=1, Hq=24), 2), (dict(parts=-1), 4), (dict(parts=65), 4), (dict(scale=0.0), 4), (dict(scale=float("nan")), 4),
    (dict(S=-1), 2), (dict(lam=float("nan")), 4), (dict(sigma=0.0), 4), (dict(sigma=float("inf")), 4), (dict(lam=3e38, sigma=1e-3), 4),
    (dict(h=0), 2), (dict(w=-1), 2), (dict(h=257), 2), (dict(w=257), 2), (dict(frames=-1), 2), (dict(q_row=1535), 2), (dict(q_row=1540), 2),
    (dict(q_row=1 << 41), 2), (dict(q=NULL), 1), (dict(o=NULL), 1), (dict(slot=NULL), 1), (dict(uv=NULL), 1), (dict(idx=NULL), 1),
    (dict(q=at(1, 8)), 2), (dict(o=at(2, 8)), 2), (dict(lse=at(2, 2)), 2), (dict(vis=at(3, 2)), 2), (dict(uv=at(16, 4)), 2), (dict(idx=at(17, 2)), 2),
    # outputs over inputs and over each other
    (dict(o=at(1)), 2), (dict(o=at(1, 10 * 1536 * 2 - 16)), 2), (dict(lse=at(2, 16)), 2), (dict(o=at(4)), 2), (dict(o=at(12, -16)), 2),
    (dict(lse=at(3, 4)), 2), (dict(lse=at(14)), 2), (dict(vis=at(2, 64)), 2), (dict(lse=at(16, 8)), 2), (dict(lse=at(15)), 2),
    # three parts of 2 tiles of 16 rows by 12 heads: no workspace, too small, NULL, misaligned, over an output
    (dict(parts=3), 2), (dict(parts=3, ws=at(30), ws_bytes=3 * 24 * 16 * 130 * 4 - 1), 2), (dict(parts=3, ws_bytes=1 << 30), 1),
    (dict(parts=3, ws=at(30, 8), ws_bytes=1 << 30), 2), (dict(parts=3, ws=at(2, 16), ws_bytes=1 << 20), 2),
])
def test_attention_rejects(L, kw, status):
    assert _attend(L, **kw) == status
    assert "paged_chunk_attention" in _lib.last_error()


def test_attention_nothing_to_do(L):
    assert _attend(L, n=0, q=NULL, o=NULL, lse=NULL, ck=NULL, cv=NULL, len=NULL, table=NULL) == 0
    assert _attend(L, n=0, B=0) == 0
    assert _attend(L, n=7, B=0, cu=at(20)) == 0


def test_bias_is_not_read_when_off(L):
    # the refusal that follows says that the grid and the pointers were not looked at
    for off in (dict(S=0), dict(lam=0.0)):
        assert _attend(L, h=0, w=0, slot=NULL, uv=NULL, idx=NULL, sigma=0.0, q=NULL, **off) == 1
        assert "q and o" in _lib.last_error()


def test_attention_workspace(L):
    n = ctypes.c_size_t(7)
    size = lambda *a: (L.rc_paged_attention_workspace_size(*a, ctypes.byref(n)), n.value)  # noqa: E731
    row = (128 + 2) * 4
    # dtype, tokens, ragged, streams, Hq, Hk, D, page, max_pages, max_keys, parts
    assert size(4, 10, 0, 2, 12, 12, 128, 64, 40, 0, 3) == (0, 3 * 2 * 12 * 16 * row)
    assert size(4, 10, 1, 2, 12, 12, 128, 64, 40, 0, 3) == (0, 3 * (10 // 16 + 2) * 12 * 16 * row)  # a tile more per stream
    assert size(1, 2, 0, 2, 32, 8, 64, 64, 40, 0, 2) == (0, 2 * 2 * 8 * 16 * (64 + 2) * 4)
    assert size(4, 10, 0, 2, 12, 12, 128, 64, 1, 0, 64) == (0, 2 * 2 * 12 * 16 * row)  # two key tiles are two parts
    assert size(4, 10, 0, 2, 12, 12, 128, 64, 40, 32, 64) == (0, 0)                     # one key tile
    assert size(4, 10, 0, 2, 12, 12, 128, 64, 40, 0, 1) == (0, 0)
    assert size(4, 0, 0, 2, 12, 12, 128, 64, 40, 0, 8) == (0, 0)
    assert size(4, 10, 0, 0, 12, 12, 128, 64, 40, 0, 8) == (2, 0)
    assert size(4, 10, 0, 2, 13, 12, 128, 64, 40, 0, 8) == (2, 0)
    assert L.rc_paged_attention_workspace_size(4, 10, 0, 2, 12, 12, 128, 64, 40, 0, 3, None) == 1
