"""What the paged cache's C entry points refuse of pools that come with a layout, checked without a GPU: every refusal is decided
on the host before anything is queued, and a call whose pools pass is refused for what is looked at after them."""

from __future__ import annotations

import ctypes
import math

import numpy as np
import pytest

from paper_2607_21848_amd import _lib
from tests.test_paged_abi_cpu import L, NULL, at  # noqa: F401

PAGES, H, PAGE, D = 3, 2, 64, 64
BASE = 4 << 30  # an address that is never dereferenced
PASSED = "out_len overlaps kv_len"


def _append(L, layout, k=0, v=1 << 26, sk=1 << 27, sv=1 << 28, dtype=4, **kw):
    a = dict(pages=PAGES, H=H, page=PAGE, D=D)
    a.update(kw)
    st = L.append_paged_kv_strided(at(1), a["H"] * a["D"], at(2), a["H"] * a["D"], dtype, 1, NULL, 1, at(3), at(3),
                                   *[None if x is None else ctypes.c_void_p(BASE + x) for x in (k, v, sk, sv)], at(20), a["pages"], a["page"], 4,
                                   a["H"], a["D"], NULL, 0, 4, 4, 8, 8, 8, 10000.0, layout, NULL)
    assert st in (1, 2)
    return _lib.last_error()


def _layout(k=(H * PAGE * D, PAGE * D, D), v=None, sk=(H * PAGE // 32, PAGE // 32, 1), sv=None):
    return _lib.PoolLayout(*k, *(v or k), *sk, *(sv or sk))


def test_layouts_that_pass(L):  # noqa: F811
    row = H * D
    for lay, kw in [
        (None, {}), (_layout(), {}),
        (_layout(k=(PAGE * row, D, row)), {}),                                                # positions before heads
        (_layout(k=(2 * PAGE * row, PAGE * D, D)), dict(v=PAGE * row)),                       # keys and values of a page
        (_layout(k=(2 * PAGE * row, D, 2 * row)), dict(v=row)),                               # of a position
        (_layout(k=(2 * PAGE * row, 2 * D, 2 * row)), dict(v=D)),                             # of a head
        (_layout(k=(PAGE * D, PAGES * PAGE * D, D)), {}),                                     # heads before pages
        (_layout(k=(PAGE * row, D, row), v=(H * PAGE * D, PAGE * D, D)), {}),                 # two layouts
        (_layout(k=(PAGE * (row + 16), D, row + 16)), {}),                                    # gaps behind rows
        # codes and scales of a page behind each other in one buffer
        (_layout(k=(20480, PAGE * D, D), sk=(20480, 2, 1)), dict(v=8192, sk=16384, sv=16384 + 4)),
        (_layout(sk=(2 * H, 1, H)), {}),                                                      # scales of blocks before heads
        (_layout(k=(7, PAGE * D, D)), dict(pages=1)), (_layout(k=(PAGE * D, 1, D)), dict(H=1)),  # distances that nothing is apart by
        (_layout(k=(16 * PAGE * row, D, row)), dict(dtype=1, sk=None, sv=None)), (_layout(sk=(-1, 5, 7)), dict(dtype=2, sk=None, sv=None, v=1 << 28)),
    ]:
        assert PASSED in _append(L, lay, **kw), (kw, _lib.last_error())


def test_layouts_that_are_refused(L):  # noqa: F811
    row = H * D
    for what, lay, kw in [
        ("negative", _layout(k=(-16, PAGE * D, D)), {}), ("too large", _layout(sk=(1 << 41, 2, 1)), {}), ("too much memory", _layout(k=(1 << 40, PAGE * D, D)), {}),
        ("16 bytes", _layout(k=(H * PAGE * D, PAGE * D, D + 8)), {}), ("16 bytes", _layout(v=(H * PAGE * D + 8, PAGE * D, D)), {}),
        ("cache_k share", _layout(k=(0, PAGE * D, D)), {}), ("cache_v share", _layout(v=(H * PAGE * D, 0, D)), {}), ("cache_k share", _layout(k=(PAGE * row, PAGE * D, D - 16)), {}),
        ("cache_k share", _layout(k=(PAGE * row, D, row - 16)), {}), ("cache_k share", _layout(k=(PAGE * row - 16, D, row)), {}),
        ("scale_v share", _layout(sv=(H * 2, 1, 1)), {}), ("scale_k share", _layout(sk=(3, 2, 1)), {}),
        ("cache_k and cache_v", _layout(), dict(v=0)), ("cache_k and cache_v", _layout(k=(2 * PAGE * row, D, 2 * row)), dict(v=row - 16)),
        ("cache_k and cache_v", _layout(k=(2 * PAGE * row, PAGE * D, D)), dict(v=PAGE * row - D)),
        ("cache_k share", _layout(k=(2 * PAGE * row, 2 * D, 2 * row)), dict(v=D, H=3)),
        ("cache_v and scale_k", _layout(k=(20480, PAGE * D, D), sk=(20480, 2, 1)), dict(v=8192, sk=16383, sv=16384 + 4)),
        ("scale_k and scale_v", _layout(k=(20480, PAGE * D, D), sk=(20480, 2, 1)), dict(v=8192, sk=16384, sv=16384 + 3)),
        # kinds of layout that are not alike count by their first and last byte
        ("cache_k and cache_v", _layout(k=(4 * PAGE * row, PAGE * D, D), v=(2 * PAGE * row, PAGE * D, D)), dict(v=PAGE * row)),
    ]:
        assert what in _append(L, lay, **kw), (what, kw, _lib.last_error())


def test_what_passes_is_apart(L):  # noqa: F811
    """Layouts and places at random: pools that pass share no byte, and pools of one layout that share none pass."""
    rng = np.random.default_rng(0)
    passed = refused = 0
    for _ in range(4000):
        n, h, page = int(rng.integers(1, 4)), int(rng.integers(1, 4)), 32

        def some():
            sizes, steps, span = {"page": n, "head": h, "row": page}, {}, D
            for d in rng.permutation(list(sizes)):
                steps[d] = span + 16 * int(rng.integers(0, 3)) * int(rng.integers(0, 40)) - 16 * int(rng.random() < 0.03)
                span = steps[d] * (sizes[d] - 1) + span
            f = 1 + int(rng.integers(0, 3))
            return tuple(f * steps[d] if d == "page" else steps[d] for d in ("page", "head", "row"))

        k = some()
        alike = rng.random() < 0.7
        v = k if alike else some()
        delta = 16 * int(rng.integers(-1200, 1200))
        sk, sv = (h, 1, 1), (h, 1, 1)
        i = np.arange(n)[:, None, None], np.arange(h)[:, None], np.arange(page)
        byte = [np.unique((sum(x * s for x, s in zip(i, st)).ravel()[:, None] + np.arange(0, D, 16)), return_counts=True) for st in (k, v)]
        alone = all((c == 1).all() for _, c in byte)
        apart = alone and not np.intersect1d(byte[0][0], byte[1][0] + delta).size
        err = _append(L, _lib.PoolLayout(*k, *v, *sk, *sv), k=1 << 20, v=(1 << 20) + delta, sk=1 << 27, sv=1 << 28, pages=n, H=h, page=page)
        if PASSED in err:
            assert apart, (k, v, delta)
            passed += 1
        else:
            refused += 1
            assert not (apart and alike and "overlap" in err), (k, delta, err)
    assert passed > 500 and refused > 500


def _attend(L, layout, o=1 << 33, **kw):  # noqa: F811
    a = dict(k=0, v=1 << 26, sk=1 << 27, sv=1 << 28, vis=NULL, dtype=4)
    a.update(kw)
    pools = [None if a[x] is None else ctypes.c_void_p(BASE + a[x]) for x in ("k", "v", "sk", "sv")]
    return L.paged_chunk_attention_strided(at(1), H * D, *pools, ctypes.c_void_p(BASE + o), at(15), a["dtype"], 1, NULL, 1, at(3), a["vis"], at(14),
                                           PAGES, PAGE, 4, H, H, D, 0, 0, NULL, 0, NULL, NULL, 0, 1 / math.sqrt(D), 0.0, 1.0, 0, 2, NULL, 0, layout,
                                           NULL), _lib.last_error()


def test_attention(L):  # noqa: F811
    row = H * D
    # refused for the workspace, which is looked at behind the pools
    for lay in (None, _layout(), _layout(k=(0, 0, 0), sk=(0, 0, 0)), _layout(k=(PAGE * row, D, row)), _layout(k=(2 * PAGE * row, D, 2 * row))):
        st, err = _attend(L, lay)
        assert st == 2 and "workspace of 0 bytes" in err
    for lay, kw, what in [(_layout(k=(-16, 0, 0)), {}, "negative"), (_layout(k=(PAGE * row, D, row + 8)), {}, "16 bytes"), (_layout(sv=(1 << 41, 0, 0)), {}, "too large"),
                          (_layout(k=(1 << 40, D, row)), {}, "too much memory"), (_layout(k=(PAGE * row * 8, D, row)), dict(o=PAGE * row * 8), "o overlaps cache_k"),
                          (_layout(sk=(1 << 20, 2, 1)), dict(o=(1 << 27) + (1 << 21)), "o overlaps scale_k")]:
        st, err = _attend(L, lay, **kw)
        assert st == 2 and what in err, (what, err)


def test_keys_that_are_copied_have_no_grid(L):  # noqa: F811
    def append(pairs, h, w):
        L.append_paged_kv(at(1), H * D, at(2), H * D, 2, 1, NULL, 1, at(3), at(3), at(4), at(5), NULL, NULL, at(20), PAGES, PAGE, 4, H, D, NULL, 0, h, w,
                          *pairs, 10000.0, NULL)
        return _lib.last_error()
    for h, w in ((0, 0), (-1, 5), (1 << 20, 1 << 20)):
        assert PASSED in append((0, 0, 0), h, w)
        assert "token grid" in append((0, 0, 1), h, w)
