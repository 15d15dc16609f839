"""append_paged_kv against its fp64 oracle: types, head sizes, page sizes, blocks that begin and end anywhere, streams of
no tokens, scales that grow, values that are not finite, pages that are none.

Tolerance. Values are copied, or rounded to the nearest code: equal. A turned key is within 6 units of 2^-24 of
(|x| + |y|) of the exact one before its rounding (as rotary_embed's), which adds half a step: 2^-8 of the value (bf16),
2^-24 (fp32), 2^-4 (e4m3; 2^-10 of the scale below its smallest normal value)."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from oracle import paged as OP
from tests.paged_helpers import BF16, DEV, F32, FP8, GIVEN, Pool, gen, values

pytestmark = pytest.mark.gpu
THETA = 10000.0


def _bands(D):
    return D // 2 - 2 * (D // 6), D // 6, D // 6


def _snapshot(pool):
    return [x.clone() for x in (pool.k, pool.v)] + [None if s is None else s.view(torch.uint8).clone() for s in pool.scales]


def _check(pool, was, k, v, cu, before, pairs, pos):
    """Everything that the pools hold now."""
    n, H, D = k.shape
    k64, v64 = (x.float().double().cpu().numpy() for x in (k, v))
    got, lens = OP.append(k64, v64, cu, before, pool.table, pool.page, pos, pairs, THETA, pool.n_pages)
    mag = np.repeat(np.abs(k64[..., 0::2]) + np.abs(k64[..., 1::2]), 2, -1)
    magnitude, turned = {}, np.arange(D) < 2 * sum(pairs)
    cap = pool.table.shape[1] * pool.page
    for s, (t0, m) in enumerate(OP.streams(n, cu, len(pool.table))):
        held = min(max(before[s], 0), cap)
        for i in range(t0, t0 + m):
            c = held + i - t0
            if c < cap and 0 <= pool.table[s, c // pool.page] < pool.n_pages:
                for h in range(H):
                    magnitude[int(pool.table[s, c // pool.page]), h, c % pool.page] = mag[i, h]
    where = np.zeros((pool.n_pages, H, pool.page), bool)
    for p, h, r in got:
        where[p, h, r] = True
    for which, x in ((0, pool.k), (1, pool.v)):
        now, old = x.float().double().cpu().numpy(), was[which].float().double().cpu().numpy()
        if pool.dtype != FP8:
            assert np.array_equal(now[~where], old[~where], equal_nan=True)
            for at, kv in got.items():
                want = kv[which]
                half = 2.0 ** -8 if pool.dtype == BF16 else 2.0 ** -24
                tol = np.where(turned & (which == 0), 6 * 2.0 ** -24 * magnitude[at] + half * np.abs(want), 0.0)
                assert ((np.abs(now[at] - want) <= tol) | (np.isnan(now[at]) & np.isnan(want))).all(), (which, at)
            continue
        sc_now, sc_old = pool.scales[which].view(torch.uint8).cpu().numpy().astype(int), was[2 + which].cpu().numpy().astype(int)
        # blocks that tokens went to, and the rows that they held before
        blocks = {}
        for (p, h, r), kv in got.items():
            blocks.setdefault((p, h, r // 32), []).append((r, kv[which], magnitude[p, h, r]))
        held_rows = {}
        for s, (t0, m) in enumerate(OP.streams(n, cu, len(pool.table))):
            held = min(max(before[s], 0), cap)
            if m and held < cap and 0 <= pool.table[s, held // pool.page] < pool.n_pages:
                held_rows[int(pool.table[s, held // pool.page]), held % pool.page // 32] = held % 32
        for p in range(pool.n_pages):
            for h in range(H):
                for b in range(pool.page // 32):
                    rows = slice(32 * b, 32 * b + 32)
                    if (p, h, b) not in blocks:
                        assert sc_now[p, h, b] == sc_old[p, h, b] and np.array_equal(now[p, h, rows], old[p, h, rows], equal_nan=True)
                        continue
                    new = blocks[p, h, b]
                    most = max([float(np.abs(x[np.isfinite(x)]).max(initial=0)) for _, x, _ in new])
                    keep = held_rows.get((p, b), 0)
                    want_e = {OP.exponent(most * f) for f in ((1 - 2.0 ** -20, 1, 1 + 2.0 ** -20) if which == 0 else (1,))}
                    if keep:
                        want_e = {max(e, sc_old[p, h, b] - 127) for e in want_e}
                    e = sc_now[p, h, b] - 127
                    assert e in want_e, (which, p, h, b, e, want_e)
                    f = 2.0 ** (sc_old[p, h, b] - 127 - e)
                    again = OP.round_e4m3(old[p, h, 32 * b:32 * b + keep] * f)
                    assert np.array_equal(now[p, h, 32 * b:32 * b + keep], again, equal_nan=True), (which, p, h, b)
                    fresh = np.zeros(32, bool)
                    fresh[:keep] = True
                    for r, x, mg in new:
                        fresh[r % 32] = True
                        aim = np.where(np.isfinite(x), x, np.nan) * 2.0 ** -e
                        code = now[p, h, r]
                        if which == 1:
                            assert np.array_equal(code, OP.round_e4m3(aim), equal_nan=True), (p, h, r)
                        else:
                            tol = np.maximum(np.abs(aim) * 2.0 ** -4, 2.0 ** -10) + 6 * 2.0 ** -24 * np.where(turned, mg, 0) * 2.0 ** -e
                            assert ((np.abs(code - aim) <= tol) | (np.isnan(code) & np.isnan(aim))).all(), (p, h, r)
                    assert np.array_equal(now[p, h, rows][~fresh], old[p, h, rows][~fresh], equal_nan=True)
    return lens


def _run(pool, k, v, cu, before, pairs, h=5, w=7, t0=3, pos=None):
    was = _snapshot(pool)
    table = torch.from_numpy(pool.table).to(DEV)
    lens = torch.tensor(before, dtype=torch.int32, device=DEV)
    at = None if pos is None else torch.from_numpy(pos).to(DEV)
    got = rv.append_paged_kv(k, v, pool.k, pool.v, table, lens, cu=None if cu is None else torch.tensor(cu, dtype=torch.int32, device=DEV),
                             pairs=pairs, theta=THETA, h=h, w=w, t0=t0, pos=at, **pool.kw())
    place = (lambda i, c: tuple(pos[i])) if pos is not None else (lambda i, c: (t0 + c // (h * w), c // w % h, c % w))
    want = _check(pool, was, k, v, cu, before, pairs, place)
    assert got.tolist() == want and lens.tolist() == list(before)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,H,before,new", [
    (32, 1, [0], [1]), (64, 5, [63], [1]), (32, 3, [31, 0, 32], [2, 1, 33]), (128, 4, [7], [300]), (32, 9, [5, 0, 17, 64], [0, 40, 16, 1]),
    (256, 2, [255, 1], [2, 95]),
])
def test_append(dtype, D, page, H, before, new):
    pool = Pool(1, dtype, [a + b for a, b in zip(before, new)], H, D, page)
    cu = np.concatenate([[0], np.cumsum(new)])
    n = int(cu[-1])
    g = gen(2)
    k, v = (values(g, GIVEN[dtype], n, H, D) * 4 for _ in range(2))
    _run(pool, k, v, cu.tolist(), before, _bands(D))


@pytest.mark.parametrize("dtype", [FP8, BF16])
def test_even_shares_strided_rows_and_given_positions(dtype):
    B, H, D, page, m = 70, 6, 128, 32, 3  # more streams than a wave has lanes
    before = [int(x) for x in np.random.default_rng(0).integers(0, 70, B)]
    rows = values(gen(3), GIVEN[dtype], B * m, 3, H, D)
    k, v = rows[:, 1], rows[:, 2]
    pos = np.random.default_rng(1).integers(-1000, 100000, (B * m, 3)).astype(np.int32)
    for cu in (None, list(range(0, B * m + 1, m))):
        _run(Pool(4, dtype, [b + m for b in before], H, D, page), k, v, cu, before, (20, 11, 13), pos=pos)


def test_uneven_shares_over_many_streams():
    B, H, D = 150, 2, 64
    rng = np.random.default_rng(5)
    new = rng.integers(0, 5, B)
    new[:3] = (0, 70, 0)
    before = rng.integers(0, 40, B).tolist()
    cu = np.concatenate([[0], np.cumsum(new)])
    n = int(cu[-1])
    # tokens behind the last stream's are nobody's
    k, v = (values(gen(6 + i), BF16, n + 9, H, D) for i in range(2))
    _run(Pool(7, FP8, [a + int(b) for a, b in zip(before, new)], H, D, 32), k, v, cu.tolist(), before, _bands(D))


def test_scales_grow_and_codes_follow():
    H, D, page = 3, 128, 32
    pool = Pool(8, FP8, [32], H, D, page)
    before = 0
    # tokens of growing and falling size: 2^-30 up to 2^20 and back
    for i, e in enumerate((-30, -30, -10, -12, 0, 5, 4, 20, 3, -40)):
        k, v = (values(gen(20 + i), BF16, 2, H, D) * 2.0 ** (e + j) for j in range(2))
        _run(pool, k, v, None, [before], _bands(D))
        before += 2


def test_values_at_the_ends():
    """Zeros, the smallest and largest values, infinities and NaN; the border between two scales."""
    H, D, page = 2, 64, 32
    pool = Pool(9, FP8, [64], H, D, page)
    k = torch.zeros(8, H, D, dtype=BF16, device=DEV)
    v = k.clone()
    v[0, 0, :4] = torch.tensor([float("inf"), float("-inf"), float("nan"), 3.0e38])
    v[1, 1, :3] = torch.tensor([448.0, -448.0, 1.0])
    v[2, 1, 5] = 1e-38
    k[3, 0, 60:62] = torch.tensor([float("nan"), float("inf")])  # behind the bands below
    _run(pool, k, v, None, [28], (8, 0, 0))
    # alone in their block: nothing but zeros, then 448 and the next bf16 value above it
    pool = Pool(10, FP8, [96], H, D, page)
    v = torch.zeros(96, H, D, dtype=BF16, device=DEV)
    v[32:64, 0, 0], v[64:, 0, 0] = 448.0, 450.0
    _run(pool, torch.zeros_like(v), v, None, [0], (0, 0, 0))
    e = pool.scales[1].view(torch.uint8).cpu().numpy().astype(int)[pool.table[0], 0, 0] - 127
    assert e.tolist() == [-100, 0, 1]


@pytest.mark.parametrize("dtype", [FP8, F32])
def test_pages_that_are_none_and_full_streams(dtype):
    """Entries outside the pool, and positions past the table's end: dropped."""
    H, D, page = 2, 64, 32
    pool = Pool(11, dtype, [160, 160, 160], H, D, page, max_pages=5)
    pool.table[0, 1], pool.table[1, 0], pool.table[2, 2] = -1, pool.n_pages, 2**31 - 1
    k, v = (values(gen(12 + i), GIVEN[dtype], 3 * 100, H, D) for i in range(2))
    _run(pool, k, v, None, [0, 100, 20], _bands(D))
    _run(pool, k, v, None, [-5, 159, 1000], _bands(D))


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
def test_zero_tokens(dtype):
    pool = Pool(13, dtype, [40, 3], 2, 64, 32)
    was = _snapshot(pool)
    k = torch.empty(0, 2, 64, dtype=GIVEN[dtype], device=DEV)
    got = rv.append_paged_kv(k, k, *pool.args(), pairs=(8, 8, 8), theta=THETA, h=3, w=3, **pool.kw())
    assert got.tolist() == [40, 3] and torch.equal(pool.k.view(torch.uint8), was[0].view(torch.uint8))


def test_caches_past_2_to_32_bytes():
    H, D, page = 40, 128, 256
    n_pages = (1 << 32) // (H * D * page) + 3
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device=DEV)
    ck, cv = (torch.empty(n_pages, H, page, D, dtype=FP8, device=DEV) for _ in range(2))
    sk, sv = (torch.zeros(n_pages, H, page // 32, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu) for _ in range(2))
    k, v = (values(gen(14 + i), BF16, 600, H, D) for i in range(2))
    rv.append_paged_kv(k, v, ck, cv, table, torch.zeros(1, dtype=torch.int32, device=DEV), pairs=(0, 0, 0), theta=THETA, h=1, w=1,
                       scale_k=sk, scale_v=sv)
    for x, cache, scale in ((k, ck, sk), (v, cv, sv)):
        for i, p in enumerate((n_pages - 1, 0, n_pages - 2)):
            rows = x[256 * i:256 * i + 256].transpose(0, 1).float()
            m = rows.shape[1]
            now = cache[p].float() * torch.exp2(scale.view(torch.uint8)[p].float() - 127).repeat_interleave(32, 1)[..., None]
            assert ((now[:, :m] - rows).abs() <= rows.abs() * 2.0 ** -4 + 1e-3).all()


def test_refusals():
    pool = Pool(15, FP8, [64], 2, 64, 32)
    ck, cv, table, lens = pool.args()
    k = values(gen(16), BF16, 4, 2, 64)
    ok = dict(pairs=(8, 8, 8), theta=THETA, h=3, w=3, **pool.kw())
    for err, args, kw in [
        (TypeError, (k.float(), k, ck, cv, table, lens), ok), (ValueError, (k[:, :1], k, ck, cv, table, lens), ok),
        (ValueError, (k, k[:2], ck, cv, table, lens), ok), (TypeError, (k, k, ck.half(), cv, table, lens), ok),
        (ValueError, (k, k, ck, cv[:1], table, lens), ok), (TypeError, (k, k, ck, cv, table, lens), {**ok, "scale_k": None}),
        (TypeError, (k, k, ck, cv, table, lens), {**ok, "scale_v": ok["scale_v"].view(torch.uint8)}), (ValueError, (k, k, ck, cv, table[0], lens), ok),
        (ValueError, (k, k, ck.cpu(), cv, table, lens), ok), (ValueError, (k, k, ck, cv, table, lens), {**ok, "pos": torch.zeros(3, 3, dtype=torch.int32, device=DEV)}),
        (ValueError, (k[:3], k[:3], ck, cv, table.repeat(2, 1), lens.repeat(2)), ok), (rv.RevisitError, (k, k, ck, cv, table, lens), {**ok, "out_len": lens}),
        (rv.RevisitError, (k, k, ck, ck, table, lens), ok), (rv.RevisitError, (k, k, ck, cv, table, lens), {**ok, "h": 0}),
        (ValueError, (k, k, ck.float().to(BF16), cv.float().to(BF16), table, lens), ok),
    ]:
        with pytest.raises(err):
            rv.append_paged_kv(*args, **kw)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("pairs", [(0, 0, 0), (64, 0, 0), (0, 64, 0), (0, 0, 64), (0, 1, 2), (63, 0, 1), (31, 33, 0)])
def test_places_in_runs(dtype, pairs):
    """Bands of any size, at places that repeat on one axis or another, in order or not, far from zero and below it."""
    H, D, page, before, n = 3, 128, 64, [20, 3], 2 * 50
    rng = np.random.default_rng(30)
    pos = np.stack([np.repeat(rng.integers(-2**30, 2**30, 10), 10), np.tile([4, 4, 4, -7], 25), rng.permutation(n)], 1).astype(np.int32)
    pos[60:] = pos[60]  # all alike
    k, v = (values(gen(31 + i), GIVEN[dtype], n, H, D) for i in range(2))
    _run(Pool(32, dtype, [b + 50 for b in before], H, D, page), k, v, None, before, pairs, pos=pos)
    _run(Pool(33, dtype, [b + 50 for b in before], H, D, page), k, v, None, before, pairs, h=1, w=1, t0=-5)


def test_turned_pairs_past_fp32():
    """A pair of finite values whose turn leaves fp32 is stored as NaN, and its block's scale comes from the others."""
    H, D, page = 1, 64, 32
    pool = Pool(34, FP8, [32], H, D, page)
    k = torch.ones(32, H, D, dtype=BF16, device=DEV)
    k[7, 0, 2:4] = torch.tensor([3.3e38, 3.3e38])
    pos = torch.zeros(32, 3, dtype=torch.int32, device=DEV)
    pos[7, 0] = 1  # theta^(-1/2) = pi / 4 for pair 1
    rv.append_paged_kv(k, torch.ones_like(k), pool.k, pool.v, torch.from_numpy(pool.table).to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV),
                       pairs=(2, 0, 0), theta=(4 / np.pi) ** 2, pos=pos, **pool.kw())
    page0 = int(pool.table[0, 0])
    got = pool.k[page0, 0].float()
    # x cos - y sin is far below y's own rounding or not, x sin + y cos = 4.7e38 in any case
    assert bool(torch.isnan(got[7, 3]))
    small = float(3.3e38 * 2.0 ** -7)  # what a rounded pi / 4 may leave of the difference
    e = int(pool.scales[0].view(torch.uint8)[page0, 0, 0]) - 127
    assert 2.0 ** e * 448 < small
    rest = torch.ones(32, D, dtype=torch.bool, device=DEV)
    rest[7, :4] = False
    back = got * 2.0 ** e
    assert bool((back[rest] <= 1).all()) and bool(torch.isfinite(back[rest]).all())
