"""paged_chunk_attention against its fp64 oracle: types, head layouts, lengths from one key on, uneven streams, what a
query sees, pages in any order and none, the bias, and values that must not be seen (tolerances: check_attention)."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from oracle import attention as OA
from tests.paged_helpers import BF16, DEV, F32, FP8, GIVEN, Pool, check_attention, gen, values

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(autouse=True, params=[0, 1 << 19], ids=["table", "wide_table"])
def room(request, monkeypatch):
    """Page tables with just the entries that the streams need, and with entries for far longer ones, for which other
    tiles are chosen."""
    monkeypatch.setattr(Pool, "room", request.param)


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _attend(pool, q, cu=None, visible=None, **kw):
    return rv.paged_chunk_attention(q, *pool.args(), cu=None if cu is None else _i32(cu), visible=None if visible is None else _i32(visible),
                                    softmax_scale=q.shape[-1] ** -0.5, **pool.kw(), **kw)


def _causal(lens, cu):
    """Queries are their stream's last positions."""
    return np.concatenate([L - (b - a) + 1 + np.arange(b - a) for L, a, b in zip(lens, cu[:-1], cu[1:])] + [np.zeros(0)]).astype(np.int32)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,Hq,Hk,lens,new", [
    (32, 1, 1, [1], [1]), (64, 4, 4, [33], [1]), (32, 8, 2, [100, 7, 64], [1, 1, 1]), (128, 5, 1, [300], [3]), (64, 6, 3, [129, 65], [9, 2]),
    (32, 2, 2, [200], [40]), (256, 3, 1, [700], [21]), (32, 4, 2, [97, 0, 260, 31], [33, 2, 0, 70]), (64, 2, 1, [500], [150]),
    (32, 2, 2, [33, 129], [129, 128]), (64, 6, 2, [300, 0, 64, 1], [200, 70, 30, 1]), (32, 1, 1, [31], [70]), (128, 3, 3, [160], [127]),
])
@pytest.mark.parametrize("causal", [False, True])
def test_shapes(dtype, D, page, Hq, Hk, lens, new, causal):
    pool = Pool(1, dtype, lens, Hk, D, page)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = values(gen(2), GIVEN[dtype], int(cu[-1]), Hq, D)
    visible = _causal(lens, cu) if causal else None
    o, lse = _attend(pool, q, cu, visible)
    check_attention(pool, q, o, lse, cu, visible)
    if len(set(new)) == 1:
        o2, lse2 = _attend(pool, q, None, visible)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("parts", [1, 2, 3, 7, 64])
@pytest.mark.parametrize("new", [[3, 1, 2, 20], [60, 0, 40, 150]])
def test_key_parts(dtype, parts, new):
    lens = [1000, 45, 0, 333]
    pool = Pool(3, dtype, lens, 2, 128, 64)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = values(gen(4), GIVEN[dtype], int(cu[-1]), 4, 128)
    visible = np.random.default_rng(0).integers(-3, 1100, int(cu[-1]))
    visible[1] = 0
    o, lse = _attend(pool, q, cu, visible, key_parts=parts)
    check_attention(pool, q, o, lse, cu, visible)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("m", [1, 17, 40, 150])
def test_what_is_not_seen_may_be_anything(dtype, m):
    """Keys and values behind a query's last one, and rows of a page behind the stream's end: NaN, infinities, the type's
    largest value. What is seen and not finite shows."""
    L, H, D, page = 170, 2, 128, 64
    pool = Pool(5, dtype, [L], H, D, page)
    q = values(gen(6), GIVEN[dtype], m, H, D)
    visible = np.arange(L - m, L) + 1
    if m == 1:
        visible[:] = 150
    bad = {FP8: [NAN, -NAN, 448.0], BF16: [NAN, INF, -INF], F32: [NAN, INF, -INF]}[dtype]
    k, v = pool.k.float(), pool.v.float()
    t = pool.table[0]
    # the rest of the last page belongs to nobody
    k[t[2], :, L % page:], v[t[2], :, L % page:] = NAN, NAN
    # positions that only the last queries see
    for j, c in enumerate((155, 156, 168, 169)):
        v[t[c // page], j % 2, c % page, 5 * j:5 * j + 3] = torch.tensor(bad, device=DEV)
    k[t[159 // page], 1, 159 % page, 3] = NAN
    pool.k, pool.v = k.to(dtype), v.to(dtype)
    o, lse = _attend(pool, q, None, visible)
    k64, _, _ = pool.held(0)
    blind = np.flatnonzero(visible <= 155)
    seen_k = np.flatnonzero(visible > 159)
    if len(blind):
        assert bool(torch.isfinite(o[blind[0]:blind[-1] + 1]).all())
    # a NaN logit makes the whole head's output and its LSE NaN
    for p in seen_k:
        assert bool(torch.isnan(o[p, 1]).all()) and bool(torch.isnan(lse[1, p]))
    keep = np.flatnonzero(visible <= 159)
    if len(keep):
        sub = slice(int(keep[0]), int(keep[-1]) + 1)
        check_attention(pool, q[sub], o[sub], lse[:, sub].contiguous(), None, visible[sub])
    # head 0 has no NaN logit: its values' own, seen or not
    one = Pool(5, dtype, [L], 1, D, page)
    one.table, one.n_pages = pool.table, pool.n_pages
    one.k, one.v = pool.k[:, :1].contiguous(), pool.v[:, :1].contiguous()
    one.scales = [None if s is None else s.view(torch.uint8)[:, :1].contiguous().view(torch.float8_e8m0fnu) for s in pool.scales]
    check_attention(one, q[:, :1], o[:, :1], lse[:1], None, visible)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("m", [3, 50])
def test_pages_that_are_none(dtype, m):
    lens = [400, 90, 64]
    pool = Pool(7, dtype, lens, 2, 64, 32)
    pool.table[0, [0, 5, 6, 12]] = (-1, pool.n_pages, 2**31 - 1, -7)
    pool.table[1, :] = -1  # a stream without any page
    q = values(gen(8), GIVEN[dtype], 3 * m, 4, 64)
    # what lies in the pool's pages must not show through entries that are none
    pool.k[0], pool.v[0] = (torch.full_like(x[0].float(), NAN).to(dtype) for x in (pool.k, pool.v))
    pool.table[pool.table == 0] = -1
    o, lse = _attend(pool, q)
    check_attention(pool, q, o, lse)
    assert bool((o[m:2 * m] == 0).all()) and bool((lse[:, m:2 * m] == -INF).all())
    # two entries of one page
    pool.table[2, :] = pool.table[2, 0]
    o, lse = _attend(pool, q)
    check_attention(pool, q, o, lse)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
def test_no_pages_at_all(dtype):
    k = torch.empty(0, 2, 32, 64, dtype=dtype, device=DEV)
    sc = dict(scale_k=torch.empty(0, 2, 1, dtype=torch.float8_e8m0fnu, device=DEV), scale_v=torch.empty(0, 2, 1, dtype=torch.float8_e8m0fnu, device=DEV))
    for m in (1, 100):
        for entries in (0, 3):
            table = torch.zeros(2, entries, dtype=torch.int32, device=DEV)
            o, lse = rv.paged_chunk_attention(values(gen(1), GIVEN[dtype], 2 * m, 4, 64), k, k, table, _i32([40, 96]), softmax_scale=0.1,
                                              **(sc if dtype == FP8 else {}))
            assert bool((o == 0).all()) and bool((lse == -INF).all())


def _bias(pool, n, cu, S, h, w, slots, seed, sigma, lam):
    """Correspondences of n queries, the slot table, and lambda B of every stream in float64."""
    rng = np.random.default_rng(seed)
    uv = (rng.uniform(-1, 1, (S, n, 2)) * (w, h) + (w / 2, h / 2)).astype(np.float32)
    idx = rng.integers(-4, 30, (S, n)).astype(np.int32)
    uv[idx < 0] = np.nan
    out = []
    for s, L in enumerate(pool.lens):
        a, b = (cu[s], cu[s + 1]) if cu is not None else (s * n // len(pool.lens), (s + 1) * n // len(pool.lens))
        frames = -(-L // (h * w))
        row = np.full(frames, -1, np.int32)
        m = min(frames, slots.shape[1])
        row[:m] = np.where(slots[s, :m] < S, slots[s, :m], -1)
        full = OA.bias_block(np.arange(b - a), frames * h * w, h, w, row, uv[:, a:b], idx[:, a:b], sigma)
        out.append(lam * full[:, :L])
    return torch.from_numpy(uv).to(DEV), torch.from_numpy(idx).to(DEV), out


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("h,w,Hq,Hk,D,lens,new,frames", [
    (8, 8, 2, 2, 128, [256], [64], 4), (5, 7, 4, 2, 64, [180, 70], [5, 35], 5), (1, 3, 1, 1, 64, [100], [2], 33), (13, 9, 2, 1, 128, [500], [117], 3),
    (30, 52, 1, 1, 128, [1560 * 2 + 11], [150], 2),
])
@pytest.mark.parametrize("seed", [10, 23])
def test_bias(dtype, h, w, Hq, Hk, D, lens, new, frames, seed):
    pool = Pool(9, dtype, lens, Hk, D, 32)
    cu = np.concatenate([[0], np.cumsum(new)])
    n, S = int(cu[-1]), 3
    rng = np.random.default_rng(seed)
    slots = rng.integers(-2, S + 2, (len(lens), frames)).astype(np.int32)  # beyond S: unbiased
    uv, idx, bias = _bias(pool, n, cu, S, h, w, slots, 11, 2.0, 1.3)
    q = values(gen(12), GIVEN[dtype], n, Hq, D)
    off_centre = np.nan_to_num(uv.cpu().numpy().astype(np.float64) - (w / 2, h / 2))
    largest = 1.3 * ((h * h + w * w) / 4 + (off_centre ** 2).sum(-1).max()) / (2 * 2.0 ** 2)
    slack = 0.0 if dtype == F32 else 8 * 2.0 ** -24 * largest
    for visible in (None, _causal(lens, cu)):
        o, lse = _attend(pool, q, cu, visible, kv_frame_slot=_i32(slots), corr_uv=uv, corr_idx=idx, h=h, w=w, lam=1.3, sigma=2.0)
        check_attention(pool, q, o, lse, cu, visible, bias=bias, slack=slack)
        off, _ = _attend(pool, q, cu, visible)
        assert torch.equal(off, o) == (not any(b.any() for b in bias))
    same, _ = _attend(pool, q, cu, visible, kv_frame_slot=_i32(slots), corr_uv=uv, corr_idx=idx, h=h, w=w, lam=0.0, sigma=2.0)
    assert torch.equal(same, off)


def test_agrees_with_the_dense_attention():
    """Pages of bf16 hold what biased_chunk_attention reads, the bias included: both are within two roundings of the same."""
    h, w, S, frames, H, D = 10, 12, 2, 6, 3, 128
    L, n = frames * h * w, 130
    pool = Pool(13, BF16, [L], H, D, 64)
    k, v, _ = pool.held(0)
    kd, vd = (torch.from_numpy(x.transpose(1, 0, 2).copy()).to(DEV).to(BF16) for x in (k, v))
    q = values(gen(14), BF16, n, H, D)
    slots = np.array([[-1, 0, 1, -1, 0, -1]], np.int32)
    uv, idx, _ = _bias(pool, n, None, S, h, w, slots, 15, 2.0, 1.0)
    want, wl = rv.biased_chunk_attention(q, kd, vd, _i32(slots[0]), uv, idx, h=h, w=w, softmax_scale=D ** -0.5, lam=1.0, sigma=2.0)
    o, lse = _attend(pool, q, kv_frame_slot=_i32(slots), corr_uv=uv, corr_idx=idx, h=h, w=w, lam=1.0, sigma=2.0)
    # each rounds its weights (2^-8; the dense one's sum too) and its output (2^-8)
    most = vd.float().abs().max()
    assert float((o.float() - want.float()).abs().max()) <= 5 * 2.0 ** -8 * float(most)
    assert float((lse - wl).abs().max()) <= 4e-3


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
def test_rows_of_nobody_and_strided_queries(dtype):
    lens, cu = [90, 33], [0, 2, 5]
    pool = Pool(16, dtype, lens, 2, 64, 32)
    rows = values(gen(17), GIVEN[dtype], 11, 3, 4, 64)
    q = rows[:, 1]
    out = torch.full((11, 4, 64), 7.0, dtype=GIVEN[dtype], device=DEV), torch.full((4, 11), 7.0, device=DEV)
    for parts in (1, 2):
        o, lse = _attend(pool, q, cu, out=out, key_parts=parts)
        assert o is out[0] and bool((o[5:] == 7).all()) and bool((lse[:, 5:] == 7).all())
        check_attention(pool, q[:5], o[:5], lse[:, :5].contiguous(), cu)


def test_many_streams_and_large_pools():
    """More streams than two waves have lanes, lengths beside the table's room, and a pool past 2^32 bytes."""
    B, H, D, page = 200, 40, 128, 256
    n_pages = (1 << 32) // (H * D * page) + 2
    rng = np.random.default_rng(18)
    ck, cv = (torch.empty(n_pages, H, page, D, dtype=FP8, device=DEV) for _ in range(2))
    sk, sv = (torch.full((n_pages, H, page // 32), 121, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu) for _ in range(2))
    pages = np.concatenate([[n_pages - 1, 0], rng.permutation(np.arange(1, n_pages - 1))[:40]])
    for c in (ck, cv):
        for p in pages:
            c[p] = (torch.randn(H, page, D, generator=gen(int(p)), device=DEV) * 64).clamp(-448, 448).to(FP8)
    table = pages[rng.integers(0, len(pages), (B, 2))].astype(np.int32)
    table[:3, 0] = n_pages - 1
    lens = rng.integers(1, 2 * page, B)
    lens[:4] = (1, 600, 512, -3)
    new = rng.integers(0, 3, B)
    new[:4] = 1
    cu = np.concatenate([[0], np.cumsum(new)])
    q = values(gen(19), BF16, int(cu[-1]), H, D)
    o, lse = rv.paged_chunk_attention(q, ck, cv, _i32(table), _i32(lens), cu=_i32(cu), scale_k=sk, scale_v=sv, softmax_scale=D ** -0.5)

    class Few:  # what three heads of six streams hold
        pass
    for s in (0, 1, 2, 3, 77, 199):
        L = int(np.clip(lens[s], 0, 2 * page))
        if cu[s + 1] == cu[s]:
            continue
        f = Few()
        f.lens, f.H, f.D = [L], H, D
        kv = [torch.cat([c[int(p)].float() for p in table[s]], 1)[:, :L].double().cpu().numpy() * 2.0 ** -6 for c in (ck, cv)]
        f.held = lambda _, kv=kv, L=L: (kv[0], kv[1], np.ones(L, bool))
        a, b = int(cu[s]), int(cu[s + 1])
        check_attention(f, q[a:b], o[a:b], lse[:, a:b].contiguous())


def test_extreme_logits():
    """Logits of +-10^4, and all of one size: the maximum that the sums go by is the row's own."""
    L, D = 200, 64
    pool = Pool(20, F32, [L], 1, D, 32)
    pool.k[:] = 0
    pool.k[..., 0] = torch.linspace(-1e5, 1e5, pool.k.shape[2], device=DEV)
    q = torch.zeros(3, 1, D, device=DEV)
    q[0, 0, 0], q[1, 0, 0] = 1.0, -1.0
    o, lse = _attend(pool, q)
    check_attention(pool, q, o, lse)


def test_refusals():
    pool = Pool(21, FP8, [64], 2, 64, 32)
    ck, cv, table, lens = pool.args()
    q = values(gen(22), BF16, 4, 4, 64)
    ok = dict(softmax_scale=0.125, **pool.kw())
    uv, idx = torch.zeros(1, 4, 2, device=DEV), torch.zeros(1, 4, dtype=torch.int32, device=DEV)
    bias = dict(corr_uv=uv, corr_idx=idx, kv_frame_slot=_i32([[0, 0]]), h=4, w=8, lam=1.0)
    rv.paged_chunk_attention(q, ck, cv, table, lens, **ok, **bias)
    for err, args, kw in [
        (TypeError, (q.float(), ck, cv, table, lens), ok), (ValueError, (q[:, :3], ck, cv, table, lens), ok), (ValueError, (q[..., :32], ck, cv, table, lens), ok),
        (ValueError, (q.cpu(), ck, cv, table, lens), ok), (ValueError, (q, ck, cv, table, lens[:0]), ok), (TypeError, (q, ck, cv, table.long(), lens), ok),
        (TypeError, (q, ck, cv, table, lens), {**ok, "scale_k": None}), (ValueError, (q, ck, cv, table, lens), {**ok, "visible": _i32([1])}),
        (rv.RevisitError, (q, ck, cv, table, lens), {**ok, "softmax_scale": 0.0}), (rv.RevisitError, (q, ck, cv, table, lens), {**ok, "key_parts": 65}),
        (rv.RevisitError, (q, ck, cv, table, lens), {**ok, "out": (q, None)}), (ValueError, (q, ck, cv, table, lens), {**ok, "cu": _i32([0])}),
        (rv.RevisitError, (q, ck, cv, table, lens), {**ok, "key_parts": 2, "workspace": torch.empty(16, dtype=torch.uint8, device=DEV)}),
        (ValueError, (q, ck, cv, table, lens), {**ok, **bias, "kv_frame_slot": _i32([0, 0])}), (rv.RevisitError, (q, ck, cv, table, lens), {**ok, **bias, "h": 0}),
        (rv.RevisitError, (q, ck, cv, table, lens), {**ok, **bias, "sigma": 0.0}), (ValueError, (q, ck, cv, table, lens), {**ok, **bias, "corr_idx": idx[:, :2]}),
    ]:
        with pytest.raises(err):
            rv.paged_chunk_attention(*args, **kw)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("D,Hq,Hk,m", [(64, 2, 1, 80), (128, 1, 1, 70), (128, 1, 1, 140), (128, 4, 1, 2)])
def test_long(dtype, D, Hq, Hk, m):
    """20000 keys, of which a query sees up to its own one."""
    L = 20000
    pool = Pool(23, dtype, [L], Hk, D, 64)
    q = values(gen(24), GIVEN[dtype], m, Hq, D)
    visible = np.linspace(1, L, m).astype(np.int32)
    for parts in (0, 1):
        o, lse = _attend(pool, q, None, visible, key_parts=parts)
        check_attention(pool, q, o, lse, None, visible)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("m", [3, 40, 150])
def test_bias_of_many_frames(dtype, m):
    """More retrieved frames than the kernels keep the correspondences of, and key frames of each of them."""
    h, w, S, D = 3, 11, 19, 64 if m == 40 else 128
    frames = 2 * S
    pool = Pool(25, dtype, [frames * h * w - 5], 1, D, 32)
    slots = np.random.default_rng(26).permutation(np.concatenate([np.arange(S), np.full(S, -1)]))[None].astype(np.int32)
    uv, idx, bias = _bias(pool, m, None, S, h, w, slots, 27, 2.0, 1.3)
    q = values(gen(28), GIVEN[dtype], m, 1, D)
    off_centre = np.nan_to_num(uv.cpu().numpy().astype(np.float64) - (w / 2, h / 2))
    largest = 1.3 * ((h * h + w * w) / 4 + (off_centre ** 2).sum(-1).max()) / (2 * 2.0 ** 2)
    o, lse = _attend(pool, q, kv_frame_slot=_i32(slots), corr_uv=uv, corr_idx=idx, h=h, w=w, lam=1.3, sigma=2.0)
    check_attention(pool, q, o, lse, bias=bias, slack=0.0 if dtype == F32 else 8 * 2.0 ** -24 * largest)


def test_bias_arguments_belong_together():
    """Slots or codes without correspondences would be a bias that is silently off."""
    pool = Pool(29, BF16, [64], 2, 64, 32)
    q = values(gen(30), BF16, 4, 2, 64)
    uv, idx, slot = torch.zeros(1, 4, 2, device=DEV), torch.zeros(1, 4, dtype=torch.int32, device=DEV), _i32([[0, 0]])
    for err, kw in [(ValueError, dict(kv_frame_slot=slot)), (ValueError, dict(corr_idx=idx)), (TypeError, dict(corr_uv=uv)),
                    (TypeError, dict(corr_uv=uv, corr_idx=idx)), (TypeError, dict(corr_uv=[0.0], corr_idx=idx, kv_frame_slot=slot))]:
        with pytest.raises(err):
            _attend(pool, q, h=4, w=8, lam=1.0, **kw)
