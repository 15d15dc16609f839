"""Pages of 8 bits at the ends of their scales: bytes that append_paged_kv itself does not write, values whose code times the
scale is past bf16's largest, NaN scales, in both operators and where a query must not see them.

Tolerances: codes and scales equal to their definition; attention as check_attention derives it."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from oracle import paged as OP
from tests.paged_helpers import BF16, DEV, FP8, Pool, check_attention, gen, values

pytestmark = pytest.mark.gpu
E8M0 = torch.float8_e8m0fnu
NAN, INF = float("nan"), float("inf")


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _byte(s):
    return s.view(torch.uint8)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("byte", [0, 1, 26, 27, 120, 246, 247, 248, 250, 254, 255])
@pytest.mark.parametrize("top", [0.0, 1.0, 2.0 ** 100, 3.0e38])
def test_append_behind_a_stored_scale(D, byte, top):
    """Rows that go to a block which holds some: its scale only grows, and held values stay what they are up to the rounding to
    it. A NaN scale stays, and so does all that the block holds and gets."""
    H, page, held, new = 2, 64, 13, 7
    pool = Pool(1, FP8, [held + new], H, D, page)
    p = int(pool.table[0, 0])
    for s in pool.scales:
        _byte(s)[p, :, 0] = byte
    code = torch.arange(D * held, device=DEV).view(held, D).to(torch.uint8)  # every code
    for c in (pool.k, pool.v):
        _byte(c)[p, :, :held] = code
    was = [_byte(x).clone() for x in (pool.k, pool.v, *pool.scales)]
    x = values(gen(2), BF16, new, H, D).clamp(-1, 1)
    x[0, :, 0] = 1.0
    x = (x.double() * top).to(BF16)
    ck, cv, table, _ = pool.args()
    rv.append_paged_kv(x, x, ck, cv, table, _i32([held]), pairs=(0, 0, 0), theta=10000.0, h=1, w=1, **pool.kw())
    e_new = OP.exponent(float(x.double().abs().max()))
    for i, (cache, scale) in enumerate(((ck, pool.scales[0]), (cv, pool.scales[1]))):
        got, old = cache[p].float().double().cpu().numpy(), torch.empty_like(cache)
        _byte(old).copy_(was[i])
        old = old[p].float().double().cpu().numpy()
        e_old = max(byte, 1) - 127
        if byte == 255:
            assert bool((_byte(scale)[p, :, 0] == 255).all())
            assert torch.equal(_byte(cache)[p, :, :held], was[i][p, :, :held])
            assert np.isnan(got[:, held:held + new]).all()
        elif e_new <= e_old:
            assert bool((_byte(scale)[p, :, 0] == byte).all()), _byte(scale)[p, :, 0]
            assert torch.equal(_byte(cache)[p, :, :held], was[i][p, :, :held])
            e = e_old
        else:
            assert bool((_byte(scale)[p, :, 0] == e_new + 127).all())
            assert np.array_equal(got[:, :held], OP.round_e4m3(old[:, :held] * 2.0 ** (e_old - e_new)), equal_nan=True)
            e = e_new
        if byte != 255:
            want = OP.round_e4m3(x.double().cpu().numpy().transpose(1, 0, 2) * 2.0 ** -e)
            assert np.array_equal(got[:, held:held + new], want)
        # the rest of the page
        assert torch.equal(_byte(cache)[p, :, held + new:], was[i][p, :, held + new:])
        assert torch.equal(_byte(scale)[p, :, 1:], was[2 + i][p, :, 1:])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("held", [0, 9])
def test_append_largest_values(D, held):
    """Finite values whose nearest code would stand for 2^128: the largest code that stands for a bf16 value instead, less than
    half a step of e4m3 (2^-4 of the value) away. What is read back is finite."""
    H, page, new = 2, 32, 6
    x = torch.zeros(new, H, D, dtype=BF16, device=DEV)
    top = torch.finfo(BF16).max
    x[0, 0, :6] = torch.tensor([top, -top, 3.3e38, -3.3e38, 3.2e38, 1.0])
    x[5, 1, -1] = -top
    pool = Pool(3, FP8, [held + new], H, D, page)
    p = int(pool.table[0, 0])
    for byte in (1, 247, 250, 254):
        for s in pool.scales:
            _byte(s)[p, :, 0] = byte
        ck, cv, table, _ = pool.args()
        rv.append_paged_kv(x, x, ck, cv, table, _i32([held]), pairs=(0, 0, 0), theta=10000.0, h=1, w=1, **pool.kw())
        for cache, scale in ((ck, pool.scales[0]), (cv, pool.scales[1])):
            b = _byte(scale)[p, :, 0].tolist()
            least = [247, 247] if held == 0 else [max(byte, 247)] * 2
            assert b == least
            back = cache[p, :, held:held + new].double() * torch.exp2(torch.tensor(b, device=DEV).double() - 127)[:, None, None]
            want = x.double().transpose(0, 1)
            assert bool(((back - want).abs() <= want.abs() * 2.0 ** -4 + 2.0 ** -10 * 2.0 ** (max(b) - 127)).all())
            assert float(back.abs().max()) == 1.875 * 2.0 ** 127
    # turned keys: by half a turn of the second pair, in fp32
    k = torch.zeros(new, H, D, dtype=BF16, device=DEV)
    k[..., 2], k[..., 3] = top, 1.0
    pos = torch.zeros(new, 3, dtype=torch.int32, device=DEV)
    pos[1::2, 0] = 1
    rv.append_paged_kv(k, k, *pool.args()[:3], _i32([0]), pairs=(2, 0, 0), theta=float(np.float32(np.pi) ** -2), pos=pos, **pool.kw())
    assert bool((pool.k[p, :, :new, 2].float().abs() == 240).all()) and _byte(pool.scales[0])[p, :, 0].tolist() == [247, 247]


@pytest.fixture(params=[0, 1 << 19], ids=["table", "wide_table"])
def room(request, monkeypatch):
    """Page tables with just the entries that the streams need, and far wider ones, for which other kernels are chosen."""
    monkeypatch.setattr(Pool, "room", request.param)


class Stored(Pool):
    """What the pages hold by their definition: byte 0 counts as 1, and 2^128 and more is infinite."""

    def held(self, s):
        k, v, have = super().held(s)
        return tuple(np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x) for x in (k, v)) + (have,)


def _attend(pool, q, visible=None, **kw):
    return rv.paged_chunk_attention(q, *pool.args(), visible=None if visible is None else _i32(visible), softmax_scale=q.shape[-1] ** -0.5, **pool.kw(), **kw)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 17, 40, 150])
@pytest.mark.parametrize("byte", [247, 248, 251, 254, 255])
def test_values_past_the_largest_that_are_not_seen(room, D, m, byte):
    """Codes whose value, with the block's scale, is infinite or NaN, at positions that only some queries see."""
    L, H, page = 170, 2, 64
    pool = Stored(5, FP8, [L], H, D, page)
    q = values(gen(6), BF16, m, H, D)
    visible = np.arange(L - m, L) + 1
    if m == 1:
        visible[:] = 150
    t = pool.table[0]
    least = 2.0 ** (255 - min(byte, 254))  # the least code value that is infinite: 256 for 247, 2 for 254
    for blk, at in ((128 // 32, (155, 156)), (160 // 32, (168, 169))):
        p, row = t[blk * 32 // page], blk * 32 % page
        pool.v[p, :, row:row + 32] = 0  # a sum that holds values near the largest may pass it
        _byte(pool.scales[1])[p, :, row // 32] = byte
        for j, c in enumerate(at):
            pool.v[p, j % 2, c % page, 3 * j:3 * j + 4] = torch.tensor([least, -least, min(448.0, 1.75 * least), least], device=DEV).to(FP8)
            if byte == 247:
                pool.v[p, :, c % page, 20:24] = torch.tensor([2.0 ** -9, -2.0 ** -9, 0.0, -0.0], device=DEV).to(FP8)
    o, lse = _attend(pool, q, visible)
    blind = np.flatnonzero(visible <= (128 if byte == 255 else 155))
    if len(blind):
        assert bool(torch.isfinite(o[blind[0]:blind[-1] + 1]).all())
    assert bool(torch.isfinite(lse).all())
    check_attention(pool, q, o, lse, None, visible)
    if m == 1:  # every query sees them all
        o, lse = _attend(pool, q)
        check_attention(pool, q, o, lse)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 17, 40, 150])
def test_nan_scales(room, D, m):
    """Blocks of keys and values whose scale is NaN: what sees a key of one has a NaN logit, what does not is as without it."""
    L, H, page = 200, 2, 32
    pool = Stored(7, FP8, [L], H, D, page)
    q = values(gen(8), BF16, m, H, D)
    visible = np.linspace(100, L, m).astype(int)
    if m == 1:
        visible[:] = 159
    _byte(pool.scales[0])[pool.table[0, 5], 1, 0] = 255  # keys 160 .. 191 of head 1
    _byte(pool.scales[1])[pool.table[0, 6], 0, 0] = 255  # values 192 .. of head 0
    o, lse = _attend(pool, q, visible)
    blind = np.flatnonzero(visible <= 160)
    seeing = np.flatnonzero(visible > 160)
    sub = slice(int(blind[0]), int(blind[-1]) + 1)
    assert bool(torch.isfinite(o[sub]).all())
    check_attention(pool, q[sub], o[sub], lse[:, sub].contiguous(), None, visible[sub])
    for p in seeing:
        assert bool(torch.isnan(o[p, 1]).all()) and bool(torch.isnan(lse[1, p]))
        assert bool(torch.isnan(o[p, 0]).all()) == (visible[p] > 192) and bool(torch.isfinite(lse[0, p]))
    # head 0 has no NaN logit
    one = Stored(7, FP8, [L], 1, D, page)
    one.table, one.n_pages = pool.table, pool.n_pages
    one.k, one.v = pool.k[:, :1], pool.v[:, :1]
    one.scales = [_byte(s)[:, :1].contiguous().view(E8M0) for s in pool.scales]
    check_attention(one, q[:, :1], o[:, :1], lse[:1], None, visible)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 17, 40, 150])
def test_scales_of_any_size(room, D, m):
    """A scale is a power of two: values under other ones give the same times their ratio, bit for bit. Byte 0 counts as 1."""
    L, page = 300, 64
    pool = Pool(9, FP8, [L], 2, D, page)
    q = values(gen(10), BF16, m, 2, D)
    got = {}
    for byte in (0, 1, 60, 127, 180):
        _byte(pool.scales[1])[:] = byte
        o, lse = _attend(pool, q)
        got[byte] = o.double()
        if byte == 127:
            check_attention(pool, q, o, lse)
    for byte in (60, 180):
        assert torch.equal(got[byte] * 2.0 ** (127 - byte), got[127])
    assert torch.equal(got[0], got[1])
    for byte, other in ((0, 1), (90, 127)):
        o = []
        for b in (byte, other):
            _byte(pool.scales[0])[:] = b
            _byte(pool.scales[1])[:] = 127
            o.append(rv.paged_chunk_attention(q, *pool.args(), softmax_scale=D ** -0.5 * 2.0 ** ((127 - b) if byte else 100), **pool.kw()))
        assert torch.equal(o[0][0], o[1][0]) and torch.equal(o[0][1], o[1][1])


@pytest.mark.parametrize("dtype", [FP8, BF16, torch.float32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("m", [1, 16, 17, 40, 150])
def test_infinite_values_that_all_see(room, dtype, D, m):
    """An infinity among the values of keys that every query of the tile sees is the output's, with its sign."""
    L, H, page = 160, 2, 32
    pool = Stored(11, dtype, [L], H, D, page)
    q = values(gen(12), {FP8: BF16}.get(dtype, dtype), m, H, D)
    p = pool.table[0, 2]
    if dtype == FP8:
        pool.v[p] = 0
        pool.v[p, :, 5, 3:5] = torch.tensor([256.0, -256.0], device=DEV).to(FP8)
        _byte(pool.scales[1])[p] = 247
    else:
        pool.v[p, :, 5, 3:5] = torch.tensor([INF, -INF], device=DEV).to(dtype)
    o, lse = _attend(pool, q)
    assert bool((o[..., 3] == INF).all()) and bool((o[..., 4] == -INF).all())
    check_attention(pool, q, o, lse)
