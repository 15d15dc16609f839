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
