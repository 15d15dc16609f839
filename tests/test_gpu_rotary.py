"""rotary_embed against its fp64 oracle: types, head layouts, strided rows, bands that do not fill the head, given
and grid positions, the way back, and values that rounding or saturation would lose.

Tolerance. cos and sin: 2^-25 of rounding to fp32, 2e-9 of their Taylor sums, and 2^-52 of the angle; 4 units of 2^-24
are allowed (test_cos_and_sin holds them to what they are, to the ends of the positions' range). A product pair adds up
to two more, so the fp32 value is within 6 * 2^-24 (|x| + |y|) of the exact one. Rounding to bf16 adds half a step, 2^-8
of the value, to e4m3 2^-4 of it (2^-10 below its smallest normal number)."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from oracle import cache as OC

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA = 10000.0


def _bound(x, want, dtype, scale=1.0):
    """Allowed distance from want (unscaled) of pairs x [n, H, D] float64."""
    mag = np.abs(x[..., 0::2]) + np.abs(x[..., 1::2])
    tol = np.repeat(6 * 2.0 ** -24 * mag, 2, axis=-1) * scale
    if dtype == torch.bfloat16:
        tol = tol + np.abs(want) * 2.0 ** -8 + 2.0 ** -134
    elif dtype == torch.float8_e4m3fn:
        tol = tol + np.maximum(np.abs(want * scale) * 2.0 ** -4, 2.0 ** -10)
    return tol


def _check(got, x, pos, pairs, inverse=False, scale=1.0):
    x64 = x.double().cpu().numpy()
    want = OC.rotary(x64, pos, pairs, THETA, inverse)
    tol = _bound(x64, want, got.dtype, scale)
    aim = want * scale
    if got.dtype == torch.float8_e4m3fn:
        aim = np.clip(aim, -448.0, 448.0)
    off = np.abs(got.float().double().cpu().numpy() - aim)
    assert (off <= tol).all(), (off / tol).max()


def _rand(seed, dtype, *shape):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,Hq,Hk,D,pairs,h,w", [
    (1, 1, 1, 8, (2, 1, 1), 1, 1), (1, 12, 12, 128, (22, 21, 21), 1, 1), (7, 3, 1, 64, (12, 10, 10), 2, 3),
    (64, 1, 1, 64, (12, 10, 10), 8, 8), (255, 2, 5, 96, (16, 16, 16), 5, 17), (1560, 12, 4, 128, (22, 21, 21), 30, 52),
    (33, 5, 5, 128, (0, 0, 7), 4, 4), (40, 3, 3, 40, (5, 4, 3), 3, 5), (129, 1, 2, 512, (86, 85, 85), 6, 7), (1025, 1, 1, 8, (2, 2, 0), 5, 41),
    (300, 40, 40, 128, (22, 21, 21), 10, 10), (50, 2, 2, 128, (0, 0, 0), 5, 5),
])
def test_grid(dtype, n, Hq, Hk, D, pairs, h, w):
    q, k = _rand(1, dtype, n, Hq, D), _rand(2, dtype, n, Hk, D)
    qo, ko = rv.rotary_embed(q, k, pairs=pairs, theta=THETA, h=h, w=w, t0=5)
    pos = OC.grid_positions(n, 5, h, w)
    _check(qo, q, pos, pairs)
    _check(ko, k, pos, pairs)
    behind = 2 * sum(pairs)
    assert torch.equal(qo[..., behind:], q[..., behind:])  # copied


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_given_positions_and_the_way_back(dtype):
    n, H, D, pairs = 333, 6, 128, (22, 21, 21)
    rng = np.random.default_rng(3)
    pos = rng.integers(-100000, 1000000, (n, 3)).astype(np.int32)
    pos[0], pos[1] = 0, (1, -1, 7)
    at = torch.from_numpy(pos).to(DEV)
    q, k = _rand(4, dtype, n, H, D), _rand(5, dtype, n, H, D)
    for inverse in (False, True):
        qo, ko = rv.rotary_embed(q, k, pairs=pairs, theta=THETA, pos=at, inverse=inverse)
        _check(qo, q, pos, pairs, inverse)
        _check(ko, k, pos, pairs, inverse)
    # a token at the origin is not turned
    assert torch.equal(qo[0], q[0])
    # q alone, without k
    alone, none = rv.rotary_embed(q, pairs=pairs, theta=THETA, pos=at, inverse=True)
    assert none is None and torch.equal(alone, qo)


@pytest.mark.parametrize("theta", [10000.0, 256.0, 1.0])
def test_cos_and_sin(theta):
    """Pairs (1, 0) become (cos, sin) themselves. Near the origin, near frame counts, and to the ends of the positions'
    range, against angles in 80 bits: the Taylor sums' remainder (2e-9), one rounding to fp32 (half a step below 1: 2^-25)
    and 2^-52 of the angle (the rounded frequency and its product)."""
    D, n = 256, 3000
    pairs = (43, 43, 42)
    rng = np.random.default_rng(11)
    pos = np.concatenate([rng.integers(-200, 200, (n // 3, 3)), rng.integers(-2 ** 20, 2 ** 20, (n // 3, 3)),
                          rng.integers(-2 ** 31, 2 ** 31, (n // 3, 3))]).astype(np.int32)
    pos[-1], pos[-2] = 2 ** 31 - 1, -2 ** 31
    x = torch.zeros(n, 1, D, device=DEV)
    x[..., 0::2] = 1.0
    for inverse in (False, True):
        got = rv.rotary_embed(x, pairs=pairs, theta=theta, pos=torch.from_numpy(pos).to(DEV), inverse=inverse)[0].double().cpu().numpy()[:, 0]
        at = 0
        for axis, m in enumerate(pairs):
            omega = np.longdouble(theta) ** (-np.arange(m).astype(np.longdouble) / m)
            phi = pos[:, axis].astype(np.longdouble)[:, None] * omega
            tol = 2.0 ** -25 + 2e-9 + 2.0 ** -52 * np.abs(phi)
            si = -np.sin(phi) if inverse else np.sin(phi)
            assert (np.abs(got[:, 2 * at:2 * (at + m):2] - np.cos(phi)) <= tol).all()
            assert (np.abs(got[:, 2 * at + 1:2 * (at + m):2] - si) <= tol).all()
            at += m


def test_gradient_against_differences():
    """The way back is the gradient: a loss that is linear in the outputs, by differences of exact steps in fp32."""
    n, H, D, pairs = 6, 2, 16, (3, 2, 2)
    q, g = _rand(6, torch.float32, n, H, D), _rand(7, torch.float32, n, H, D)
    grad = rv.rotary_embed(g, pairs=pairs, theta=THETA, h=2, w=2, inverse=True)[0].double().cpu()
    step = torch.zeros(n * H * D, device=DEV)
    base = rv.rotary_embed(q, pairs=pairs, theta=THETA, h=2, w=2)[0].double()
    for i in range(0, n * H * D, 7):
        step.zero_()
        step[i] = 2.0 ** 10  # the outputs are linear in q: a large step, so that their rounding does not count
        moved = rv.rotary_embed(q + step.view(n, H, D), pairs=pairs, theta=THETA, h=2, w=2)[0].double()
        num = float(((moved - base) * g.double()).sum() / 2 ** 10)
        # two outputs change; each is within 6 * 2^-24 of 2^10 + a few, times |g| below 5
        assert abs(num - float(grad.view(-1)[i])) <= 2 * 6 * 2.0 ** -24 * 2 * 5 + 6 * 2.0 ** -24 * 10


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float8_e4m3fn)])
def test_packed_rows_into_cache_rows(dtype, out):
    """q and k read out of packed q, k, v rows; keys written into the rows of a cache that lie further apart."""
    n, H, D, pairs = 77, 3, 128, (22, 21, 21)
    rows = _rand(8, dtype, n, 3, H, D)
    cache = torch.zeros(n + 9, 2, H, D, device=DEV).to(out)
    q_out = torch.empty(n, H, D, dtype=out, device=DEV)
    k_out = cache[4:4 + n, 1]
    qo, ko = rv.rotary_embed(rows[:, 0], rows[:, 1], pairs=pairs, theta=THETA, h=7, w=11, out=(q_out, k_out), fp8_scale=(2.0, 0.5))
    assert qo is q_out and ko is k_out
    pos = OC.grid_positions(n, 0, 7, 11)
    fp8 = out == torch.float8_e4m3fn
    _check(q_out, rows[:, 0], pos, pairs, scale=2.0 if fp8 else 1.0)
    _check(k_out, rows[:, 1], pos, pairs, scale=0.5 if fp8 else 1.0)
    cache[4:4 + n, 1] = 0.0
    assert not cache.float().any()  # nothing else was written


def test_in_place():
    n, H, D, pairs = 130, 4, 64, (12, 10, 10)
    rows = _rand(9, torch.bfloat16, n, 3, H, D)
    want = rv.rotary_embed(rows[:, 0], rows[:, 1], pairs=pairs, theta=THETA, h=5, w=13)
    v = rows[:, 2].clone()
    rv.rotary_embed(rows[:, 0], rows[:, 1], pairs=pairs, theta=THETA, h=5, w=13, out=(rows[:, 0], rows[:, 1]))
    assert torch.equal(rows[:, 0], want[0]) and torch.equal(rows[:, 1], want[1]) and torch.equal(rows[:, 2], v)
    with pytest.raises(rv.RevisitError):  # another row distance in the same place
        rv.rotary_embed(rows.view(-1)[:n * H * D].view(n, H, D), pairs=pairs, theta=THETA, h=5, w=13, out=(rows[:, 0], None))


def test_fp8_values():
    """Rounding to nearest even, saturation at 448, small values, infinities and NaN, at an angle of 0."""
    vals = [0.0, -0.0, 1.0, 1.0625, 1.1875, -1.0625, 447.0, 448.0, 460.0, 1e4, -1e4, float("inf"), -float("inf"), float("nan"),
            2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -11, 17.0, 19.0, 240.0, 464.0, 3e38, 0.3]
    x = torch.tensor(vals, device=DEV).bfloat16().view(1, 1, 24)
    got = rv.rotary_embed(x, pairs=(0, 0, 0), theta=THETA, h=1, w=1, out_dtype=torch.float8_e4m3fn)[0].float().cpu().view(-1)
    want = x.float().cpu().view(-1).clamp(-448, 448).to(torch.float8_e4m3fn).float()
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


def test_far_strides():
    """Rows whose offsets pass 32 bits."""
    n, H, D, pairs = 3, 1, 128, (22, 21, 21)
    row = 1 << 30  # 4 GiB of bf16 between the first row and the last
    big = torch.zeros((n - 1) * row + H * D, dtype=torch.bfloat16, device=DEV)
    q = big.as_strided((n, H, D), (row, D, 1))
    q.copy_(_rand(10, torch.bfloat16, n, H, D))
    got, _ = rv.rotary_embed(q, pairs=pairs, theta=THETA, h=1, w=1, t0=3)
    _check(got, q, OC.grid_positions(n, 3, 1, 1), pairs)


def test_no_tokens():
    q = torch.empty(0, 2, 128, dtype=torch.bfloat16, device=DEV)
    qo, _ = rv.rotary_embed(q, pairs=(22, 21, 21), theta=THETA, h=1, w=1)
    assert qo.shape == q.shape
