"""Pins of the oracle of the cache operators: relative positions and the inverse of the rotary embedding, its
agreement with the packing oracle's temporal turn, weights that add up to the queries, the choice against a
plain loop, the move against indexing."""

from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import attention as OA
from oracle import cache as OC
from oracle import kvpack as OK


def test_rotary_scores_depend_on_relative_positions():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 48))
    a, b, d = np.array([[5, 2, 7]]), np.array([[1, 9, 3]]), np.array([[40, -6, 11]])
    dot = lambda x, y: float((OC.rotary(q, x, (10, 8, 6), 100.0) * OC.rotary(k, y, (10, 8, 6), 100.0)).sum())  # noqa: E731
    assert dot(a, b) == pytest.approx(dot(a + d, b + d), abs=1e-12)
    assert abs(dot(a, b) - dot(a + d, b)) > 1e-3


def test_rotary_inverse_is_the_transpose():
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 6, 3, 32))
    pos = rng.integers(-50, 50, (6, 3))
    args = (pos, (6, 5, 3), 10000.0)
    assert np.allclose(OC.rotary(OC.rotary(x, *args), *args, inverse=True), x, atol=1e-12)
    # <R x, y> = <x, R^T y>
    assert (OC.rotary(x, *args) * y).sum() == pytest.approx((x * OC.rotary(y, *args, inverse=True)).sum(), abs=1e-10)


def test_rotary_gradient_by_differences():
    rng = np.random.default_rng(2)
    x, g = rng.standard_normal((2, 2, 1, 12))
    pos = rng.integers(0, 9, (2, 3))
    args = (pos, (2, 2, 1), 50.0)
    grad = OC.rotary(g, *args, inverse=True)
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = 1e-4
        num = ((OC.rotary(x + d, *args) - OC.rotary(x - d, *args)) * g).sum() / 2e-4
        assert num == pytest.approx(grad[i], abs=1e-8)


def test_rotary_time_band_is_the_packing_turn():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 2, 16))
    pos = np.stack([np.full(4, 7), np.arange(4), np.arange(4)], 1)
    at7 = OC.rotary(x, pos, (3, 3, 2), 10000.0)
    moved = OK.rotate_temporal(at7, 5, 3, 10000.0)
    pos[:, 0] += 5
    assert np.allclose(moved, OC.rotary(x, pos, (3, 3, 2), 10000.0), atol=1e-12)


def test_grid_positions():
    p = OC.grid_positions(14, 3, 2, 3)
    assert p[0].tolist() == [3, 0, 0] and p[5].tolist() == [3, 1, 2] and p[6].tolist() == [4, 0, 0] and p[13].tolist() == [5, 0, 1]


def test_weights_add_up_to_the_queries():
    rng = np.random.default_rng(4)
    h, w, S, Lq, H, D = 3, 4, 2, 10, 2, 8
    Lk = 4 * h * w
    q, k, v = rng.standard_normal((Lq, H, D)), rng.standard_normal((Lk, H, D)), rng.standard_normal((Lk, H, D))
    slot = np.array([-1, 1, 0, -1], np.int32)
    uv, idx = (rng.random((S, Lq, 2)) * [w, h]).astype(np.float32), rng.integers(-2, h * w, (S, Lq)).astype(np.int32)
    A = OC.logits(q, k, slot, uv, idx, h, w, 1 / math.sqrt(D), 1.0, 2.0)
    _, lse = OA.biased_attention(q, k, v, slot, uv, idx, h, w, 1 / math.sqrt(D), 1.0, 2.0)
    W = OC.key_weight(A, lse)
    # the oracle's LSE (below 8) is rounded to fp32: a query's weights add up to 1 within 2^-22
    near = Lq * 2.0 ** -22
    assert W.sum(axis=1) == pytest.approx([Lq] * H, abs=near)
    lse = np.array(lse)
    lse[0, 3], lse[1, :2] = np.nan, [np.inf, -np.inf]
    W = OC.key_weight(A, lse, prev=np.ones((H, Lk)), decay=0.5)
    assert W.sum(axis=1) == pytest.approx([Lq - 1 + Lk / 2, Lq - 2 + Lk / 2], abs=near)


def test_choice_by_a_plain_loop():
    rng = np.random.default_rng(5)
    weight = rng.integers(0, 4, (3, 2, 24)).astype(np.float32)
    weight[1, 0, 9] = np.nan
    idx, score = OC.select_kept(weight, 2, 7, 2, 3)
    for s in range(3):
        total = [sum(float(weight[s, h, 2 * u + i]) for h in range(2) for i in range(2)) for u in range(12)]
        left, kept = set(range(2, 9)), [0, 1, 9, 10, 11]
        for _ in range(2):
            best = None
            for u in sorted(left):
                if math.isnan(total[u]):
                    continue
                if best is None or total[u] > total[best]:
                    best = u
            kept.append(best)
            left.discard(best)
        assert idx[s].tolist() == sorted(kept)
        assert np.array_equal(score[s], np.float32([total[u] for u in idx[s]]), equal_nan=True)


def test_move_by_indexing():
    rng = np.random.default_rng(6)
    src, dst = rng.standard_normal((2, 12, 3, 8)), np.zeros((2, 7, 3, 8))
    sel = np.array([[[3, 0]], [[2, 9]]])
    got = OC.compact(src, sel, 3, dst, 1)
    assert np.array_equal(got[0, 1:4], src[0, 9:12]) and np.array_equal(got[0, 4:7], src[0, :3])
    assert np.array_equal(got[1, 1:4], src[1, 6:9]) and not got[1, 4:7].any() and not got[:, 0].any()
