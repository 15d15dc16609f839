"""Pins of the paged cache's oracle: e4m3 rounding against torch's type, exponents against their definition, the
attention against its closed cases."""

from __future__ import annotations

import math

import numpy as np
import torch

from oracle import paged as OP


def test_e4m3_values_and_rounding():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(OP.E4M3.astype(np.float32), want, equal_nan=True)
    v = np.unique(want[np.isfinite(want)]).astype(np.float64)
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(np.inf)), np.nextafter(mid.astype(np.float32), np.float32(-np.inf)),
                        np.random.default_rng(0).uniform(-448, 448, 10000).astype(np.float32)]).astype(np.float32)
    got = torch.from_numpy(x).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(OP.round_e4m3(x).astype(np.float32), got)
    assert np.isnan(OP.round_e4m3(np.nan))


def test_exponent():
    for e in (-100, -99, -3, 0, 5, 119):
        for m in (448.0, 447.9, 224.1):
            assert OP.exponent(m * 2.0 ** e) == e
        assert OP.exponent(448.0 * 2.0 ** e * (1 + 2.0 ** -24)) == e + 1
    assert OP.exponent(0) == OP.exponent(1e-40) == OP.LOW
    assert OP.exponent(float(np.finfo(np.float32).max)) == 120


def test_append_places_and_drops():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    table = np.array([[3, 1], [0, -1]], np.int32)
    got, lens = OP.append(k, v, [0, 4, 7], [30, 62], table, 32, lambda i, c: (c, 0, 0), (4, 0, 0), 100.0, 4)
    assert lens == [34, 64]
    # stream 0: rows 30, 31 of page 3 and 0, 1 of page 1; stream 1: its second page is none
    assert sorted({(p, r) for p, _, r in got}) == [(1, 0), (1, 1), (3, 30), (3, 31)]
    assert np.array_equal(got[1, 1, 0][1], v[2, 1])
    phi = 32 * 100.0 ** (-np.arange(4) / 4)
    z = (k[2, 1, 0::2] + 1j * k[2, 1, 1::2]) * np.exp(1j * phi)
    assert np.allclose(got[1, 1, 0][0][0::2], z.real) and np.allclose(got[1, 1, 0][0][1::2], z.imag)


def test_attend_closed_cases():
    q, k, v = np.zeros((3, 2, 4)), np.zeros((1, 5, 4)), np.arange(20.0).reshape(1, 5, 4)
    vis = np.array([[1, 1, 1, 1, 1], [0, 0, 0, 0, 0], [0, 1, 0, 0, 0]], bool)
    o, lse = OP.attend(q, k, v, vis, 0.5)
    assert np.allclose(o[0], v[0].mean(0)) and np.allclose(lse[:, 0], math.log(5))
    assert (o[1] == 0).all() and (lse[:, 1] == -np.inf).all()
    assert np.allclose(o[2], v[0, 1]) and np.allclose(lse[:, 2], 0)
    bias = np.array([[0, 0, -1e9, -1e9, -1e9]] * 3)
    assert np.allclose(OP.attend(q, k, v, vis, 0.5, bias)[0][0], v[0, :2].mean(0))
