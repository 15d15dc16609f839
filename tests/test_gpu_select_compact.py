"""select_kept and compact_kv against their fp64 oracle. The choice is compared for equality (scores are sums in double
rounded once; test weights with ties are small whole numbers, whose sums are exact). Moved bytes are compared for
equality, turned keys within 6 * 2^-24 (|x| + |y|) of the exact value plus the storage type's half step."""

from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from oracle import cache as OC

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _choice(weight, **kw):
    idx, score = rv.select_kept(torch.from_numpy(weight).to(DEV), **kw)
    want, want_score = OC.select_kept(weight, kw["unit"], kw["keep"], kw.get("first", 0), kw.get("last", 0))
    assert np.array_equal(idx.cpu().numpy(), want)
    assert np.array_equal(score.cpu().numpy(), want_score, equal_nan=True)


@pytest.mark.parametrize("sets,heads,n,unit,keep,first,last", [
    (1, 1, 1, 1, 1, 0, 0), (1, 1, 1, 1, 1, 1, 0), (3, 2, 2, 3, 1, 0, 0), (30, 12, 18, 65, 12, 3, 6), (2, 1, 64, 1, 64, 5, 5),
    (5, 1, 1000, 1, 500, 100, 150), (2, 3, 1023, 1, 17, 0, 17), (4, 1, 1025, 1, 1024, 1, 0), (2, 1, 4096, 1, 1, 0, 0), (1, 12, 7, 1560, 3, 1, 1),
    (3, 1, 28081, 1, 9999, 1560, 3120), (2, 1, 70001, 1, 35000, 11, 13), (1, 1, 300007, 1, 1234, 0, 5), (2, 5, 40, 1, 20, 20, 0),
    (2, 1, 37, 2, 20, 0, 20), (7, 1, 2047, 1, 1000, 0, 0), (1, 2, 65537, 1, 65000, 0, 0),
    (3, 7, 4681, 1, 2000, 10, 20), (3, 8, 4097, 1, 2000, 10, 20), (2, 32, 64, 16, 9, 1, 1), (2, 31, 64, 17, 9, 1, 1), (2, 8, 64, 16, 9, 1, 1), (3, 1, 17, 480, 5, 0, 2), (5, 13, 630, 1, 300, 7, 7), (4, 40, 18, 40, 11, 0, 0), (1, 3, 63, 7, 62, 0, 1),
    (2, 40, 66, 3, 30, 4, 5), (1, 1, 33000, 1, 100, 0, 0), (1, 1, 32768, 1, 100, 0, 0), (1, 32768, 1, 1, 1, 0, 0), (2, 5, 65, 9, 64, 0, 0),
])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal"])
def test_choice(sets, heads, n, unit, keep, first, last, kind):
    rng = np.random.default_rng(n + keep)
    shape = (sets, heads, n * unit)
    if kind == "spread":
        weight = np.exp(1.5 * rng.standard_normal(shape)).astype(np.float32)
    elif kind == "ties":
        weight = rng.integers(0, 5, shape).astype(np.float32)
    else:
        weight = np.full(shape, 0.25, np.float32)
    _choice(weight, unit=unit, keep=keep, first=first, last=last)


def test_choice_of_special_values():
    rng = np.random.default_rng(0)
    vals = np.array([0.0, -0.0, 1.0, -1.0, math.inf, -math.inf, math.nan, 1e-45, -1e-45, 3e38, -3e38, 1e-38], np.float32)
    weight = rng.choice(vals, (6, 1, 3000)).astype(np.float32)
    weight[5] = math.nan
    for keep in (1, 100, 1500, 2900, 3000):
        _choice(weight, unit=1, keep=keep)
    pair = rng.choice(vals[:6], (4, 2, 200)).astype(np.float32)  # sums of infinities of both signs are NaN
    _choice(pair, unit=2, keep=40, first=3, last=2)
    _choice(np.full((1, 2, 6), 3e38, np.float32), unit=2, keep=2)  # the sum passes fp32: infinite


@pytest.mark.parametrize("sets,heads,n,unit,keep,first,last", [
    (1, 1, 32769, 1, 9000, 0, 0), (1, 1, 37440, 1, 20000, 1560, 4680), (28, 1, 37441, 1, 1, 0, 0), (60, 1, 70001, 1, 35000, 17, 0),
    (128, 1, 131073, 1, 65537, 1, 1), (129, 1, 131073, 1, 100, 1, 1), (1, 1, 1048577, 1, 300000, 0, 0), (1, 1, 2300001, 1, 1150000, 0, 70000),
    (1, 1, 1 << 21, 1, 1 << 21, 1, 0), (3, 2, 90001, 3, 40000, 5, 0), (1, 12, 37440, 1, 37439, 0, 0), (2, 1, 280800, 1, 280000, 200000, 80000),
    (1, 1, 65536, 1, 30, 10, 19), (1, 1, 65536, 1, 65535, 65535, 0), (1, 1, 65536, 1, 65536, 65536, 0),
])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "binade", "mostly zero"])
def test_choice_from_long_sets(sets, heads, n, unit, keep, first, last, kind):
    """Around the sizes where a set is shared out over workgroups, to several blocks in a share. Sets repeat
    after the second, so that the oracle has two to choose from."""
    rng = np.random.default_rng(n + keep)
    shape = (min(sets, 2), heads, n * unit)
    if kind == "spread":
        weight = np.exp(1.5 * rng.standard_normal(shape, np.float32))
    elif kind == "ties":
        weight = rng.integers(0, 5, shape).astype(np.float32)
    elif kind == "equal":
        weight = np.full(shape, 0.25, np.float32)
    elif kind == "binade":  # one bin of the first digit, so that all units are listed
        weight = rng.integers(1 << 20, (1 << 20) + (1 << 16), shape).astype(np.float32)
    else:
        weight = np.where(rng.random(shape, np.float32) < 0.01, 1.0 + rng.random(shape, np.float32), 0.0).astype(np.float32)
    of = np.arange(sets) % len(weight)
    idx, score = rv.select_kept(torch.from_numpy(weight).to(DEV)[torch.from_numpy(of).to(DEV)], unit=unit, keep=keep, first=first, last=last)
    want, want_score = OC.select_kept(weight, unit, keep, first, last)
    assert np.array_equal(idx.cpu().numpy(), want[of])
    assert np.array_equal(score.cpu().numpy(), want_score[of], equal_nan=True)


def test_choice_from_long_sets_in_a_graph():
    """Choice and move by token, captured once; every replay of new weights equals the eager calls."""
    H, D, n, keep = 2, 64, 50001, 20000
    w = torch.rand(1, H, n, device=DEV)
    kv = [torch.randn(1, n, H, D, device=DEV) for _ in range(2)]
    out = [torch.zeros(1, keep, H, D, device=DEV) for _ in range(2)]
    idx = (torch.zeros(H, keep, dtype=torch.int32, device=DEV), torch.zeros(H, keep, device=DEV))
    ws = torch.empty(rv.select_workspace_size(H, 1, n, 1), dtype=torch.uint8, device=DEV)

    def run():
        rv.select_kept(w.view(H, 1, n), unit=1, keep=keep, first=7, last=300, out=idx, workspace=ws)
        rv.compact_kv(*kv, idx[0].view(1, H, keep), *out, unit=1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for seed in range(4):
        w.copy_(torch.rand(1, H, n, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) ** (1 + 3 * seed))
        ws.fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*idx, *out)]
        run()
        assert all(torch.equal(a, b) for a, b in zip(got, (*idx, *out)))
        want, _ = OC.select_kept(w.view(H, 1, n).cpu().numpy(), 1, keep, 7, 300)
        assert np.array_equal(got[0].cpu().numpy(), want)


def test_choice_of_special_values_in_long_sets():
    rng = np.random.default_rng(3)
    vals = np.array([0.0, -0.0, 1.0, -1.0, math.inf, -math.inf, math.nan, 1e-45, -1e-45, 3e38, -3e38, 1e-38], np.float32)
    weight = rng.choice(vals, (3, 1, 90000)).astype(np.float32)
    weight[2] = math.nan
    for keep in (1, 20000, 60000, 89000, 90000):
        _choice(weight, unit=1, keep=keep, first=keep // 5)


def test_choice_without_scores_and_into_buffers():
    w = torch.rand(3, 2, 100, device=DEV)
    idx, score = rv.select_kept(w, unit=5, keep=8, first=1, last=2)
    out = (torch.full((3, 8), -9, dtype=torch.int32, device=DEV), None)
    got, none = rv.select_kept(w, unit=5, keep=8, first=1, last=2, out=out,
                               workspace=torch.empty(max(16, rv.select_workspace_size(3, 2, 20, 5)), dtype=torch.uint8, device=DEV))
    assert got is out[0] and none is None and torch.equal(got, idx)
    idx, score = rv.select_kept(w, unit=5, keep=0)
    assert idx.shape == (3, 0) and score.shape == (3, 0)
    with pytest.raises(rv.RevisitError):
        rv.select_kept(w, unit=5, keep=21)
    with pytest.raises(ValueError, match="whole number"):
        rv.select_kept(w, unit=7, keep=2)
    with pytest.raises(ValueError, match="contiguous"):
        rv.select_kept(w.transpose(0, 1), unit=5, keep=2)


def _kv(seed, dtype, *shape):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kdt, vdt = (torch.float8_e4m3fn, torch.bfloat16) if dtype == "fp8" else (dtype, dtype)
    return torch.randn(*shape, generator=g, device=DEV).to(kdt), torch.randn(*shape, generator=g, device=DEV).to(vdt)


def _host(t):
    return t.float().double().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, "fp8"])
@pytest.mark.parametrize("L,H,D,unit,units,keep,by_head,extra,row0", [
    (1, 1, 16, 1, 1, 1, False, 0, 0), (2, 3, 128, 6, 9, 4, False, 5, 7), (3, 2, 64, 1, 300, 111, True, 0, 0), (1, 12, 128, 35, 8, 8, False, 0, 3),
    (2, 5, 32, 7, 20, 13, True, 3, 1), (1, 2, 512, 3, 40, 21, True, 0, 0), (4, 1, 128, 390, 6, 2, False, 0, 0),
])
def test_move(dtype, L, H, D, unit, units, keep, by_head, extra, row0):
    rng = np.random.default_rng(keep)
    src = _kv(1, dtype, L, unit * units + extra, H, D)
    dst = _kv(2, dtype, L, row0 + unit * keep + 2, H, D)
    sel = np.stack([[np.sort(rng.choice(units, keep, replace=False)) for _ in range(H if by_head else 1)] for _ in range(L)]).astype(np.int32)
    sel[0, 0, 0] = rng.choice([-1, units, 2 ** 31 - 1])  # no such unit
    sel[-1, -1, -1] = sel[-1, -1, 0]  # one taken twice, out of order
    w, ow = torch.rand(L, H, unit * units, device=DEV), torch.rand(L, H, row0 + unit * keep + 3, device=DEV)
    want = [OC.compact(_host(s[:, :unit * units]), sel, unit, _host(d), row0) for s, d in zip(src, dst)]
    flat = lambda x: _host(x).transpose(0, 2, 1)[..., None]  # noqa: E731
    want_w = OC.compact(flat(w), sel, unit, flat(ow), row0)[..., 0].transpose(0, 2, 1)
    rv.compact_kv(*src, torch.from_numpy(sel).to(DEV), *dst, unit=unit, dst_row0=row0, weight=w, out_weight=ow)
    assert np.array_equal(_host(dst[0]), want[0]) and np.array_equal(_host(dst[1]), want[1]) and np.array_equal(_host(ow), want_w)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,D,unit,units,keep,by_head,n_t,fpu,given", [
    (2, 128, 6, 9, 5, False, 22, 1, False), (3, 64, 4, 12, 7, True, 12, 3, True), (1, 128, 1, 200, 90, True, 64, 1, True),
    (2, 40, 9, 5, 5, False, 7, 0, True), (12, 128, 30, 6, 4, False, 1, 2, False),
])
def test_move_with_turned_keys(dtype, H, D, unit, units, keep, by_head, n_t, fpu, given):
    rng = np.random.default_rng(keep)
    L, theta, dst_pos = 2, 10000.0, 4
    src, dst = _kv(3, dtype, L, unit * units, H, D), _kv(4, dtype, L, unit * keep, H, D)
    sel = np.stack([[np.sort(rng.choice(units, keep, replace=False)) for _ in range(H if by_head else 1)] for _ in range(L)]).astype(np.int32)
    pos = rng.integers(-5000, 100000, units).astype(np.int32)
    pos[sel[0, 0, 0]] = dst_pos  # this one stays where it was
    was = pos if given else np.arange(units) * fpu
    delta = dst_pos + np.arange(keep) * fpu - was[sel].astype(np.int64)
    want = OC.compact(_host(src[0]), sel, unit, _host(dst[0]), 0, delta, n_t, theta)
    plain = OC.compact(_host(src[0]), sel, unit, _host(dst[0]), 0)
    want_v = OC.compact(_host(src[1]), sel, unit, _host(dst[1]), 0)
    rv.compact_kv(*src, torch.from_numpy(sel).to(DEV), *dst, unit=unit, src_pos=torch.from_numpy(pos).to(DEV) if given else None,
                  dst_pos=dst_pos, frames_per_unit=fpu, rope_t_pairs=n_t, rope_theta=theta)
    got = _host(dst[0])
    mag = np.repeat(np.abs(plain[..., 0::2]) + np.abs(plain[..., 1::2]), 2, axis=-1)
    tol = 6 * 2.0 ** -24 * mag + (np.abs(want) * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    assert (np.abs(got - want) <= tol).all()
    assert np.array_equal(got[..., 2 * n_t:], plain[..., 2 * n_t:])  # not temporal: copied
    assert np.array_equal(_host(dst[1]), want_v)
    if given:
        assert np.array_equal(got[0, :unit, 0], plain[0, :unit, 0])  # did not move: copied


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,D,unit,n_t", [(12, 96, 30, 17), (12, 40, 47, 7), (5, 80, 60, 40), (3, 112, 73, 1), (1, 24, 1500, 5), (2, 8, 2100, 3), (7, 512, 9, 100)])
def test_move_of_large_units_with_turned_keys(dtype, H, D, unit, n_t):
    """Units of whole blocks that all heads share, at head sizes whose vectors do not divide a block: a thread's vectors lie in
    different places of a head; the last turned pair lies inside a vector."""
    rng = np.random.default_rng(D)
    L, units, keep, theta, fpu, dst_pos = 2, 5, 3, 10000.0, 1, 9
    assert unit * H * D * (2 if dtype == torch.bfloat16 else 4) // 16 >= 1024
    src, dst = _kv(8, dtype, L, unit * units, H, D), _kv(9, dtype, L, unit * keep + 1, H, D)
    after = [d[:, unit * keep:].clone() for d in dst]
    sel = np.stack([[np.sort(rng.choice(units, keep, replace=False))] for _ in range(L)]).astype(np.int32)
    delta = dst_pos + np.arange(keep) * fpu - sel.astype(np.int64) * fpu
    x = _host(src[0])
    want = OC.compact(x, sel, unit, _host(dst[0]), 0, delta, n_t, theta)
    plain = OC.compact(x, sel, unit, _host(dst[0]), 0)
    rv.compact_kv(*src, torch.from_numpy(sel).to(DEV), *dst, unit=unit, dst_pos=dst_pos, frames_per_unit=fpu, rope_t_pairs=n_t, rope_theta=theta)
    got = _host(dst[0])
    mag = np.repeat(np.abs(plain[..., 0::2]) + np.abs(plain[..., 1::2]), 2, axis=-1)
    tol = 6 * 2.0 ** -24 * mag + (np.abs(want) * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
    assert (np.abs(got - want)[:, :unit * keep] <= tol[:, :unit * keep]).all()
    assert np.array_equal(got[..., 2 * n_t:], plain[..., 2 * n_t:])
    assert np.array_equal(_host(dst[1])[:, :unit * keep], OC.compact(_host(src[1]), sel, unit, _host(dst[1]), 0)[:, :unit * keep])
    assert all(torch.equal(d[:, unit * keep:], a) for d, a in zip(dst, after))


def test_move_of_infinite_keys_that_stay():
    k, v = _kv(5, torch.bfloat16, 1, 4, 1, 128)
    k[0, 1] = math.inf
    k[0, 2] = math.nan
    dst = torch.zeros_like(k), torch.zeros_like(v)
    rv.compact_kv(k, v, torch.tensor([[[0, 1, 2, 3]]], dtype=torch.int32, device=DEV), *dst, unit=1, frames_per_unit=1, rope_t_pairs=22,
                  rope_theta=10000.0)
    assert torch.equal(dst[0].view(torch.int16), k.view(torch.int16))


def test_move_past_32_bits():
    """Source offsets past 2^32 bytes: three layers of a cache of 2.9 GB each, a few units of it moved."""
    L, H, D, unit, units = 3, 40, 128, 3600, 78
    src_k = torch.zeros(L, unit * units, H, D, dtype=torch.bfloat16, device=DEV)
    src_k[2, 77 * unit + 5] = _kv(6, torch.bfloat16, H, D)[0]
    dst = [torch.ones(L, unit, H, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    sel = torch.tensor([[[0]], [[1]], [[77]]], dtype=torch.int32, device=DEV)
    rv.compact_kv(src_k, src_k, sel, *dst, unit=unit)
    assert torch.equal(dst[0][2], src_k[2, 77 * unit:]) and torch.equal(dst[1][2], dst[0][2]) and not dst[0][:2].any()


def test_refusals():
    k, v = _kv(7, torch.bfloat16, 1, 12, 2, 128)
    sel = torch.zeros(1, 1, 3, dtype=torch.int32, device=DEV)
    with pytest.raises(rv.RevisitError, match="overlap"):
        rv.compact_kv(k, v, sel, k, torch.empty_like(v), unit=4)
    with pytest.raises(rv.RevisitError, match="dst_rows"):
        rv.compact_kv(k, v, sel, torch.empty_like(k), torch.empty_like(v), unit=4, dst_row0=1)
    with pytest.raises(ValueError, match="sel"):
        rv.compact_kv(k, v, sel.view(1, 3, 1), torch.empty_like(k), torch.empty_like(v), unit=4)
    k8 = k.to(torch.float8_e4m3fn)
    with pytest.raises(rv.RevisitError, match="fp8"):
        rv.compact_kv(k8, v, sel, torch.empty_like(k8), torch.empty_like(v), unit=4, rope_t_pairs=22, rope_theta=1e4)
