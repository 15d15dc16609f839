"""The cache operators on launches of more than 2^32 threads (more than 2^22 workgroups of 256: rows of a grid) and on
arrays whose offsets pass 32 bits many times over."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def test_rotary_of_64_gib():
    """2^22 workgroups and some more move 16 KiB each, in place; the same tokens alone give the same bits."""
    H, D, pairs = 16, 128, (22, 21, 21)
    n = ((1 << 22) + 100) * 8192 // (H * D)  # 8192 elements a workgroup
    x = torch.zeros(n, H, D, dtype=torch.bfloat16, device=DEV)
    at = [0, 1, n // 3, n // 2 + 5, n - 2, n - 1]
    g = torch.Generator(device=DEV).manual_seed(1)
    rows = torch.randn(len(at), H, D, generator=g, device=DEV).bfloat16()
    pos = torch.tensor([[i // 1560, i % 1560 // 52, i % 52] for i in at], dtype=torch.int32, device=DEV)
    want, _ = rv.rotary_embed(rows, pairs=pairs, theta=1e4, pos=pos)
    for i, t in enumerate(at):
        x[t] = rows[i]
    rv.rotary_embed(x, pairs=pairs, theta=1e4, h=30, w=52, out=(x, None))
    for i, t in enumerate(at):
        assert torch.equal(x[t], want[i])
        x[t] = 0.0
    assert not any(c.any() for c in x.split(n // 16))


def test_scores_of_2_to_24_units():
    sets, units, unit = (1 << 14) + 3, 1024, 512
    w = torch.zeros(sets, 1, units * unit, device=DEV)
    chosen = [0, 77, 1 << 13, sets - 1]
    rng = np.random.default_rng(2)
    want = {}
    for s in chosen:
        u = np.sort(rng.choice(units, 5, replace=False))
        want[s] = u
        for i, x in enumerate(u):
            w[s, 0, int(x) * unit + 13 * i] = 1.0 + i
    idx, score = rv.select_kept(w, unit=unit, keep=5)
    for s in chosen:
        assert idx[s].tolist() == want[s].tolist() and sorted(score[s].tolist()) == [1.0, 2.0, 3.0, 4.0, 5.0]
    assert (idx[1] == torch.arange(5, device=DEV)).all() and not score[1].any()


def test_choice_from_2_to_30_units():
    """The largest set: 256 workgroups of 1024 blocks each; nearly all scores are equal, and the smaller units of them stay."""
    n, keep, last = 1 << 30, 100000, 50
    w = torch.zeros(1, 1, n, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(5)
    at = torch.randint(1 << 20, n - 1000, (70000,), generator=g, device=DEV).unique()
    w[0, 0, at] = 1.0 + torch.rand(len(at), generator=g, device=DEV)
    idx, score = rv.select_kept(w, unit=1, keep=keep, last=last)
    zeros = keep - last - len(at)
    want = torch.cat([torch.arange(zeros, device=DEV), at, torch.arange(n - last, n, device=DEV)]).int()
    assert torch.equal(idx[0], want) and torch.equal(score[0], w[0, 0, want.long()])


def test_move_of_64_gib():
    """One unit moved to more than 4096 places (repeats are allowed): 2^22 workgroups and some more."""
    H, D, unit = 16, 128, 4096  # 16 MiB a unit: 1024 workgroups
    k = torch.randn(1, 2 * unit, H, D, device=DEV).bfloat16()
    keep = 2060
    dst = [torch.zeros(1, keep * unit, H, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    sel = torch.ones(1, 1, keep, dtype=torch.int32, device=DEV)
    sel[0, 0, 1000] = 0
    rv.compact_kv(k, k, sel, *dst, unit=unit)
    for d in dst:
        for i in (0, 1, 999, 1000, 1001, keep - 1):
            u = 0 if i == 1000 else 1
            assert torch.equal(d[0, i * unit:(i + 1) * unit], k[0, u * unit:(u + 1) * unit])
