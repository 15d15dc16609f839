"""What the tolerances of the other tests of paged_chunk_attention leave open: two numbers for each probability of up to 16 rows,
and the bias over ranges longer than the kernels keep tables of."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import paged as OP
from tests.paged_helpers import BF16, F32, FP8, GIVEN, Pool, check_attention, gen, values
from tests.test_gpu_paged_attention import _attend, _bias, _i32

pytestmark = pytest.mark.gpu


def _bf16(x):
    return torch.from_numpy(x).to(BF16).double().numpy()


@pytest.mark.parametrize("dtype", [FP8, BF16])
@pytest.mark.parametrize("D,Hq,Hk,lens,m", [(64, 2, 2, [5], 1), (128, 2, 2, [40, 7], 1), (128, 8, 1, [300], 2), (64, 4, 2, [90, 33], 8), (128, 1, 1, [900], 16)])
@pytest.mark.parametrize("parts", [0, 1, 2])
def test_probabilities_of_few_rows(dtype, D, Hq, Hk, lens, m, parts):
    """Up to 16 rows: the sum over keys keeps a probability within 2^-16 of itself. Heavy keys whose values are +-1 cancel in
    the output, so that its own rounding (half a step, 2^-8 of it) is smaller than what one bf16 number would leave of them.

    Bound: a logit within D + 6 units of 2^-24 of its terms' magnitudes, the exponential within 2^-22, the rest of the
    sums L + 16 units; a probability as two bf16 numbers: 2^-8 2^-8."""
    pool = Pool(1, dtype, lens, Hk, D, 32)
    g = gen(2)
    sign = torch.randint(0, 2, pool.v.shape, generator=g, device=pool.v.device) * 2.0 - 1.0
    pool.v = sign.to(dtype)
    if dtype == FP8:
        for s in pool.scales:
            s.view(torch.uint8).fill_(127)
        pool.k = values(g, torch.float32, *pool.k.shape).to(dtype)
    else:
        pool.k = values(g, dtype, *pool.k.shape)
    n = len(lens) * m
    q = values(g, BF16, n, Hq, D) * 0.5
    o, _ = _attend(pool, q, key_parts=parts)
    got, q64 = o.double().cpu().numpy(), q.double().cpu().numpy()
    one_number = 0
    for s, (t0, rows) in enumerate(OP.streams(n, None, len(lens))):
        k, v, _ = pool.held(s)
        L = lens[s]
        for h in range(Hq):
            kk, vv = k[h // (Hq // Hk)], v[h // (Hq // Hk)]
            a = q64[t0:t0 + rows, h] @ kk.T * D ** -0.5
            d = (D + 6) * 2.0 ** -24 * (np.abs(q64[t0:t0 + rows, h]) @ np.abs(kk).T * D ** -0.5).max(1) + 2.0 ** -22
            p = np.exp(a - a.max(1, keepdims=True))
            want = p @ vv / p.sum(1, keepdims=True)
            tol = 2 * d[:, None] + 2.0 ** -16 + 2 * (L + 16) * 2.0 ** -24 + 2.0 ** -8 * np.abs(want)
            assert (np.abs(got[t0:t0 + rows, h] - want) <= tol).all(), (s, h, (np.abs(got[t0:t0 + rows, h] - want) / tol).max())
            one_number += (np.abs(_bf16(p) @ vv / p.sum(1, keepdims=True) - want) > tol).sum()
    # A probability rounded to one bf16 number would be found out, but not among many keys alike: of 900 such roundings
    # 2^-9 / sqrt(3 * 900) = 4e-5 is left, less than the logits' part of the bound.
    assert one_number > 0 or max(lens) > 300


def _biased(dtype, D, m, h, w, frames, S, seed, parts=0, page=64):
    pool = Pool(seed, dtype, [frames * h * w - 5], 1, D, page)
    rng = np.random.default_rng(seed)
    slots = rng.integers(-S, S, (1, frames)).astype(np.int32)  # half of the frames retrieved
    uv, idx, bias = _bias(pool, m, None, S, h, w, slots, seed + 1, 2.0, 1.3)
    q = values(gen(seed + 2), GIVEN[dtype], m, 1, D)
    off_centre = np.nan_to_num(uv.cpu().numpy().astype(np.float64) - (w / 2, h / 2))
    largest = 1.3 * ((h * h + w * w) / 4 + (off_centre ** 2).sum(-1).max()) / (2 * 2.0 ** 2)
    o, lse = _attend(pool, q, kv_frame_slot=_i32(slots), corr_uv=uv, corr_idx=idx, h=h, w=w, lam=1.3, sigma=2.0, key_parts=parts)
    # the separable form's slack as in the other tests of the bias
    check_attention(pool, q, o, lse, bias=bias, slack=0.0 if dtype == F32 else 8 * 2.0 ** -24 * largest)


@pytest.mark.parametrize("dtype", [FP8, BF16])
@pytest.mark.parametrize("D,m", [(128, 150), (128, 100), (64, 80)])
@pytest.mark.parametrize("wide", [False, True])
def test_bias_past_the_tables_of_a_tile_kernel(dtype, D, m, wide, monkeypatch):
    """171 frames of 9 x 13 tokens, 626 tiles in one part: the tables of 512 tiles wrap, and frames end within tiles everywhere."""
    monkeypatch.setattr(Pool, "room", (1 << 19) if wide else 0)
    _biased(dtype, D, m, 9, 13, 171, 3, 40, parts=1)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("m", [3, 20])
@pytest.mark.parametrize("parts", [1, 5])
def test_bias_of_more_frames_than_are_kept(dtype, m, parts):
    """300 frames of 3 x 11 tokens: slots from frame 256 on come from memory; 20 correspondences, 16 of them kept."""
    _biased(dtype, 128 if m == 3 else 64, m, 3, 11, 300, 20, 50, parts=parts, page=32)
