"""Oracle of the operators around the attention cache: rotary positions, the
weight of every key, the choice of kept units and their move.

TEST INFRASTRUCTURE ONLY. All arithmetic is float64 on the exact values of the
inputs; nothing is rounded to a storage type (a test compares within the
rounding it allows).

* rotary: pair j of a band of n pairs is the complex number x_{2i} + i x_{2i+1}
  times exp(i P theta^(-j / n)), P the token's position on the band's axis;
  bands of time, row and column in this order, pairs behind them untouched;
* weight: out = decay prev + sum_p exp(A_pk - LSE_p), A the biased logits
  of ``attention`` and queries without a finite LSE left out;
* choice: unit scores are sums in float64 rounded once to float32; the protected
  ends and the largest of the rest, the smaller unit first among equals, NaN
  below every number;
* move: dst[row0 + i unit + r] = src[sel[i] unit + r], the keys' temporal pairs
  turned by the unit's change of frame position.
"""

from __future__ import annotations

import numpy as np

from . import attention


def grid_positions(n, t0, h, w):
    """(time, row, column) of tokens 0..n-1 of a grid whose first frame is t0: [n, 3]."""
    r = np.arange(n)
    return np.stack([t0 + r // (h * w), r // w % h, r % w], axis=-1)


def rotary(x, pos, pairs, theta, inverse=False):
    """x [n, H, D] float64 embedded at pos [n, 3] (complex arithmetic)."""
    out = np.array(x, dtype=np.float64, copy=True)
    at = 0
    for axis, n in enumerate(pairs):
        if n == 0:
            continue
        omega = np.float64(theta) ** (-(np.arange(n) / np.float64(n)))
        phi = np.asarray(pos)[:, axis].astype(np.float64)[:, None] * omega
        turn = np.exp((-1j if inverse else 1j) * phi)[:, None, :]
        z = (out[..., 2 * at:2 * (at + n):2] + 1j * out[..., 2 * at + 1:2 * (at + n):2]) * turn
        out[..., 2 * at:2 * (at + n):2], out[..., 2 * at + 1:2 * (at + n):2] = z.real, z.imag
        at += n
    return out


def logits(q, k, slot, corr_uv, corr_idx, h, w, scale, lam, sigma):
    """Biased logits [H, Lq, Lk] in float64."""
    Lq, H, _ = q.shape
    Lk = k.shape[0]
    A = np.einsum("phd,khd->hpk", np.asarray(q, np.float64), np.asarray(k, np.float64)) * scale
    if corr_uv is not None and lam != 0:
        A += lam * attention.bias_block(np.arange(Lq), Lk, h, w, slot, corr_uv, corr_idx, sigma)[None]
    return A


def key_weight(A, lse, prev=None, decay=1.0):
    """Weights [H, Lk] of logits A [H, Lq, Lk] under lse [H, Lq]."""
    lse = np.asarray(lse, np.float64)
    ok = np.isfinite(lse)
    with np.errstate(invalid="ignore", over="ignore"):
        p = np.where(ok[:, :, None], np.exp(np.where(ok[:, :, None], A, 0.0) - np.where(ok, lse, 0.0)[:, :, None]), 0.0)
    out = p.sum(axis=1)
    return out if prev is None else out + np.float64(decay) * np.asarray(prev, np.float64)


def unit_scores(weight, unit):
    """Scores [sets, n_units] float32 of weights [sets, heads, n_units * unit]."""
    s, heads, cols = weight.shape
    with np.errstate(invalid="ignore", over="ignore"):
        return weight.astype(np.float64).reshape(s, heads, cols // unit, unit).sum(axis=(1, 3)).astype(np.float32)


def select_kept(weight, unit, keep, first, last):
    """Kept units [sets, keep] int32, ascending, and their scores."""
    score = unit_scores(weight, unit)
    n = score.shape[1]
    out = np.empty((score.shape[0], keep), np.int32)
    for i, row in enumerate(score):
        free = list(range(first, n - last))
        free.sort(key=lambda u: (0, -float(row[u]), u) if not np.isnan(row[u]) else (1, 0.0, u))
        out[i] = sorted([*range(first), *free[:keep - first - last], *range(n - last, n)])
    return out, np.take_along_axis(score, out.astype(np.int64), axis=1)


def compact(src, sel, unit, dst, row0, delta=None, n_t=0, theta=1.0):
    """dst [L, rows, H, D] float64 with the units sel [L, 1 or H, keep] of src moved in; with delta
    [L, sel heads, keep] the first n_t pairs turned by delta positions."""
    out = np.array(dst, dtype=np.float64, copy=True)
    L, _, H, _ = src.shape
    n_units = src.shape[1] // unit
    for layer in range(L):
        for hd in range(H):
            s = hd if sel.shape[1] > 1 else 0
            for i, u in enumerate(sel[layer, s]):
                if not 0 <= u < n_units:
                    continue
                x = np.asarray(src[layer, u * unit:(u + 1) * unit, hd], np.float64)
                if n_t:
                    pos = np.full((unit, 1), delta[layer, s, i])
                    x = rotary(x[:, None, :], pos, (n_t,), theta)[:, 0]
                out[layer, row0 + i * unit:row0 + (i + 1) * unit, hd] = x
    return out
