"""Oracle of the paged cache: what append_paged_kv stores and what paged_chunk_attention makes of it.

TEST INFRASTRUCTURE ONLY. float64 on the exact values of the inputs, one position at a time; nothing is rounded
but where the cache's definition rounds (the codes and scales of 8-bit pages).

* position c of stream s lies in row c mod page of page table[s][c // page], if that is a page;
* scales: of the 32 positions of a block, per head, 2^e with the least e >= -100 that brings the largest finite new
  value to 448 2^e or below, never below the stored e where the block held positions of the stream;
* codes: the nearest e4m3 value of x 2^-e, ties to even, of those that stand for less than 2^128; NaN where x is not finite;
* attention: softmax over the keys below min(length, visible) that have a page, biased in retrieved frames.
"""

from __future__ import annotations

import math

import numpy as np

from . import cache as OC

BLOCK, LOW = 32, -100


def _e4m3_values():
    v = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        v[b] = (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if b & 128 else 1)
    v[0x7f] = v[0xff] = np.nan
    return v


E4M3 = _e4m3_values()


def round_e4m3(x):
    """Nearest e4m3 value, ties to the even mantissa, |x| <= 448 (beyond by less than half a step too); NaN stays."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.clip(np.floor(np.log2(np.where(a > 0, a, 1.0))), -6, 8)
    step = 2.0 ** (e - 3)
    return np.copysign(np.rint(a / step) * step, x)


def exponent(m):
    """Least integer e >= LOW with m <= 448 * 2^e."""
    if m == 0:
        return LOW
    e = max(LOW, math.frexp(m)[1] - 10)
    while m > 448 * 2.0 ** e:
        e += 1
    return e


def streams(n, cu, B):
    """(first token, tokens) of every stream."""
    return [(s * (n // B), n // B) for s in range(B)] if cu is None else [(int(cu[s]), int(cu[s + 1] - cu[s])) for s in range(B)]


def append(k, v, cu, kv_len, table, page, pos, pairs, theta, n_pages):
    """{(page, head, row): (key, value)} in float64, unrounded, of everything that is stored, and the new lengths.
    pos: a function of (token, position) to (time, row, column)."""
    n, H, _ = k.shape
    B, max_pages = table.shape
    got, lens = {}, []
    cap = max_pages * page
    for s, (t0, m) in enumerate(streams(n, cu, B)):
        held = min(max(int(kv_len[s]), 0), cap)
        lens.append(min(held + m, cap))
        for i in range(t0, t0 + m):
            c = held + i - t0
            if c >= cap or not 0 <= table[s, c // page] < n_pages:
                continue
            at = np.array([pos(i, c)], np.float64)
            kk = OC.rotary(k[i:i + 1], at, pairs, theta)[0]
            for h in range(H):
                got[int(table[s, c // page]), h, c % page] = (kk[h], v[i, h])
    return got, lens


def attend(q, k, v, visible, scale, bias=None):
    """One stream's attention. q [m, Hq, D], k, v [Hk, L, D] float64 (rows of no page NaN-free and listed in
    `visible`), visible [m, L] bool, bias None or [m, L]. Returns (o [m, Hq, D], lse [Hq, m])."""
    m, Hq, D = q.shape
    G = Hq // k.shape[0]
    o, lse = np.zeros((m, Hq, D)), np.full((Hq, m), -np.inf)
    for h in range(Hq):
        for p in range(m):
            on = np.flatnonzero(visible[p])
            if not on.size:
                continue
            a = k[h // G, on] @ q[p, h] * scale
            if bias is not None:
                a = a + bias[p, on]
            top = a.max()
            w = np.exp(a - top)
            lse[h, p] = top + np.log(w.sum())
            o[p, h] = (w / w.sum()) @ v[h // G, on]
    return o, lse
