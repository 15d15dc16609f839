"""Paged caches for the tests: pools with pages in any order, and what a stream's pages hold in float64."""

from __future__ import annotations

import numpy as np
import torch

from oracle import paged as OP

DEV = "cuda:0"
GIVEN = {torch.bfloat16: torch.bfloat16, torch.float32: torch.float32, torch.float8_e4m3fn: torch.bfloat16}
BF16, F32, FP8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def values(g, dtype, *shape):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


class Pool:
    """A pool of pages full of values, the page table of streams of `lens` positions, and what they hold."""

    room = 0  # positions that a table has entries for, at least

    def __init__(self, seed, dtype, lens, H, D, page, spare=2, max_pages=None):
        g = gen(seed)
        self.dtype, self.lens, self.H, self.D, self.page = dtype, list(lens), H, D, page
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g, device=DEV).cpu().numpy()
        self.table = np.full((len(lens), max_pages or max(need + [1, self.room // page])), -1, np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, H, page, D)
        x = [torch.randn(*shape, generator=g, device=DEV) * torch.exp2(torch.randint(-3, 3, (H, 1, 1), generator=g, device=DEV).float()) for _ in range(2)]
        self.scales = [None, None]
        if dtype == FP8:
            # any scales at all, also far from what the values would ask for
            byte = [torch.randint(120, 126, (self.n_pages, H, page // 32), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
            self.scales = [b.view(torch.float8_e8m0fnu) for b in byte]
            x = [(v / torch.exp2(b.float() - 127).repeat_interleave(32, 2)[..., None]).clamp(-448, 448) for v, b in zip(x, byte)]
        self.k, self.v = (v.to(dtype) for v in x)

    def args(self):
        return self.k, self.v, torch.from_numpy(self.table).to(DEV), torch.tensor(self.lens, dtype=torch.int32, device=DEV)

    def kw(self):
        return dict(scale_k=self.scales[0], scale_v=self.scales[1])

    def held(self, s):
        """(k, v) [H, L, D] float64 of stream s, and which positions have a page."""
        out = []
        have = np.zeros(self.lens[s], bool)
        for x, sc in ((self.k, self.scales[0]), (self.v, self.scales[1])):
            full = x.float().double().cpu().numpy()
            if sc is not None:
                full = full * np.repeat(sc.float().double().cpu().numpy(), 32, 2)[..., None]
            got = np.zeros((self.H, self.lens[s], self.D))
            for i in range(-(-self.lens[s] // self.page)):
                p = self.table[s, i]
                a, b = i * self.page, min(self.lens[s], (i + 1) * self.page)
                if 0 <= p < self.n_pages:
                    got[:, a:b] = full[p, :, :b - a]
                    have[a:b] = True
            out.append(got)
        return out[0], out[1], have


def check_attention(pool, q, o, lse, cu=None, visible=None, scale=None, bias=None, slack=0.0):
    """o and lse against the oracle on every stream, within what the roundings allow.

    A logit is a sum of D products in fp32 (off by D + 6 units of 2^-24 of the sum of their magnitudes, the scale and the
    exponent's FMA included, and 2^-22 of a bias beside it); a probability is off by that, 2^-22 of the
    exponential and, for bf16 values, half a step of bf16 (2^-8) in the product with the values alone; sums of L / 16
    probabilities a lane and of L products by 2^-24 each; the output by half a step of its type. An empty row is exact.
    `slack`: what a bias in separable form may add to a logit's error (8 units of its largest term)."""
    n, Hq, D = q.shape
    scale = scale or D ** -0.5
    q64 = q.float().double().cpu().numpy()
    o64, l64 = o.float().double().cpu().numpy(), lse.double().cpu().numpy()
    B = len(pool.lens)
    vis = None if visible is None else np.asarray(visible)
    worst = 0.0
    for s, (t0, m) in enumerate(OP.streams(n, cu, B)):
        if m == 0:
            continue
        k, v, have = pool.held(s)
        L = pool.lens[s]
        on = np.broadcast_to(have, (m, L)).copy()
        if vis is not None:
            on &= np.arange(L) < vis[t0:t0 + m, None]
        b = None if bias is None else bias[s]
        want, wl = OP.attend(q64[t0:t0 + m], k, v, on, scale, b)
        kk, vv = np.where(np.isfinite(k), np.abs(k), 0), np.where(np.isfinite(v), np.abs(v), 0)
        for h in range(Hq):
            mag = np.abs(q64[t0:t0 + m, h]) @ kk[h // (Hq // pool.H)].T * scale if L else np.zeros((m, 0))
            d = np.where(on, (D + 6) * 2.0 ** -24 * mag + (0 if b is None else np.abs(b) * 2.0 ** -22), 0).max(1, initial=0) + 2.0 ** -22 + slack
            rows = on.any(1)
            tol_l = d + (L / 16 + 16) * 2.0 ** -24 + 4 * 2.0 ** -24 * np.abs(np.where(rows, wl[h], 0))
            got_l = l64[h, t0:t0 + m]
            assert np.array_equal(got_l[~rows], wl[h][~rows])  # -inf
            assert (np.abs(got_l - np.where(rows, wl[h], 0))[rows] <= tol_l[rows]).all(), ("lse", s, h, np.abs(got_l - wl[h])[rows].max())
            half = {BF16: 2.0 ** -8, F32: 2.0 ** -24}[q.dtype]
            # sum of w |v| over the keys that a query sees
            wsum = np.zeros((m, D))
            for p in np.flatnonzero(rows):
                j = np.flatnonzero(on[p])
                a = k[h // (Hq // pool.H), j] @ q64[t0 + p, h] * scale + (0 if b is None else b[p, j])
                w = np.exp(a - wl[h, p])
                wsum[p] = w @ vv[h // (Hq // pool.H), j]
            tol = (2 * d[:, None] + (0 if q.dtype == F32 else 2.0 ** -8) + 2 * (L + 16) * 2.0 ** -24) * wsum + half * np.abs(np.where(np.isfinite(want[:, h]), want[:, h], 0)) + 1e-30
            with np.errstate(invalid="ignore"):  # inf - inf
                off = np.abs(o64[t0:t0 + m, h] - want[:, h])
            same = (np.isnan(want[:, h]) & np.isnan(o64[t0:t0 + m, h])) | (want[:, h] == o64[t0:t0 + m, h])
            ok = same | (off <= tol)
            assert ok.all(), ("o", s, h, np.argwhere(~ok)[:4], (off / tol)[~ok].max())
            with np.errstate(invalid="ignore"):
                worst = max(worst, float(np.nanmax(np.where(same, 0, off / tol), initial=0)))
            assert (o64[t0:t0 + m, h][~rows] == 0).all()
    return worst
