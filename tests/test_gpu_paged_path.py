"""The paged cache as it is used: streams that grow chunk by chunk, keys turned and appended, the chunk's queries over what
the stream holds; the same in a captured graph, on two streams at once, and from one loop closure to the next."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from oracle import cache as OC
from tests.paged_helpers import BF16, DEV, F32, FP8, GIVEN, check_attention, gen, values

pytestmark = pytest.mark.gpu
THETA, PAIRS = 10000.0, (22, 21, 21)


class Cache:
    """Two streams' pages, as a serving loop keeps them."""

    def __init__(self, dtype, B, H, D, page, most, n_pages):
        self.dtype, self.B, self.H, self.D, self.page = dtype, B, H, D, page
        self.k, self.v = (torch.zeros(n_pages, H, page, D, device=DEV).to(dtype) for _ in range(2))
        self.scales = [torch.zeros(n_pages, H, page // 32, dtype=torch.uint8, device=DEV).view(torch.float8_e8m0fnu) for _ in range(2)] if dtype == FP8 else [None] * 2
        self.table = torch.randperm(n_pages, generator=gen(0), device=DEV)[:B * most].int().view(B, most).contiguous()
        self.n = torch.zeros(B, dtype=torch.int32, device=DEV)

    def append(self, k, v, n=None, **kw):
        return rv.append_paged_kv(k, v, self.k, self.v, self.table, self.n if n is None else n, scale_k=self.scales[0], scale_v=self.scales[1], theta=THETA, **kw)

    def attend(self, q, n=None, **kw):
        return rv.paged_chunk_attention(q, self.k, self.v, self.table, self.n if n is None else n, scale_k=self.scales[0], scale_v=self.scales[1],
                                        softmax_scale=self.D ** -0.5, **kw)

    # what check_attention asks for
    @property
    def lens(self):
        return self.n.tolist()

    def held(self, s):
        L, out = self.lens[s], []
        for x, sc in ((self.k, self.scales[0]), (self.v, self.scales[1])):
            full = x[self.table[s].long()] if sc is None else x.view(torch.uint8)[self.table[s].long()].view(FP8)
            full = full.float().double()
            if sc is not None:
                full = full * torch.exp2(sc.view(torch.uint8)[self.table[s].long()].double() - 127).repeat_interleave(32, 2)[..., None]
            out.append(full.transpose(0, 1).flatten(1, 2)[:, :L].cpu().numpy())
        return out[0], out[1], np.ones(L, bool)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
def test_streams_that_grow(dtype):
    """Chunks of 2 x 5 x 7 tokens and single tokens in turn; every attention against what the pages hold, and what the pages
    hold against every key and value that ever went in."""
    B, H, D, page, h, w = 2, 2, 128, 64, 5, 7
    c = Cache(dtype, B, H, D, page, 8, 20)
    ks, vs = [[] for _ in range(B)], [[] for _ in range(B)]
    for step, new in enumerate(([70, 70], [1, 1], [35, 70], [0, 1], [70, 0], [1, 1])):
        cu = np.concatenate([[0], np.cumsum(new)])
        n = int(cu[-1])
        rows = values(gen(step), GIVEN[dtype], n, 3, H, D)  # q, k and v of one projection
        at = c.n.clone()
        even = None if len(set(new)) == 1 else torch.tensor(cu, dtype=torch.int32, device=DEV)
        c.n = c.append(rows[:, 1], rows[:, 2], cu=even, pairs=PAIRS, h=h, w=w)
        seen = np.concatenate([int(a) + 1 + np.arange(m) for a, m in zip(at.tolist(), new)]).astype(np.int32)
        for visible in (None, seen):
            o, lse = c.attend(rows[:, 0], cu=even, visible=None if visible is None else torch.from_numpy(visible).to(DEV))
            check_attention(c, rows[:, 0], o, lse, cu.tolist(), visible)
        for s in range(B):
            ks[s].append(rows[cu[s]:cu[s + 1], 1].float().double().cpu().numpy())
            vs[s].append(rows[cu[s]:cu[s + 1], 2].float().double().cpu().numpy())
            k, v = np.concatenate(ks[s]), np.concatenate(vs[s])
            turned = OC.rotary(k, OC.grid_positions(len(k), 0, h, w), PAIRS, THETA)
            mag = np.repeat(np.abs(k[..., 0::2]) + np.abs(k[..., 1::2]), 2, -1)
            for got, want, m in ((c.held(s)[0], turned, mag), (c.held(s)[1], v, 0)):
                got, tol = got.transpose(1, 0, 2), 6 * 2.0 ** -24 * m
                if dtype == FP8:  # two roundings at most matter: below a grown scale's smallest normal value; scales here are at most 2^-5 (|x| < 14)
                    tol = tol + np.maximum(2.0 ** -4 * np.abs(want), 2 * 2.0 ** -10 * 2.0 ** -5)
                else:
                    tol = tol + (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * np.abs(want)
                assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("dtype", [FP8, BF16])
def test_captured(dtype):
    """One graph of append and attention, its lengths on the device: replayed with eager work between, each replay
    against the same calls made eagerly."""
    B, H, D, page = 3, 2, 128, 32
    q, k, v = (torch.empty(B, x, D, dtype=BF16, device=DEV) for x in (4, 2, 2))
    o, lse = torch.empty(B, 4, D, dtype=BF16, device=DEV), torch.empty(4, B, device=DEV)
    c, e = Cache(dtype, B, H, D, page, 16, 50), Cache(dtype, B, H, D, page, 16, 50)
    ws = torch.empty(max(16, rv.paged_attention_workspace_size(dtype, B, False, B, 4, H, D, page, 16, 0, 4)), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(c.n)

    def step(c, out):
        c.append(k, v, pairs=PAIRS, h=4, w=4, out_len=out)
        c.attend(q, n=out, key_parts=4, out=(o, lse), workspace=ws)
        c.n.copy_(out)

    for x in (q, k, v):
        x.normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(c, out)
    torch.cuda.current_stream().wait_stream(side)
    step(e, out)  # the pages of both hold the same
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(c, out)
    for c_ in (c, e):
        c_.n.copy_(torch.tensor([0, 40, 95]))
    for i in range(40):
        for j, x in enumerate((q, k, v)):
            x.copy_(values(gen(100 + 3 * i + j), BF16, *x.shape))
        g.replay()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        step(e, torch.empty_like(out))
        assert torch.equal(o, got[0]) and torch.equal(lse, got[1])
        assert torch.equal(c.n, e.n)
    assert torch.equal(c.k.view(torch.uint8), e.k.view(torch.uint8)) and torch.equal(c.v.view(torch.uint8), e.v.view(torch.uint8))


def test_two_streams_at_once():
    """Calls of two device streams with workspaces of their own give what they give one after the other."""
    B, H, D, page = 4, 4, 128, 64
    jobs = []
    for i in range(2):
        c = Cache(FP8, B, H, D, page, 20, 100)
        k, v = (values(gen(200 + 2 * i + j), BF16, B * 900, H, D) for j in range(2))
        c.n = c.append(k, v, pairs=PAIRS, h=30, w=30)
        jobs.append((c, values(gen(210 + i), BF16, B * 2, 8, D)))
    want = [c.attend(q, key_parts=5) for c, q in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for i, ((c, q), s) in enumerate(zip(jobs, streams)):
            with torch.cuda.stream(s):
                got[i].append(c.attend(q, key_parts=5))
    torch.cuda.synchronize()
    for i in range(2):
        for o, lse in got[i]:
            assert torch.equal(o, want[i][0]) and torch.equal(lse, want[i][1])


def test_loop_closure_over_pages():
    """Correspondence of a turned camera into a stored frame, then the biased attention over the stream's 8-bit pages: against
    the dense attention over the same values."""
    h, w, H, D = 12, 16, 2, 128
    hw = h * w
    c = Cache(FP8, 1, H, D, 32, 24, 30)
    k, v = (values(gen(300 + j), BF16, 4 * hw, H, D) for j in range(2))
    c.n = c.append(k, v, pairs=PAIRS, h=h, w=w)
    K = torch.tensor([[8.0, 8.0, 8.0, 6.0]], device=DEV)
    src = torch.eye(4, device=DEV)[None]
    a = 0.2
    tgt = src.clone()
    tgt[0, 0, 0] = tgt[0, 2, 2] = np.cos(a)
    tgt[0, 0, 2], tgt[0, 2, 0] = np.sin(a), -np.sin(a)
    uv, idx = rv.reproject_rotation(tgt, K, src, K, h=h, w=w, p=1)
    q = values(gen(310), BF16, hw, H, D)
    slot = torch.tensor([[-1, 0, -1, -1]], dtype=torch.int32, device=DEV)
    o, lse = c.attend(q, kv_frame_slot=slot, corr_uv=uv, corr_idx=idx, h=h, w=w, lam=1.0, sigma=2.0)
    kd, vd, _ = c.held(0)
    kd, vd = (torch.from_numpy(x.transpose(1, 0, 2).copy()).to(DEV).to(BF16) for x in (kd, vd))
    want, wl = rv.biased_chunk_attention(q, kd, vd, slot[0], uv, idx, h=h, w=w, softmax_scale=D ** -0.5, lam=1.0, sigma=2.0)
    # each rounds its weights (2^-8; the dense one's sum too) and its output (2^-8)
    assert float((o.float() - want.float()).abs().max()) <= 5 * 2.0 ** -8 * float(vd.float().abs().max())
    assert float((lse - wl).abs().max()) <= 4e-3
    plain, _ = c.attend(q)
    assert float((plain.float() - o.float()).abs().max()) > 0.01  # the bias is seen
