"""The cache operators run together, as a stream uses them: embed the chunk's queries and keys into the cache, attend,
weigh the keys, choose the frames that stay, move them into a smaller cache and attend over that. Against fp64 on the
host, captured into a graph and replayed, and on two streams at once."""

from __future__ import annotations

import threading

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from oracle import attention as OA
from oracle import cache as OC

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F, h, w, H, D = 3, 6, 10, 2, 128
HW, NF, KEEP = h * w, 9, 6
PAIRS, THETA = (22, 21, 21), 10000.0
KW = dict(h=h, w=w, softmax_scale=D ** -0.5, lam=1.0, sigma=2.0)


class Path:
    def __init__(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        new = lambda *s: torch.randn(*s, generator=g, device=DEV).bfloat16()  # noqa: E731
        self.proj = new(F * HW, 3, H, D)           # the chunk's projection
        self.k, self.v = new(1, NF * HW, H, D), new(1, NF * HW, H, D)  # the cache; its last F frames are the chunk's
        self.slot = torch.full((NF,), -1, dtype=torch.int32, device=DEV)
        self.slot[F:F + 2] = torch.arange(2, dtype=torch.int32, device=DEV)
        self.uv = torch.rand(2, F * HW, 2, generator=g, device=DEV) * torch.tensor([float(w), float(h)], device=DEV)
        self.idx = torch.randint(-2, HW, (2, F * HW), generator=g, device=DEV, dtype=torch.int32)
        self.prev = torch.rand(1, H, NF * HW, generator=g, device=DEV)
        e = lambda *s, dt=torch.float32: torch.empty(*s, dtype=dt, device=DEV)  # noqa: E731
        self.q = e(F * HW, H, D, dt=torch.bfloat16)
        self.o, self.lse = e(F * HW, H, D, dt=torch.bfloat16), e(H, F * HW)
        self.weight, self.small_weight = e(1, H, NF * HW), e(1, H, KEEP * HW)
        self.kept = e(1, KEEP, dt=torch.int32), e(1, KEEP)
        self.small = e(1, KEEP * HW, H, D, dt=torch.bfloat16), e(1, KEEP * HW, H, D, dt=torch.bfloat16)
        self.o2, self.lse2 = e(F * HW, H, D, dt=torch.bfloat16), e(H, F * HW)
        self.none = torch.full((KEEP,), -1, dtype=torch.int32, device=DEV)
        b = lambda n: torch.empty(max(16, n), dtype=torch.uint8, device=DEV)  # noqa: E731
        self.ws = [b(rv.attention_workspace_size(torch.bfloat16, F * HW, NF * HW, H, D)),
                   b(rv.key_weight_workspace_size(torch.bfloat16, F * HW, NF * HW, H, D, h, w, 2)),
                   b(rv.select_workspace_size(1, H, NF, HW)),
                   b(rv.attention_workspace_size(torch.bfloat16, F * HW, KEEP * HW, H, D))]

    def run(self):
        cache = self.k[0, (NF - F) * HW:]
        rv.rotary_embed(self.proj[:, 0], self.proj[:, 1], pairs=PAIRS, theta=THETA, h=h, w=w, t0=NF - F, out=(self.q, cache))
        rv.biased_chunk_attention(self.q, self.k[0], self.v[0], self.slot, self.uv, self.idx, **KW, out=(self.o, self.lse), workspace=self.ws[0])
        rv.attention_key_weight(self.q, self.k[0], self.lse, self.slot, self.uv, self.idx, **KW, prev=self.prev[0], decay=0.5,
                                out=self.weight[0], workspace=self.ws[1])
        rv.select_kept(self.weight, unit=HW, keep=KEEP, first=F, last=1, out=self.kept, workspace=self.ws[2])
        rv.compact_kv(self.k, self.v, self.kept[0].view(1, 1, KEEP), *self.small, unit=HW, weight=self.weight, out_weight=self.small_weight,
                      frames_per_unit=1, rope_t_pairs=PAIRS[0], rope_theta=THETA)
        rv.biased_chunk_attention(self.q, self.small[0][0], self.small[1][0], self.none, None, None, **KW, out=(self.o2, self.lse2),
                                  workspace=self.ws[3])

    def outputs(self):
        return [self.q, self.k, self.o, self.lse, self.weight, *self.kept, *self.small, self.small_weight, self.o2, self.lse2]

    def clear(self):
        for t in (self.q, self.o, self.lse, self.weight, *self.kept, *self.small, self.small_weight, self.o2, self.lse2):
            t.zero_()
        self.k[0, (NF - F) * HW:].zero_()


def test_path_against_the_oracle():
    p = Path(1)
    p.run()
    n = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    half = 2.0 ** -8
    pos = OC.grid_positions(F * HW, NF - F, h, w)
    for got, x in ((p.q, p.proj[:, 0]), (p.k[0, (NF - F) * HW:], p.proj[:, 1])):
        want = OC.rotary(n(x), pos, PAIRS, THETA)
        assert (np.abs(n(got) - want) <= np.abs(want) * half + 1e-5).all()
    args = (p.slot.cpu().numpy(), p.uv.cpu().numpy(), p.idx.cpu().numpy())
    A = OC.logits(n(p.q), n(p.k[0]), *args, h, w, D ** -0.5, 1.0, 2.0)
    weight = OC.key_weight(A, n(p.lse), n(p.prev[0]), 0.5)
    assert np.abs(n(p.weight[0]) - weight).max() <= 1e-4 * weight.max()  # single bounds: test_gpu_key_weight.py
    kept, score = OC.select_kept(p.weight.cpu().numpy(), HW, KEEP, F, 1)
    assert np.array_equal(p.kept[0].cpu().numpy(), kept) and np.array_equal(p.kept[1].cpu().numpy(), score)
    delta = (np.arange(KEEP) - kept)[:, None, :]
    want = OC.compact(n(p.k), kept[:, None, :], HW, np.zeros((1, KEEP * HW, H, D)), 0, delta, PAIRS[0], THETA)
    assert (np.abs(n(p.small[0]) - want) <= np.abs(want) * half + 1e-5).all()
    assert np.array_equal(n(p.small[1]), OC.compact(n(p.v), kept[:, None, :], HW, np.zeros((1, KEEP * HW, H, D)), 0))
    o, lse = OA.biased_attention(n(p.q), n(p.small[0][0]), n(p.small[1][0]), p.none.cpu().numpy(), None, None, h, w, D ** -0.5, 1.0, 2.0)
    assert np.abs(n(p.o2) - o).max() <= 2e-2 and np.abs(n(p.lse2) - lse).max() <= 4e-3


def test_path_replays_in_a_graph():
    p, ref, other = Path(2), Path(2), Path(3)
    ref.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        p.run()
    for _ in range(4):
        p.clear()
        graph.replay()
        other.run()  # the library's eager work beside the replay
        torch.cuda.synchronize()
        for got, want in zip(p.outputs(), ref.outputs()):
            assert torch.equal(got, want)
        torch.ones(1 << 20, device=DEV).sum().item()


def test_two_streams_at_once():
    paths, refs = [Path(4), Path(5)], [Path(4), Path(5)]
    for r in refs:
        r.run()
    torch.cuda.synchronize()
    errors = []

    def work(p, ref):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(5):
                    p.clear()
                    p.run()
                    s.synchronize()
                    for got, want in zip(p.outputs(), ref.outputs()):
                        assert torch.equal(got, want)
        except BaseException as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(paths, refs)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
