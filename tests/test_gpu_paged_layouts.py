"""Pools whose pages, heads and positions lie anywhere: append_paged_kv and paged_chunk_attention give the same bits as over
contiguous pools, which the other tests hold against the oracle, and touch nothing between the rows."""

from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from tests.paged_helpers import BF16, DEV, F32, FP8, GIVEN, Pool, gen, values

pytestmark = pytest.mark.gpu
E8M0 = torch.float8_e8m0fnu


def _bytes(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x.contiguous().view(torch.uint8)


def _like(x, shape, fill=0x5a):
    """Memory of x's type, every byte `fill`."""
    return torch.full((*shape[:-1], shape[-1] * x.element_size()), fill, dtype=torch.uint8, device=DEV).view(x.dtype)


def _views(x, y, how):
    """The contents of x and y, both [pages, H, rows, D] (or scales [pages, H, blocks]), as views of memory laid out another
    way, and that memory."""
    n, H, r, tail = x.shape[0], x.shape[1], x.shape[2], tuple(x.shape[3:])
    at = (0, 2, 1) + tuple(range(3, x.dim()))
    if how == "positions":  # [pages, rows, H, D], keys and values each
        mem = [_like(x, (n, r, H, *tail)) for _ in range(2)]
        got = [m.permute(at) for m in mem]
    elif how == "both":     # keys and values of a page beside each other
        mem = [_like(x, (n, 2, H, r, *tail))]
        got = [mem[0][:, 0], mem[0][:, 1]]
    elif how == "pairs":    # of a position: [pages, rows, 2, H, D]
        mem = [_like(x, (n, r, 2, H, *tail))]
        got = [mem[0][:, :, i].permute(at) for i in range(2)]
    elif how == "heads":    # [H, pages, rows, D], and values inside a larger pool with gaps behind each row
        mem = [_like(x, (H, n, r, *tail)), _like(x, (n + 1, H + 2, r, *tail[:-1], tail[-1] + 32) if tail else (n + 1, H + 2, r + 3))]
        got = [mem[0].transpose(0, 1), mem[1][1:, 1:1 + H, :, :tail[-1]] if tail else mem[1][1:, 1:1 + H, :r]]
    else:                   # "values": only the values' pool is a view
        mem = [x.clone(), _like(x, (n, r, H, *tail))]
        got = [mem[0], mem[1].permute(at)]
    for g, src in zip(got, (x, y)):
        _bytes(g).copy_(_bytes(src)) if g.element_size() == 1 else g.copy_(src)
    return got, mem


def _other(pool, how):
    """The pool's tensors (k, v, scale_k, scale_v) laid out as `how` says, and their memory."""
    kv, mem = _views(pool.k, pool.v, how)
    if pool.scales[0] is None:
        return (*kv, None, None), mem
    sc, mem_s = _views(*pool.scales, how)
    return (*kv, *sc), mem + mem_s


def _same(a, b):
    assert torch.equal(_bytes(a), _bytes(b))


LAYOUTS = ["positions", "both", "pairs", "heads", "values"]


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("D,H,page,before,new", [(64, 5, 64, [63, 0], [1, 130]), (128, 3, 32, [31, 7, 32], [2, 1, 33]), (128, 1, 128, [10], [300])])
def test_append(how, dtype, D, H, page, before, new):
    pool = Pool(1, dtype, [a + b for a, b in zip(before, new)], H, D, page)
    (k2, v2, sk2, sv2), mem = _other(pool, how)
    ck, cv, table, _ = pool.args()
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
    lens = torch.tensor(before, dtype=torch.int32, device=DEV)
    g = gen(2)
    kw = dict(pairs=(D // 2 - 20, 9, 11), theta=10000.0, cu=cu, h=5, w=7)
    for size in (4.0, 2.0 ** 9):  # the second time scales grow, and held codes are rounded again
        k, v = (values(g, GIVEN[dtype], sum(new), H, D) * size for _ in range(2))
        want = rv.append_paged_kv(k, v, ck, cv, table, lens, **kw, **pool.kw())
        got = rv.append_paged_kv(k, v, k2, v2, table, lens, scale_k=sk2, scale_v=sv2, **kw)
        assert torch.equal(want, got)
        for a, b in zip((ck, cv, *pool.scales), (k2, v2, sk2, sv2)):
            if a is not None:
                _same(a, b)
    # nothing but the pools' own elements has changed
    for t in (k2, v2, sk2, sv2):
        if t is not None:
            _bytes(t).zero_() if t.element_size() == 1 else t.zero_()
    kv, mem0 = _views(torch.zeros_like(ck), torch.zeros_like(cv), how)
    if pool.scales[0] is not None:
        mem0 += _views(*(torch.zeros_like(_bytes(s)).view(E8M0) for s in pool.scales), how)[1]
    for a, b in zip(mem, mem0):
        _same(a, b)


def _bias(S, n, h, w, B, frames, seed):
    g = gen(seed)
    uv = torch.rand(S, n, 2, generator=g, device=DEV) * torch.tensor([w, h], device=DEV, dtype=torch.float32)
    idx = torch.randint(-3, 20, (S, n), generator=g, device=DEV, dtype=torch.int32)
    slot = torch.randint(-1, S, (B, frames), generator=g, device=DEV, dtype=torch.int32)
    return dict(corr_uv=uv, corr_idx=idx, kv_frame_slot=slot, h=h, w=w, lam=1.0, sigma=2.0)


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
@pytest.mark.parametrize("D,Hq,Hk,page,lens,new", [
    (64, 4, 2, 32, [70, 200, 33], [1, 2, 1]), (128, 3, 3, 64, [300], [1]), (128, 8, 2, 64, [500, 31], [6, 3]), (64, 2, 2, 64, [300, 90], [40, 10]),
    (64, 2, 1, 32, [700], [80]), (128, 2, 2, 128, [900], [100]), (128, 2, 1, 32, [1000, 333], [150, 300]),
])
def test_attention(how, dtype, D, Hq, Hk, page, lens, new):
    pool = Pool(3, dtype, lens, Hk, D, page)
    pool.table[0, len(pool.table[0]) // 2] = -1  # a page that is none
    # not seen by every query: NaN, infinity; behind the last key
    k, v = pool.k.float(), pool.v.float()
    L, t = lens[0], pool.table[0]
    if t[(L - 1) // page] >= 0:
        v[t[(L - 1) // page], :, (L - 1) % page, :3] = torch.tensor([float("nan"), 448.0, -float("inf") if dtype != FP8 else 0.0], device=DEV)
    pool.k, pool.v = k.to(dtype), v.to(dtype)
    (k2, v2, sk2, sv2), _ = _other(pool, how)
    ck, cv, table, n_held = pool.args()
    cu = np.concatenate([[0], np.cumsum(new)])
    n = int(cu[-1])
    q = values(gen(4), GIVEN[dtype], n, Hq, D)
    visible = torch.tensor(np.concatenate([L - m + 1 + np.arange(m) for L, m in zip(lens, new)]), dtype=torch.int32, device=DEV)
    cu = torch.tensor(cu, dtype=torch.int32, device=DEV)
    for kw in (dict(), dict(visible=visible), dict(visible=visible, key_parts=3, **_bias(2, n, 6, 8, len(lens), 9, 5))):
        want, wl = rv.paged_chunk_attention(q, ck, cv, table, n_held, cu=cu, softmax_scale=D ** -0.5, **pool.kw(), **kw)
        got, gl = rv.paged_chunk_attention(q, k2, v2, table, n_held, cu=cu, softmax_scale=D ** -0.5, scale_k=sk2, scale_v=sv2, **kw)
        assert torch.equal(want.nan_to_num(nan=7.0), got.nan_to_num(nan=7.0)) and torch.equal(wl.nan_to_num(nan=7.0), gl.nan_to_num(nan=7.0))


def test_scales_alone():
    """Contiguous pools of 8 bits whose scales lie another way."""
    pool = Pool(5, FP8, [200], 3, 128, 64)
    ck, cv, table, lens = pool.args()
    sk, sv = (_bytes(s).transpose(1, 2).contiguous().transpose(1, 2).view(E8M0) for s in pool.scales)
    assert not sk.is_contiguous()
    q = values(gen(6), BF16, 5, 3, 128)
    a = rv.paged_chunk_attention(q, ck, cv, table, lens, softmax_scale=0.1, **pool.kw())
    b = rv.paged_chunk_attention(q, ck, cv, table, lens, softmax_scale=0.1, scale_k=sk, scale_v=sv)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    new = values(gen(7), BF16, 20, 3, 128)
    start = torch.tensor([150], dtype=torch.int32, device=DEV)
    kw = dict(pairs=(22, 21, 21), theta=10000.0, h=4, w=4)
    k2, v2 = _bytes(ck).clone().view(FP8), _bytes(cv).clone().view(FP8)
    rv.append_paged_kv(new, new, ck, cv, table, start, **kw, **pool.kw())
    rv.append_paged_kv(new, new, k2, v2, table, start, scale_k=sk, scale_v=sv, **kw)
    for x, y in ((ck, k2), (cv, v2), (pool.scales[0], sk), (pool.scales[1], sv)):
        _same(x, y)


def test_many_pages_apart():
    """Rows further apart than 2^32 bytes from the pool's first one."""
    H, D, page = 2, 128, 256
    big = torch.empty((1 << 32) + page * H * D, dtype=torch.uint8, device=DEV)
    far = torch.as_strided(big, (2, H, page, D), (1 << 32, D, H * D, 1)).view(FP8)
    sk, sv = (torch.zeros(2, H, page // 32, dtype=torch.uint8, device=DEV).view(E8M0) for _ in range(2))
    near = torch.zeros(2, H, page, D, dtype=torch.uint8, device=DEV).view(FP8)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device=DEV)
    zero, full = (torch.tensor([x], dtype=torch.int32, device=DEV) for x in (0, 400))
    k, v = (values(gen(8 + i), BF16, 400, H, D) for i in range(2))
    kw = dict(pairs=(0, 0, 0), theta=10000.0, h=1, w=1, scale_k=sk, scale_v=sv)
    rv.append_paged_kv(k, v, far, near, table, zero, **kw)
    back = far.float() * torch.exp2(sk.view(torch.uint8).float() - 127).repeat_interleave(32, 2)[..., None]
    got = back[[1, 0]].transpose(0, 1).flatten(1, 2)[:, :400].transpose(0, 1)
    # half a step of e4m3: 2^-4 of the value, 2^-10 of the scale below its smallest normal
    half = torch.maximum(k.float().abs() * 2.0 ** -4, 2.0 ** -10 * torch.exp2(sk.view(torch.uint8).float().max() - 127))
    assert bool(((got - k.float()).abs() <= half).all())
    dense = [x.contiguous() for x in (far, near)]
    for m in (1, 150):
        q = values(gen(10), BF16, m, H, D)
        a = rv.paged_chunk_attention(q, far, near, table, full, softmax_scale=0.1, scale_k=sk, scale_v=sv)
        b = rv.paged_chunk_attention(q, *dense, table, full, softmax_scale=0.1, scale_k=sk, scale_v=sv)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_refusals():
    """Views that append could not write without a race, rows that are none, and keys over values."""
    pool = Pool(11, FP8, [64], 2, 64, 32)
    ck, cv, table, lens = pool.args()
    k = values(gen(12), BF16, 4, 2, 64)
    kw = dict(pairs=(8, 8, 8), theta=10000.0, h=3, w=3, **pool.kw())
    n = pool.n_pages
    one = ck[:1].view(torch.uint8).expand(n, 2, 32, 64).view(FP8)                     # every page the same
    wide = torch.zeros(n, 2, 32, 128, dtype=torch.uint8, device=DEV).view(FP8)
    odd = torch.zeros(n, 2, 32, 72, dtype=torch.uint8, device=DEV).view(FP8)[..., :64]  # rows 72 bytes apart
    both = torch.zeros(n, 2, 3, 32, 64, dtype=torch.uint8, device=DEV).view(FP8)
    for err, a, b in [(rv.RevisitError, one, cv), (ValueError, wide[..., ::2], cv), (rv.RevisitError, odd, cv), (rv.RevisitError, both[:, :, 0], both[:, :, 0]),
                      (rv.RevisitError, wide[..., :64], wide[..., 16:80]), (ValueError, ck.transpose(2, 3), cv), (ValueError, wide.transpose(1, 2), cv)]:
        with pytest.raises(err):
            rv.append_paged_kv(k, k, a, b, table, lens, **kw)
    q = values(gen(13), BF16, 4, 2, 64)
    for err, a, b in [(ValueError, wide[..., ::2], cv), (rv.RevisitError, odd, cv), (ValueError, ck, wide), (ValueError, wide.transpose(1, 2), cv)]:
        with pytest.raises(err):
            rv.paged_chunk_attention(q, a, b, table, lens, softmax_scale=0.1, **pool.kw())
    # reading is another matter: one page for all
    o, _ = rv.paged_chunk_attention(q, one, one, table, lens, softmax_scale=0.1, **pool.kw())
    same = one.contiguous()
    p, _ = rv.paged_chunk_attention(q, same, same, table, lens, softmax_scale=0.1, **pool.kw())
    assert torch.equal(o, p)


@pytest.mark.parametrize("dtype", [FP8, BF16])
def test_in_a_graph(dtype):
    """Captured once over views of one tensor for keys and values, replayed as the stream grows."""
    H, D, page, n_pages = 4, 128, 64, 6
    pool = Pool(14, dtype, [n_pages * page - 1], H, D, page, spare=0)
    (k2, v2, sk2, sv2), _ = _other(pool, "pairs")
    ck, cv, table, _ = pool.args()
    k, v, q = (torch.zeros(3, H, D, dtype=GIVEN[dtype], device=DEV) for _ in range(3))
    held, after = (torch.full((1,), 5, dtype=torch.int32, device=DEV) for _ in range(2))
    kw = dict(pairs=(22, 21, 21), theta=10000.0, h=4, w=4, out_len=after)

    def step(a, b, sa, sb):
        rv.append_paged_kv(k, v, a, b, table, held, scale_k=sa, scale_v=sb, **kw)
        return rv.paged_chunk_attention(q, a, b, table, after, softmax_scale=0.1, scale_k=sa, scale_v=sb, key_parts=2)
    step(k2, v2, sk2, sv2)
    step(ck, cv, *pool.scales)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = step(k2, v2, sk2, sv2)
    g = gen(15)
    for _ in range(4):
        for x in (k, v, q):
            x.copy_(values(g, GIVEN[dtype], 3, H, D))
        graph.replay()
        a, b = o.clone(), lse.clone()
        want = step(ck, cv, *pool.scales)
        torch.cuda.synchronize()
        assert torch.equal(a, want[0]) and torch.equal(b, want[1])
        _same(ck, k2), _same(cv, v2)
        held.copy_(after)


@pytest.mark.parametrize("dtype", [FP8, BF16, F32])
def test_keys_without_a_rotation_need_no_grid(dtype):
    pool, other = (Pool(16, dtype, [70], 2, 64, 32) for _ in range(2))
    ck, cv, table, _ = pool.args()
    k, v = (values(gen(17 + i), GIVEN[dtype], 60, 2, 64) for i in range(2))
    start = torch.tensor([10], dtype=torch.int32, device=DEV)
    rv.append_paged_kv(k, v, ck, cv, table, start, pairs=(0, 0, 0), theta=10000.0, **pool.kw())
    rv.append_paged_kv(k, v, other.k, other.v, table, start, pairs=(0, 0, 0), theta=10000.0, h=3, w=5, t0=9, **other.kw())
    for a, b in zip((ck, cv, *pool.scales), (other.k, other.v, *other.scales)):
        if a is not None:
            _same(a, b)
    if dtype != FP8:
        rows = torch.cat([ck[p] for p in table[0].tolist()], 1)[:, 10:70]
        _same(rows.transpose(0, 1), k)


def test_pools_without_heads_are_refused():
    pool = torch.zeros(2, 0, 32, 64, dtype=BF16, device=DEV)
    table, lens = torch.zeros(1, 2, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    q = values(gen(19), BF16, 3, 2, 64)
    for heads in (2, 0):
        with pytest.raises(ValueError):
            rv.paged_chunk_attention(q[:, :heads], pool, pool, table, lens, softmax_scale=0.1)
    with pytest.raises(rv.RevisitError):
        rv.append_paged_kv(q[:, :0], q[:, :0], pool, pool, table, lens, pairs=(0, 0, 0), theta=10000.0)
