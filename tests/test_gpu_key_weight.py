"""attention_key_weight against its fp64 oracle: types, lengths from one query and one key on, frames that end inside a
tile, biased and unbiased frames, queries without an LSE, the query parts.

Tolerance, per logit. The dot product is a sum of D products in fp32: within (D + 4) 2^-24 of scale |q| . |k|. The bias
is within 4 * 2^-24 of itself where it is evaluated directly (fp32) and within 32 * 2^-24 of lam (h^2 + w^2) / (4 sigma^2)
where it is a sum of products on the matrix cores (bf16, fp8; correspondences on the grid). LSE, its multiple and the sum of
the three are rounded: 4 * 2^-24 of |A| + 2 |LSE|. A weight is then within that, relatively, plus 2^-22 for the
exponential, and the sum of n weights adds n/16 + 20 roundings (16 queries of a tile first). A weight below fp32's normal
range (2^-126; the bias of a far key makes such) may be taken as 0."""

from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2607_21848_amd as rv
from oracle import cache as OC

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def _case(seed, dtype, Lq, nf, h, w, H, D, S, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    Lk = nf * h * w
    q, k = (spread * torch.randn(n, H, D, generator=g, device=DEV) for n in (Lq, Lk))
    q, k = (x.to(dtype) for x in (q, k))
    slot = torch.full((nf,), -1, dtype=torch.int32, device=DEV)
    at = min(1, nf - S)
    slot[at:at + S] = torch.arange(S, dtype=torch.int32, device=DEV).flip(0)
    uv = idx = None
    if S:
        uv = torch.rand(S, Lq, 2, generator=g, device=DEV) * torch.tensor([float(w), float(h)], device=DEV)
        idx = torch.randint(-3, h * w, (S, Lq), generator=g, device=DEV, dtype=torch.int32)
        uv[idx < -1] = math.nan
    return q, k, slot, uv, idx


def _oracle(q, k, slot, uv, idx, h, w, scale, lam, sigma):
    n = lambda x: None if x is None else (x.float() if x.dtype != torch.float32 and x.is_floating_point() else x).cpu().numpy()  # noqa: E731
    A = OC.logits(n(q), n(k), n(slot), n(uv), n(idx), h, w, scale, lam, sigma)
    m = A.max(axis=2)
    return A, np.ascontiguousarray((m + np.log(np.exp(A - m[:, :, None]).sum(axis=2))).astype(np.float32))


def _tolerance(q, k, A, lse, h, w, scale, lam, sigma, D, biased):
    a, b = (np.abs(x.float().cpu().numpy().astype(np.float64)) for x in (q, k))
    rel = (D + 4) * U * scale * np.einsum("phd,khd->hpk", a, b) + 4 * U * (np.abs(A) + 2 * np.abs(lse.astype(np.float64))[:, :, None])
    if biased:
        rel = rel + 32 * U * abs(lam) * (h * h + w * w) / (4 * sigma * sigma)
    p = np.exp(A - lse.astype(np.float64)[:, :, None])
    return (p * (np.expm1(rel) + 2.0 ** -22)).sum(axis=1) + p.sum(axis=1) * (A.shape[1] / 16 + 20) * U + A.shape[1] * 2.0 ** -126


SHAPES = [
    # Lq, frames, h, w, H, S
    (1, 1, 1, 1, 1, 0), (1, 1, 1, 1, 1, 1), (1, 24, 5, 13, 3, 0), (31, 3, 4, 8, 2, 2), (33, 4, 8, 8, 1, 2), (64, 4, 8, 8, 1, 2),
    (97, 5, 3, 11, 3, 3), (128, 2, 1, 257, 2, 1), (200, 7, 9, 7, 2, 5), (65, 18, 2, 3, 4, 6), (300, 3, 16, 20, 2, 0), (1, 6, 30, 52, 2, 3),
    (129, 2, 33, 31, 3, 2), (700, 2, 7, 19, 1, 1),
]


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 128), (torch.float32, 64), (torch.float8_e4m3fn, 128)])
@pytest.mark.parametrize("Lq,nf,h,w,H,S", SHAPES)
def test_weights(dtype, D, Lq, nf, h, w, H, S):
    q, k, slot, uv, idx = _case(Lq + nf, dtype, Lq, nf, h, w, H, D, S)
    scale, lam, sigma = D ** -0.5, 1.3, 2.0
    A, lse = _oracle(q, k, slot, uv, idx, h, w, scale, lam, sigma)
    tol = _tolerance(q, k, A, lse, h, w, scale, lam, sigma, D, S > 0)
    want = OC.key_weight(A, lse)
    lse_d = torch.from_numpy(lse).to(DEV)
    kw = dict(h=h, w=w, softmax_scale=scale, lam=lam, sigma=sigma)
    if S and dtype != torch.float32 and max(h, w) > 256:  # beyond the bias tables of the attention
        with pytest.raises(rv.RevisitError, match="256"):
            rv.attention_key_weight(q, k, lse_d, slot, uv, idx, **kw)
        return
    for parts in (0, 1, 2, 5, 64):
        got = rv.attention_key_weight(q, k, lse_d, slot, uv, idx, query_parts=parts, **kw)
        off = np.abs(got.double().cpu().numpy() - want)
        assert (off <= tol).all(), (parts, (off / tol).max())
    # the weights of before, faded; into their own place
    prev = torch.rand(got.shape, device=DEV)
    want = OC.key_weight(A, lse, prev.cpu().numpy(), 0.75)
    tol = tol + (0.75 * prev.cpu().numpy().astype(np.float64) + want) * U
    got = rv.attention_key_weight(q, k, lse_d, slot, uv, idx, prev=prev, decay=0.75, **kw)
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()
    again = rv.attention_key_weight(q, k, lse_d, slot, uv, idx, prev=prev, decay=0.75, out=prev, **kw)
    assert again is prev and torch.equal(prev, got)


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64), (torch.float8_e4m3fn, 128)])
def test_queries_without_an_lse(dtype, D):
    """Rows whose LSE is NaN or infinite add nothing, even where their logits are not finite."""
    Lq, nf, h, w, H, S = 70, 4, 5, 9, 2, 2
    q, k, slot, uv, idx = _case(9, dtype, Lq, nf, h, w, H, D, S)
    scale, lam, sigma = D ** -0.5, 1.0, 2.0
    A, lse = _oracle(q, k, slot, uv, idx, h, w, scale, lam, sigma)
    tol = _tolerance(q, k, A, lse, h, w, scale, lam, sigma, D, True)
    lse[0, 3], lse[1, :40], lse[0, 64:] = np.nan, np.inf, -np.inf
    want = OC.key_weight(A, lse)
    q = q.float()
    q[64:, 0], q[:40, 1] = math.nan, 3e38 if dtype != torch.float8_e4m3fn else 448.0
    got = rv.attention_key_weight(q.to(dtype), k, torch.from_numpy(lse).to(DEV), slot, uv, idx, h=h, w=w, softmax_scale=scale, lam=lam,
                                  sigma=sigma)
    off = np.abs(got.double().cpu().numpy() - want)
    assert (off <= tol).all(), (off / tol).max()
    none = rv.attention_key_weight(q.to(dtype), k, torch.full((H, Lq), math.nan, device=DEV), slot, uv, idx, h=h, w=w,
                                   softmax_scale=scale, lam=lam, sigma=sigma)
    assert not none.any()


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 64), (torch.float8_e4m3fn, 128)])
def test_sharp_rows(dtype, D):
    """Logits far apart: one key has nearly all of a query's weight and the others' underflow to 0."""
    Lq, nf, h, w, H = 100, 3, 7, 10, 2
    q, k, slot, _, _ = _case(10, dtype, Lq, nf, h, w, H, D, 0, spread=6.0)
    A, lse = _oracle(q, k, slot, None, None, h, w, D ** -0.5, 0.0, 1.0)
    tol = _tolerance(q, k, A, lse, h, w, D ** -0.5, 0.0, 1.0, D, False)
    got = rv.attention_key_weight(q, k, torch.from_numpy(lse).to(DEV), None, None, None, h=h, w=w, softmax_scale=D ** -0.5, lam=0.0, sigma=1.0)
    off = np.abs(got.double().cpu().numpy() - OC.key_weight(A, lse))
    assert (off <= tol).all(), (off / tol).max()


def test_no_queries():
    k = torch.randn(30, 2, 128, device=DEV).bfloat16()
    q = torch.empty(0, 2, 128, dtype=torch.bfloat16, device=DEV)
    lse, prev = torch.empty(2, 0, device=DEV), torch.rand(2, 30, device=DEV)
    kw = dict(h=5, w=6, softmax_scale=0.1, lam=0.0, sigma=1.0)
    assert torch.equal(rv.attention_key_weight(q, k, lse, None, None, None, prev=prev, decay=0.5, **kw), 0.5 * prev)
    assert not rv.attention_key_weight(q, k, lse, None, None, None, out=torch.ones(2, 30, device=DEV), **kw).any()


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float32, 128), (torch.float8_e4m3fn, 128)])
def test_whole_chunk_under_its_own_attention(dtype, D):
    """A loop-closure chunk with the LSE that the attention returned: the weights of a head add up to its queries."""
    h, w, H, nf, S = 30, 52, 3, 6, 3
    q, k, slot, uv, idx = _case(11, dtype, 3 * h * w, nf, h, w, H, D, S)
    v = torch.randn(k.shape, device=DEV).to(torch.bfloat16 if dtype != torch.float32 else dtype)
    uv = uv.nan_to_num(1.0)
    kw = dict(h=h, w=w, softmax_scale=D ** -0.5, lam=1.0, sigma=2.0)
    _, lse = rv.biased_chunk_attention(q, k, v, slot, uv, idx, **kw)
    got = rv.attention_key_weight(q, k, lse, slot, uv, idx, **kw)
    total = got.double().sum(1)
    # the bf16 / fp8 attention sums probabilities rounded to bf16: its LSE is within 4e-3 (its own tests' bar)
    near = 4e-3 if dtype != torch.float32 else 1e-4
    assert ((total / q.shape[0] - 1).abs() <= near).all()
    assert torch.equal(got, rv.attention_key_weight(q, k, lse, slot, uv, idx, **kw))  # the same bits again


def test_retrieved_slots_out_of_range_are_unbiased():
    h, w, H, D, nf = 4, 5, 2, 128, 4
    q, k, slot, uv, idx = _case(12, torch.bfloat16, 40, nf, h, w, H, D, 2)
    slot[:] = torch.tensor([2, -7, 1000, 1], dtype=torch.int32)
    A, lse = _oracle(q, k, torch.tensor([-1, -1, -1, 1]), uv, idx, h, w, 0.1, 1.0, 2.0)
    got = rv.attention_key_weight(q, k, torch.from_numpy(lse).to(DEV), slot, uv, idx, h=h, w=w, softmax_scale=0.1, lam=1.0, sigma=2.0)
    off = np.abs(got.double().cpu().numpy() - OC.key_weight(A, lse))
    assert (off <= _tolerance(q, k, A, lse, h, w, 0.1, 1.0, 2.0, D, True)).all()


@pytest.mark.parametrize("dtype,D,Lq", [(torch.bfloat16, 128, 90), (torch.bfloat16, 128, 7), (torch.float32, 64, 90), (torch.float8_e4m3fn, 128, 90)])
def test_a_part_of_the_keys_under_the_whole_lse(dtype, D, Lq):
    """The LSE may be that of more keys than are weighed: a range of frames gets the weights it has among all."""
    h, w, H, nf, S = 5, 7, 2, 9, 4
    q, k, slot, uv, idx = _case(14, dtype, Lq, nf, h, w, H, D, S)
    A, lse = _oracle(q, k, slot, uv, idx, h, w, D ** -0.5, 1.0, 2.0)
    tol = _tolerance(q, k, A, lse, h, w, D ** -0.5, 1.0, 2.0, D, True)
    frames = slice(2, 7)
    rows = slice(2 * h * w, 7 * h * w)
    got = rv.attention_key_weight(q, k[rows].contiguous(), torch.from_numpy(lse).to(DEV), slot[frames].contiguous(), uv, idx, h=h, w=w,
                                  softmax_scale=D ** -0.5, lam=1.0, sigma=2.0)
    off = np.abs(got.double().cpu().numpy() - OC.key_weight(A, lse)[:, rows])
    assert (off <= tol[:, rows]).all(), (off / tol[:, rows]).max()


@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float8_e4m3fn, 128), (torch.float32, 64), (torch.float32, 128)])
def test_long_sums_of_one_value(dtype, D):
    """9600 queries that all give a key the same weight, in one part: 300 tiles of 32. A lane's sum, half of them, may round
    at each of 16 weights, at each of up to 18 tiles that are added up by themselves and at each of up to 19 such
    groups, then once with the other half: within 54 * 2^-24. Tile after tile it would round 300 times, near its end always the
    same way, for some of these values by nearly half a step each time: about 73 * 2^-24 in all."""
    H, Lq, h, w = 64, 9600, 5, 8
    q = torch.zeros(Lq, H, D, device=DEV).to(dtype)
    k = torch.zeros(h * w, H, D, device=DEV).to(dtype)
    kw = dict(h=h, w=w, softmax_scale=D ** -0.5, lam=0.0, sigma=1.0, query_parts=1)
    at = np.float32(-math.log(2.0 ** -12 * 1.7))
    values = at + np.arange(H, dtype=np.float32) * np.spacing(at)  # one for each head: their last bits run through all places
    lse = torch.full((H, Lq), math.inf, device=DEV)
    lse[:, 7] = torch.from_numpy(values).to(DEV)
    one = rv.attention_key_weight(q, k, lse, None, None, None, **kw).double()  # a single query's weight
    assert (one[:, :1] == one).all() and ((one[:, 0] * 2 ** 12 / 1.7 - 1).abs() < 1e-4).all()
    lse[:] = lse[:, 7:8].clone()
    got = rv.attention_key_weight(q, k, lse, None, None, None, **kw).double()
    assert ((got / (Lq * one) - 1).abs() <= 54 * U).all(), float((got / (Lq * one) - 1).abs().max() / U)


@pytest.mark.parametrize("Lq", [32, 9600])
@pytest.mark.parametrize("dtype,D", [(torch.bfloat16, 128), (torch.float8_e4m3fn, 128), (torch.float32, 64), (torch.float32, 128)])
def test_no_common_error_of_the_exponent(dtype, D, Lq):
    """Logits of 0 under LSEs around 80: the mean of many sums shows what all weights have in common. A query's exponent,
    115 in units of log 2, may round by 2^-18, which is 2.7e-6 of its weight and as often up as down: over 64 heads of
    Lq queries the mean is within 6 of its standard deviations (2.7e-6 / sqrt(3) / sqrt(64 Lq)), and 8 * 2^-24 for the exponentials' and
    the sums' own. A log2 e that is rounded to fp32 makes it 1.1e-6 throughout."""
    H, h, w = 64, 5, 8
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k = torch.zeros(Lq, H, D, device=DEV).to(dtype), torch.zeros(h * w, H, D, device=DEV).to(dtype)
    lse = 79.0 + 2.0 * torch.rand(H, Lq, generator=g, device=DEV)
    got = rv.attention_key_weight(q, k, lse, None, None, None, h=h, w=w, softmax_scale=D ** -0.5, lam=0.0, sigma=1.0).double()
    want = (-lse.double()).exp().sum(1)
    off = (got[:, 0] / want - 1).mean().abs()
    assert off <= 6 * 2.7e-6 / math.sqrt(3 * 64 * Lq) + 8 * U, float(off)


def _distances(uv, h, w):
    """Squared distances [S, Lq, h * w] of the token centres from the correspondences, float64."""
    t = np.arange(h * w)
    u = uv.cpu().numpy().astype(np.float64)
    return (u[..., :1] - (t % w + 0.5)) ** 2 + (u[..., 1:] - (t // w + 0.5)) ** 2


def _bias_bound(uv, d2, h, w, lam, sigma):
    """How far a bias of squared distance d2 may be off on the matrix cores, uv [..., 2] the correspondences. Its whole part,
    the distance of token centres times a factor of 6 bits, is added without rounding. On an axis of n tokens the other terms
    are, for a factor of 1, n (f + n / 128), n^2 / 256 and n^2 / 256 + n f + f^2 at most, f what uv is away from its token centre
    and 1/64 what the factor may be off from 6 bits; S is their sum. They cancel to no more than d2, so that no partial
    sum passes S / 2 + d2: 16 additions and the terms' own rounding. The factor and the product are off by 5 * 2^-24 of the
    bias. (Against |a|^2 - 2 a.u + |u|^2 in fp32, whose terms are n^2 / 4 each.)"""
    S = 0.0
    for axis, n in ((0, w), (1, h)):
        u = uv[..., axis].cpu().numpy().astype(np.float64)
        f = np.abs(u - np.clip(np.floor(u), 0, n - 1) - 0.5)
        S = S + 2 * n * f + n * n / 64 + f * f
    return U * abs(lam) / (2 * sigma * sigma) * (9 * S[..., None] + 21 * d2)


@pytest.mark.parametrize("dtype,Lq", [(torch.bfloat16, 7), (torch.bfloat16, 100), (torch.float8_e4m3fn, 5), (torch.float8_e4m3fn, 70)])
@pytest.mark.parametrize("h,w,nf", [(256, 256, 1), (45, 80, 2), (30, 52, 3), (1, 256, 2), (256, 1, 2), (255, 256, 1), (256, 253, 1), (2, 3, 9), (5, 13, 7), (8, 16, 4), (11, 14, 5), (7, 9, 6)])
def test_bias_beside_the_correspondence(dtype, Lq, h, w, nf):
    """Queries of zeros one at a time (the others have no LSE): a weight is exp of its bias alone. Frames of one, two, three
    and five blocks of keys put up to four of them into a workgroup."""
    H, D, lam, sigma = 2, 128, 1.0, 2.0
    g = torch.Generator(device=DEV).manual_seed(h * w)
    q, k = torch.zeros(Lq, H, D, device=DEV).to(dtype), torch.randn(nf * h * w, H, D, generator=g, device=DEV).to(dtype)
    S = nf
    slot = torch.arange(S, dtype=torch.int32, device=DEV).flip(0).contiguous()
    uv = torch.rand(S, Lq, 2, generator=g, device=DEV) * torch.tensor([float(w), float(h)], device=DEV)
    uv[:, 0] = torch.tensor([0.0, 0.0])
    uv[:, 1] = torch.tensor([w - 2.0 ** -16, h - 2.0 ** -16])
    uv[:, 2] = torch.tensor([1e-6, h / 2])
    uv[:, 3] = torch.tensor([w / 2 + 0.5, 0.3])
    uv[:, 4] = torch.tensor([-1.7, h + 2.3])  # beside the grid
    idx = torch.zeros(S, Lq, dtype=torch.int32, device=DEV)
    by_key = lambda x: x[slot.cpu().numpy()].transpose(1, 0, 2).reshape(Lq, nf * h * w)  # noqa: E731
    d2 = _distances(uv, h, w)
    bound, d2 = by_key(_bias_bound(uv, d2, h, w, lam, sigma)), by_key(d2)
    B = -lam / (2 * sigma * sigma) * d2
    for p in sorted({0, 1, 2, 3, 4, Lq // 2, Lq - 1}):
        lse = torch.full((H, Lq), math.inf, device=DEV)
        lse[:, p] = 0.0
        got = rv.attention_key_weight(q, k, lse, slot, uv, idx, h=h, w=w, softmax_scale=D ** -0.5, lam=lam, sigma=sigma)
        tol = np.exp(B[p]) * (np.expm1(bound[p] + 4 * U * np.abs(B[p])) + 2.0 ** -22) + 2.0 ** -126
        off = np.abs(got.double().cpu().numpy() - np.exp(B[p]))
        assert (off <= tol).all(), (p, (off / tol).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("Lq,nf,h,w,S", [(90, 2, 45, 80, 1), (200, 1, 100, 120, 1), (20, 2, 60, 90, 2), (130, 30, 3, 5, 20), (130, 6, 12, 13, 5)])
def test_biased_weights_of_large_grids(dtype, Lq, nf, h, w, S):
    """As test_weights, with the bound on the bias of above; the products are added to the bias, so that their D + 4
    roundings also count its size."""
    H, D, lam, sigma = 2, 128, 1.3, 2.0
    q, k, slot, uv, idx = _case(h + w, dtype, Lq, nf, h, w, H, D, S)
    uv = uv.nan_to_num(0.0)
    A, lse = _oracle(q, k, slot, uv, idx, h, w, D ** -0.5, lam, sigma)
    plain = _tolerance(q, k, A, lse, h, w, D ** -0.5, lam, sigma, D, False)
    of = slot.cpu().numpy()
    there = (idx >= 0).cpu().numpy()[..., None]
    d2 = np.where(there, _distances(uv, h, w), 0.0)
    bound = np.where(there, _bias_bound(uv, d2, h, w, lam, sigma), 0.0) + (D + 4) * U * lam / (2 * sigma * sigma) * d2
    rel = np.where((of >= 0)[:, None, None], bound[of], 0.0).transpose(1, 0, 2).reshape(Lq, nf * h * w)
    p = np.exp(A - lse.astype(np.float64)[:, :, None])
    tol = plain + (p * np.expm1(rel)[None]).sum(axis=1)
    got = rv.attention_key_weight(q, k, torch.from_numpy(lse).to(DEV), slot, uv, idx, h=h, w=w, softmax_scale=D ** -0.5, lam=lam, sigma=sigma)
    off = np.abs(got.double().cpu().numpy() - OC.key_weight(A, lse))
    assert (off <= tol).all(), (off / tol).max()


def test_refusals_of_the_binding():
    q, k, slot, uv, idx = _case(13, torch.bfloat16, 40, 4, 4, 5, 2, 128, 2)
    lse = torch.zeros(2, 40, device=DEV)
    kw = dict(h=4, w=5, softmax_scale=0.1, lam=1.0, sigma=2.0)
    with pytest.raises(ValueError, match="lse"):
        rv.attention_key_weight(q, k, lse[:, :39].contiguous(), slot, uv, idx, **kw)
    with pytest.raises(ValueError, match="contiguous"):
        rv.attention_key_weight(q[::2], k, lse[:, ::2].contiguous(), slot, uv, idx, **kw)
    with pytest.raises(ValueError, match="whole number"):
        rv.attention_key_weight(q, k, lse, slot, uv, idx, **dict(kw, w=7))
    with pytest.raises(rv.RevisitError):
        rv.attention_key_weight(q, k, lse, slot, uv, idx, query_parts=2, workspace=torch.empty(16, dtype=torch.uint8, device=DEV), **kw)
