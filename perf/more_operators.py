"""The paged cache, as cases that can be timed and compared: new keys and values of several streams put into its
pages with the rotary position on the way, and the attention that reads them there, pages in the inputs' type or in 8
bits with a power-of-two scale for each 32 tokens of a head.

With `own` false a pass computes the plain form, elementary torch operations in 32 bits (64 for angles); with `own`
true it makes the calls of this package. Inputs come from a seed: q, k and v are N(0, 1) times a factor of
their head between 1/4 and 4, pages lie in the pool in any order, correspondences lie a few tokens beside their token.
"""

import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32  # tokens that share a scale
LOW = -100  # smallest exponent of a scale
F = 3  # latent frames per chunk
SIGMA, LAM, THETA, T0 = 2.0, 1.0, 10000.0, 2
E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
STORED = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": E4M3}
GIVEN = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2, "fp8": 1}


def listed():
    return [
        # -- new keys and values into their pages
        # one token of one stream, as a token-wise loop appends it: launch and latency only
        {"name": "append_one_token", "kind": "append", "cache": "fp8", "streams": 1, "tokens": 1, "ragged": False, "before": 1000,
         "H": 12, "D": 128, "page": 64, "packed": False, "given": True, "h": 30, "w": 52},
        # a token of each of 128 streams of uneven lengths, whose last blocks are partly full: scales grow, codes are rounded again
        {"name": "append_batch", "kind": "append", "cache": "fp8", "streams": 128, "tokens": 1, "ragged": True, "before": 250,
         "H": 8, "D": 128, "page": 64, "packed": False, "given": True, "h": 30, "w": 52},
        # one layer of a 30 x 52 chunk of three frames, k and v out of the projection's packed rows
        {"name": "append_chunk", "kind": "append", "cache": "fp8", "streams": 1, "tokens": 4680, "ragged": False, "before": 14040,
         "H": 12, "D": 128, "page": 64, "packed": True, "given": False, "h": 30, "w": 52},
        # prompts of uneven lengths into pages of their own type, shared heads of 64
        {"name": "append_prompts", "kind": "append", "cache": "bf16", "streams": 8, "tokens": 2000, "ragged": True, "before": 500,
         "H": 8, "D": 64, "page": 32, "packed": False, "given": True, "h": 1, "w": 1},
        # a chunk at 720p with 40 heads, the largest
        {"name": "append_720p", "kind": "append", "cache": "fp8", "streams": 1, "tokens": 10800, "ragged": False, "before": 300,
         "H": 40, "D": 128, "page": 128, "packed": False, "given": False, "h": 45, "w": 80},
        # -- attention over the pages
        # one query token over one frame: launch and latency only
        {"name": "attend_one_token", "kind": "attend", "cache": "fp8", "streams": 1, "queries": 1, "ragged": False, "keys": 1560,
         "Hq": 12, "Hk": 12, "D": 128, "page": 64, "causal": False, "ret": 0, "h": 30, "w": 52},
        # one query token over a long cache: its keys and values are read once
        {"name": "attend_one_query", "kind": "attend", "cache": "fp8", "streams": 1, "queries": 1, "ragged": False, "keys": 37440,
         "Hq": 12, "Hk": 12, "D": 128, "page": 64, "causal": False, "ret": 0, "h": 30, "w": 52},
        # a token of each of 64 streams of uneven lengths, four query heads to a key head
        {"name": "attend_batch", "kind": "attend", "cache": "fp8", "streams": 64, "queries": 1, "ragged": True, "keys": 16384,
         "Hq": 32, "Hk": 8, "D": 128, "page": 64, "causal": True, "ret": 0, "h": 1, "w": 1},
        # prompts of uneven lengths behind what their streams hold, a token sees those up to itself
        {"name": "attend_prompts", "kind": "attend", "cache": "bf16", "streams": 8, "queries": 2000, "ragged": True, "keys": 4000,
         "Hq": 16, "Hk": 4, "D": 64, "page": 32, "causal": True, "ret": 0, "h": 1, "w": 1},
        # a chunk of the preview grid in fp32, one chunk of keys retrieved
        {"name": "attend_preview_f32", "kind": "attend", "cache": "f32", "streams": 1, "queries": 1170, "ragged": False, "keys": 7020,
         "Hq": 12, "Hk": 12, "D": 128, "page": 64, "causal": False, "ret": 3, "h": 15, "w": 26},
        # one layer of the Wan-1.3B loop closure (two retrieved chunks) over 8 bits
        {"name": "attend_wan13b", "kind": "attend", "cache": "fp8", "streams": 1, "queries": 4680, "ragged": False, "keys": 28080,
         "Hq": 12, "Hk": 12, "D": 128, "page": 64, "causal": False, "ret": 6, "h": 30, "w": 52},
        # a window at 720p with 40 heads, the largest
        {"name": "attend_720p", "kind": "attend", "cache": "fp8", "streams": 1, "queries": 10800, "ragged": False, "keys": 43200,
         "Hq": 40, "Hk": 40, "D": 128, "page": 128, "causal": False, "ret": 3, "h": 45, "w": 80},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.4:
        while True:
            few = rng.random() < 0.4
            c = {"kind": "append", "cache": rng.choice(["fp8", "fp8", "bf16", "f32"]), "streams": _log(rng, 1, 256) if few else _log(rng, 1, 12),
                 "tokens": rng.randint(1, 4) if few else _log(rng, 5, 10800), "ragged": rng.random() < 0.5,
                 "before": _log(rng, 1, 400 if few else 4000), "H": _log(rng, 1, 40), "D": rng.choice([64, 128, 128]),
                 "page": rng.choice([32, 64, 128, 256]), "packed": rng.random() < 0.5, "given": rng.random() < 0.5,
                 "h": _log(rng, 1, 45), "w": _log(rng, 1, 80)}
            if (c["tokens"] + c["before"]) * c["streams"] * c["H"] * c["D"] <= 11100 * 40 * 128:
                return c
    while True:
        few = rng.random() < 0.4
        c = {"kind": "attend", "cache": rng.choice(["fp8", "fp8", "fp8", "bf16", "f32"]), "streams": _log(rng, 1, 64) if few else _log(rng, 1, 6),
             "queries": rng.randint(1, 8) if few else _log(rng, 9, 10800), "ragged": rng.random() < 0.5, "keys": _log(rng, 33, 50000),
             "Hq": 0, "Hk": _log(rng, 1, 40), "D": rng.choice([64, 128, 128]), "page": rng.choice([32, 64, 128, 256]),
             "causal": rng.random() < 0.4, "ret": 0, "h": _log(rng, 5, 45), "w": _log(rng, 7, 80)}
        c["Hq"] = c["Hk"] * rng.choice([1, 1, 2, 4, 5, 8])
        c["ret"] = min(rng.choice([0, 0, 3, 6]), c["keys"] // (c["h"] * c["w"]))
        most = 1e9 if c["cache"] == "f32" else 1.86e10
        if c["queries"] <= c["keys"] and c["streams"] * c["Hk"] * c["D"] * c["keys"] <= 43200 * 40 * 128 and _pairs(c) * c["Hq"] <= most:
            return c


# ---- lengths --------------------------------------------------------------


def _uneven(i, most, least):
    """Stream i's share of a ragged batch, from least to most."""
    return least + int((most - least) * ((0.35 + 0.6180339887 * i) % 1.0))


def _new(c):
    """New tokens (queries) of every stream."""
    n = c["tokens"] if c["kind"] == "append" else c["queries"]
    return [_uneven(i, n, 1) if c["ragged"] else n for i in range(c["streams"])]


def _held(c):
    """Tokens that every stream's pages hold before (append) or in all (attend)."""
    if c["kind"] == "append":
        return [_uneven(i, c["before"], 0) if c["ragged"] else c["before"] for i in range(c["streams"])]
    return [max(n, _uneven(i + 3, c["keys"], c["keys"] // 4)) if c["ragged"] else c["keys"] for i, n in enumerate(_new(c))]


def _pairs(c):
    """(query, key) pairs of a head, over all streams."""
    return float(sum(n * L - (n * (n - 1) // 2 if c["causal"] else 0) for n, L in zip(_new(c), _held(c))))


def _bands(D):
    """Rotary pairs of time, row and column: the last two a sixth of the head each (22, 21, 21 at D 128)."""
    return D // 2 - 2 * (D // 6), D // 6, D // 6


# ---- inputs ---------------------------------------------------------------


def _values(g, dtype, n, H, D):
    x = torch.randn(n, H, D, generator=g, device=DEV)
    return (x * torch.exp2(torch.arange(H, device=DEV) * 1.7 % 4 - 2)[:, None]).to(dtype)


def _exponent(m):
    """Smallest integer e >= LOW with m <= 448 2^e, as fp32; m >= 0 and finite."""
    frac, e = torch.frexp(m)  # m = frac 2^e, frac in [1/2, 1); 448 = 0.875 * 2^9
    return torch.where(m > 0, e - 9 + (frac > 0.875).int(), LOW).clamp(min=LOW).float()


def _pages(g, c, n_pages):
    """A pool of pages that hold values: [n_pages, H, page, D], and the scales [n_pages, H, page / 32] of 8 bits."""
    H, D, P = c.get("Hk") or c["H"], c["D"], c["page"]
    if c["cache"] != "fp8":
        return _values(g, STORED[c["cache"]], n_pages * P, H, D).view(n_pages, P, H, D).transpose(1, 2).contiguous(), None
    x = _values(g, torch.float32, n_pages * P, H, D).view(n_pages, P // BLOCK, BLOCK, H, D).permute(0, 3, 1, 2, 4)
    e = _exponent(x.abs().amax((3, 4)))
    code = (x * torch.exp2(-e)[..., None, None]).to(E4M3).reshape(n_pages, H, P, D)
    return code, (e + 127).to(torch.uint8).view(E8M0)


def prepare(case, seed):
    g, c = torch.Generator(device=DEV).manual_seed(seed), case
    append = c["kind"] == "append"
    new, held, P = _new(c), _held(c), c["page"]
    B, n, D = c["streams"], sum(new), c["D"]
    in_all = [L + m if append else L for L, m in zip(held, new)]
    need = [-(-L // P) for L in in_all]
    n_pages = sum(need) + 2
    order = torch.randperm(n_pages, generator=g, device=DEV).int().cpu()
    table = torch.full((B, max(need)), -1, dtype=torch.int32)
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m]
        at += m
    s = {"case": c, "n_pages": n_pages, "table": table.to(DEV), "len": torch.tensor(held, dtype=torch.int32, device=DEV)}
    cu = torch.tensor([0] + new).cumsum(0)
    s["cu"] = cu.int().to(DEV) if c["ragged"] else None  # even shares need no list
    s["stream"] = torch.repeat_interleave(torch.arange(B), torch.tensor(new)).to(DEV)
    s["place"] = (torch.arange(n) - cu[:-1][s["stream"].cpu()]).to(DEV)
    for name in ("k", "v"):
        s["cache_" + name], s["scale_" + name] = _pages(g, c, n_pages)
    if append:
        dt, H = GIVEN[c["cache"]], c["H"]
        if c["packed"]:  # the projection's rows hold q, k and v one after the other
            rows = torch.stack([_values(g, dt, n, H, D) for _ in range(3)], 1)
            s["k"], s["v"] = rows[:, 1], rows[:, 2]
        else:
            s["k"], s["v"] = _values(g, dt, n, H, D), _values(g, dt, n, H, D)
        s["pos"] = None
        if c["given"]:
            s["pos"] = torch.stack([torch.randint(0, m, (n,), generator=g, device=DEV) for m in (1000, max(2, c["h"]), max(2, c["w"]))], 1).int()
        s["axis"] = torch.cat([torch.full((m,), a) for a, m in enumerate(_bands(D))]).to(DEV)
        s["omega"] = torch.cat([THETA ** (-torch.arange(m, dtype=torch.float64) / m) for m in _bands(D)]).to(DEV)
        return s
    s["q"] = torch.randn(n, c["Hq"], D, generator=g, device=DEV).to(GIVEN[c["cache"]])
    # queries are their stream's last tokens
    s["seen"] = (s["len"][s["stream"]] - torch.tensor(new, device=DEV)[s["stream"]] + s["place"] + 1).int() if c["causal"] else None
    s["slot"] = s["uv"] = s["idx"] = None
    S, hw = c["ret"], c["h"] * c["w"]
    if S:
        slot = torch.full((B, -(-max(held) // hw)), -1, dtype=torch.int32)
        first = min(F, slot.shape[1] - S)  # retrieved frames stand behind the anchor chunk
        slot[:, first:first + S] = torch.arange(S, dtype=torch.int32)
        tok = s["place"] % hw
        uv = torch.stack([tok % c["w"] + 0.5, tok // c["w"] + 0.5], -1) + 3.0 * torch.randn(S, n, 2, generator=g, device=DEV)
        inside = (uv >= 0).all(-1) & (uv[..., 0] < c["w"]) & (uv[..., 1] < c["h"])
        shown = inside & (torch.rand(S, n, generator=g, device=DEV) > 0.1)
        s["slot"], s["uv"] = slot.to(DEV), uv.contiguous()
        s["idx"] = torch.where(shown, uv[..., 1].floor().int() * c["w"] + uv[..., 0].floor().int(), -4).int().contiguous()
    return s


# ---- the plain form -------------------------------------------------------


def _plain_append(s, c):
    P, D, B = c["page"], c["D"], c["streams"]
    at = s["len"].long()[s["stream"]] + s["place"]  # position in the cache
    if s["pos"] is not None:
        pos = s["pos"].double()
    else:
        hw = c["h"] * c["w"]
        pos = torch.stack([T0 + at // hw, at % hw // c["w"], at % c["w"]], 1).double()
    phi = pos[:, s["axis"]] * s["omega"]  # angles in 64 bits
    co, si = phi.cos().float()[:, None], phi.sin().float()[:, None]
    k = s["k"].float()
    a, b, m = k[..., 0:2 * len(s["omega"]):2], k[..., 1:2 * len(s["omega"]):2], 2 * len(s["omega"])
    k = torch.cat([torch.stack([a * co - b * si, a * si + b * co], -1).flatten(-2), k[..., m:]], -1)
    page, row = s["table"][s["stream"], at // P].long(), at % P
    for x, cache, scale in ((k, s["cache_k"], s["scale_k"]), (s["v"].float(), s["cache_v"], s["scale_v"])):
        if scale is None:
            cache[page, :, row] = x.to(cache.dtype)
            continue
        per = s["table"].shape[1] * P // BLOCK  # blocks of a stream
        block = s["stream"] * per + at // BLOCK
        top = torch.zeros(B * per, c["H"], device=DEV).index_reduce_(0, block, torch.where(x.isfinite(), x.abs(), 0.0).amax(-1), "amax")
        e = _exponent(top)  # [blocks, H]
        # the first block of a stream may hold tokens already: its scale only grows, its codes are rounded again
        j = torch.arange(BLOCK, device=DEV)
        first = s["len"].long() // BLOCK * BLOCK
        page0, row0 = s["table"].gather(1, (first // P)[:, None])[:, 0].long(), first % P
        held = (j < (s["len"] - first)[:, None])[:, None, :, None]
        byte, code = scale.view(torch.uint8), cache.view(torch.uint8)
        was = byte[page0, :, row0 // BLOCK].float() - 127
        b0 = torch.arange(B, device=DEV) * per + first // BLOCK
        e[b0] = torch.where(held.any(2)[..., 0], torch.maximum(e[b0], was), e[b0])
        rows = row0[:, None] + j
        old = code[page0[:, None], :, rows].transpose(1, 2).contiguous()  # [B, H, 32, D]
        again = (old.view(E4M3).float() * torch.exp2(was - e[b0])[..., None, None]).to(E4M3).view(torch.uint8)
        code[page0[:, None], :, rows] = torch.where(held, again, old).transpose(1, 2)
        byte[page, :, row // BLOCK] = (e[block] + 127).to(torch.uint8)
        code[page, :, row] = (x * torch.exp2(-e[block])[..., None]).to(E4M3).view(torch.uint8)
    new = torch.bincount(s["stream"], minlength=B)
    return s["cache_k"], s["cache_v"], s["scale_k"], s["scale_v"], (s["len"] + new).int()


def _dense(cache, scale, table):
    """What the pages of a stream hold, one after the other: [B, H, tokens, D] in fp32."""
    t = table.clamp(min=0).long()
    if scale is None:
        x = cache[t].float()
    else:
        x = cache.view(torch.uint8)[t].view(E4M3).float().unflatten(3, (-1, BLOCK))
        x = (x * torch.exp2(scale.view(torch.uint8)[t].float() - 127)[..., None, None]).flatten(3, 4)
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attend(s, c):
    B, Hq, Hk, D, S = c["streams"], c["Hq"], c["Hk"], c["D"], c["ret"]
    Lk, m = max(_held(c)), max(_new(c))
    st, pl = s["stream"], s["place"]
    k, v = (_dense(s["cache_" + x], s["scale_" + x], s["table"])[:, :, :Lk].flatten(0, 1).contiguous() for x in ("k", "v"))
    q = torch.zeros(B, m, Hq, D, device=DEV)
    q[st, pl] = s["q"].float()
    q = q.unflatten(2, (Hk, -1)).permute(0, 2, 1, 3, 4).reshape(B * Hk, -1, D)  # rows: (query, head of the group)
    a = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(D ** -0.5).view(B, Hk, m, Hq // Hk, Lk)
    if S:  # minus the squared distance of a key's token from the query's correspondence in its frame
        hw, w = c["h"] * c["w"], c["w"]
        uv, ok = torch.zeros(S, B, m, 2, device=DEV), torch.zeros(S, B, m, dtype=torch.bool, device=DEV)
        uv[:, st, pl], ok[:, st, pl] = s["uv"], s["idx"] >= 0
        j = torch.arange(Lk, device=DEV)
        sl = s["slot"].long()[:, j // hw]  # [B, Lk]
        x, y = (j % hw % w + 0.5), (j % hw // w + 0.5)
        for i in range(S):
            dx, dy = x - uv[i, :, :, None, 0], y - uv[i, :, :, None, 1]
            bias = (dx * dx + dy * dy).mul_(-LAM / (2 * SIGMA ** 2))
            a.add_(torch.where((sl == i)[:, None] & ok[i][..., None], bias, 0.0)[:, None, :, None])
    seen = torch.zeros(B, m, dtype=torch.int32, device=DEV)
    seen[st, pl] = s["len"][st] if s["seen"] is None else torch.minimum(s["seen"], s["len"][st])
    a.masked_fill_((torch.arange(Lk, device=DEV) >= seen[..., None])[:, None, :, None], -math.inf)
    top = a.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)  # a query that sees no key
    p = a.sub_(top).exp_()
    l = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(B * Hk, -1, Lk), v).view(B, Hk, m, -1, D) / torch.where(l > 0, l, 1.0)
    o = o.permute(0, 2, 1, 3, 4).flatten(2, 3)[st, pl].to(s["q"].dtype)
    lse = (top + l.log())[..., 0].permute(0, 2, 1, 3).flatten(2, 3)[st, pl]
    return o, lse.t().contiguous()


# ---- one pass -------------------------------------------------------------


def run(state):
    s, c = state, state["case"]
    if not own:
        return _plain_append(s, c) if c["kind"] == "append" else _plain_attend(s, c)
    import paper_2607_21848_amd as rv
    pages = (s["cache_k"], s["cache_v"], s["table"], s["len"])
    if c["kind"] == "append":
        n = rv.append_paged_kv(s["k"], s["v"], *pages, cu=s["cu"], scale_k=s["scale_k"], scale_v=s["scale_v"], pairs=_bands(c["D"]),
                               theta=THETA, h=c["h"], w=c["w"], t0=T0, pos=s["pos"])
        return s["cache_k"], s["cache_v"], s["scale_k"], s["scale_v"], n
    return rv.paged_chunk_attention(s["q"], *pages, cu=s["cu"], scale_k=s["scale_k"], scale_v=s["scale_v"], visible=s["seen"],
                                    kv_frame_slot=s["slot"], corr_uv=s["uv"], corr_idx=s["idx"], h=c["h"], w=c["w"],
                                    softmax_scale=c["D"] ** -0.5, lam=LAM, sigma=SIGMA)


# ---- what a pass cannot do without ----------------------------------------


def work(case):
    c = case
    n, size, given = sum(_new(c)), SIZE[c["cache"]], 4 if c["cache"] == "f32" else 2
    if c["kind"] == "append":
        rows = 2.0 * c["H"] * c["D"]
        scales = 2.0 * c["H"] * n / BLOCK if size == 1 else 0
        return {"bytes": n * rows * (given + size) + scales + (12 * n if c["given"] else 0), "flops": 3 * n * rows}
    held = float(sum(_held(c)))
    kv = held * 2 * c["Hk"] * (c["D"] * size + (1 / BLOCK if size == 1 else 0))
    return {"bytes": kv + n * c["Hq"] * (2 * c["D"] * given + 4) + 12 * c["ret"] * n, "flops": 4.0 * c["D"] * c["Hq"] * _pairs(c)}


# ---- the same in 64 bits --------------------------------------------------


def _exact_append(c, s):
    P, D, H, new, held = c["page"], c["D"], c["H"], _new(c), _held(c)
    full = {}
    for name in ("k", "v"):
        full[name] = s["cache_" + name].float().double()
        if s["scale_" + name] is not None:
            full["scale_" + name] = s["scale_" + name].float().double()
    table, at = s["table"].cpu(), 0
    for i, (m, L) in enumerate(zip(new, held)):
        p = torch.arange(L, L + m)
        if s["pos"] is not None:
            pos = s["pos"][at:at + m].double()
        else:
            frame, inside = p // (c["h"] * c["w"]), p % (c["h"] * c["w"])
            pos = torch.stack([T0 + frame, inside // c["w"], inside % c["w"]], 1).double().to(DEV)
        turn = torch.cat([pos[:, a:a + 1] * torch.tensor([THETA ** (-j / b) for j in range(b)], device=DEV, dtype=torch.float64)
                          for a, b in enumerate(_bands(D))], 1)[:, None]
        k = s["k"][at:at + m].double()
        b = 2 * turn.shape[-1]
        z = torch.view_as_complex(k[..., :b].unflatten(-1, (-1, 2)).contiguous()) * torch.polar(torch.ones_like(turn), turn)
        k[..., :b] = torch.view_as_real(z).flatten(-2)
        page, row = table[i, p // P].long().to(DEV), (p % P).to(DEV)
        for name, x in (("k", k), ("v", s["v"][at:at + m].double())):
            to = full[name]
            if "scale_" + name not in full:
                to[page, :, row] = x
                continue
            # a scale is the least power of two that brings its block's largest value to 448 or below
            blocks = (p // BLOCK - L // BLOCK).to(DEV)
            most = torch.stack([x[blocks == j].abs().amax((0, 2)) for j in range(int(blocks[-1]) + 1)])
            e = torch.ceil(torch.log2(most / 448)).clamp(min=LOW)
            scale = full["scale_" + name]
            if L % BLOCK:
                pg, r = int(table[i, L // P]), L % P // BLOCK
                e[0] = torch.maximum(e[0], torch.log2(scale[pg, :, r]))
                r0 = L // BLOCK * BLOCK % P
                to[pg, :, r0:r0 + L % BLOCK] *= (scale[pg, :, r] / torch.exp2(e[0]))[:, None, None]
            scale[page, :, row // BLOCK] = torch.exp2(e[blocks])
            to[page, :, row] = x * torch.exp2(-e[blocks])[..., None]
        at += m
    return full["k"], full["v"], full.get("scale_k"), full.get("scale_v"), None


def _exact_attend(c, s):
    Hq, Hk, D, G, hw = c["Hq"], c["Hk"], c["D"], c["Hq"] // c["Hk"], c["h"] * c["w"]
    n, at = sum(_new(c)), 0
    o, lse = torch.empty(n, Hq, D, device=DEV, dtype=torch.float64), torch.empty(Hq, n, device=DEV, dtype=torch.float64)
    for i, (m, L) in enumerate(zip(_new(c), _held(c))):
        pages = s["table"][i, :-(-L // c["page"])].long()
        rows = slice(at, at + m)
        j = torch.arange(L, device=DEV)
        bias = None
        if c["ret"]:
            bias = torch.zeros(m, L, device=DEV, dtype=torch.float64)
            kx, ky = (j % hw % c["w"]).double() + 0.5, torch.div(j % hw, c["w"], rounding_mode="floor").double() + 0.5
            for f, slot in enumerate(s["slot"][i].tolist()):
                if slot < 0 or f * hw >= L:
                    continue
                u, to = s["uv"][slot, rows].double(), slice(f * hw, min(L, (f + 1) * hw))
                d = -LAM * ((u[:, :1] - kx[to]) ** 2 + (u[:, 1:] - ky[to]) ** 2) / (2 * SIGMA ** 2)
                bias[:, to] = torch.where((s["idx"][slot, rows] >= 0)[:, None], d, 0.0)
        hidden = None if s["seen"] is None else j >= s["seen"][rows][:, None]
        for hk in range(Hk):
            kv = []
            for name in ("k", "v"):
                x = s["cache_" + name][pages, hk] if s["scale_" + name] is None else s["cache_" + name].view(torch.uint8)[pages, hk].view(E4M3)
                x = x.float().double()
                if s["scale_" + name] is not None:
                    x = x * s["scale_" + name].view(torch.uint8)[pages, hk].view(E8M0).float().double().repeat_interleave(BLOCK, 1)[..., None]
                kv.append(x.flatten(0, 1)[:L])
            for h in range(hk * G, (hk + 1) * G):
                a = s["q"][rows, h].double() @ kv[0].t().contiguous() / math.sqrt(D)
                if bias is not None:
                    a += bias
                if hidden is not None:
                    a.masked_fill_(hidden, -math.inf)
                lse[h, rows] = torch.logsumexp(a, 1)
                o[rows, h] = (a - lse[h, rows, None]).exp_() @ kv[1]
        at += m
    return o, lse


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_append(case, s) if case["kind"] == "append" else _exact_attend(case, s)
