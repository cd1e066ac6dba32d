"""Paged caches for the tests: pools with whatever earlier sequences left in them, and the operators' definitions in 64 bits."""
import math

import numpy as np
import torch

from paper_2602_02199_b200 import binding as Bn

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def build(lens, *, H, G, D=128, page_size=16, dtype="bf16", token_major=False, weights=True, max_pages=None, spare=3, seed=0, scale=1.0,
          stale=math.nan, seen=None, whole_table=False):
    """A PagedKV of sequences of the given lengths. Rows that no sequence holds are `stale`, table entries without a page
    (all but `whole_table` gives) are numbers far outside the pool."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = len(lens)
    need = [-(-x // page_size) for x in lens]
    max_pages = max(max_pages or 0, max(need), 1)
    if whole_table:
        need = [max_pages] * n
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((n, max_pages), 1 << 30, dtype=torch.int32, device="cuda")
    at = 0
    for b in range(n):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    shape = (n_pages, page_size, H, D) if token_major else (n_pages, H, page_size, D)
    k = (scale * torch.randn(shape, generator=gen, device="cuda")).to(TYPES[dtype])
    v = torch.randn(shape, generator=gen, device="cuda").to(TYPES[dtype])
    if token_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    w = torch.rand(n_pages, H, page_size, generator=gen, device="cuda")
    pos = torch.full((n_pages, H, page_size), -7, dtype=torch.int32, device="cuda")
    held = torch.zeros(n_pages, page_size, dtype=torch.bool, device="cuda")
    for b in range(n):
        j = torch.arange(lens[b], device="cuda")
        page, off = table[b, j // page_size].long(), j % page_size
        held[page, off] = True
        pos[page, :, off] = j.to(torch.int32)[:, None].expand(-1, H)
    if stale is not None:
        for x in (k, v):
            x.transpose(1, 2)[~held] = stale
    state = torch.tensor([lens, lens if seen is None else seen], dtype=torch.int32, device="cuda")
    cache = Bn.PagedKV(k, v, table, n_q_heads=H * G, weights=w if weights else None, pos=pos, state=state)
    return cache, gen


def queries(cache, gen, scale=1.0, strided=False):
    n, hq, d = cache._q_shape
    if strided:
        x = (scale * torch.randn(n, 3, hq, d + 8, generator=gen, device="cuda")).to(cache.k_pages.dtype)
        return x[:, 1, :, :d]
    return (scale * torch.randn(n, hq, d, generator=gen, device="cuda")).to(cache.k_pages.dtype)


def rows(cache, b, length):
    """Pages and rows in them of a sequence's entries."""
    j = torch.arange(length, device="cuda")
    return cache.page_table[b, j // cache.cfg.page_size].long(), j % cache.cfg.page_size


def attention64(cache, q, scale=None):
    """(out, lse, what every weight grows by, bounds of the errors of the three) in 64 bits.

    Bounds. A score is a sum of D products of 16-bit numbers, exact in fp32, added up in D / 16 steps of an MMA, two chains of
    them and their sum, each off by at most 2^-22 of the magnitudes added, S = sum |q_i k_i| scale: d = (D / 16 + 4) 2^-22 S at
    most. A weight e^x is then off by d, relatively, and by 2^-21 for the exponential, its argument's rounding (in d) and the
    splitting into terms; the sums of len / 64 blocks and of the parts of up to 320 CTAs round once each, 2^-24, and the MMA's
    own sum of 16 products 2^-20. Numerator and denominator both: twice."""
    c = cache.cfg
    H, G, D, n = c.n_kv_heads, c.n_q_heads // c.n_kv_heads, c.head_dim, c.n_seqs
    scale = scale or D ** -0.5
    lens = cache.lens.tolist()
    out = torch.zeros(n, H * G, D, dtype=torch.float64, device="cuda")
    lse = torch.full((n, H * G), -math.inf, dtype=torch.float64, device="cuda")
    grow = torch.zeros(c.n_pages, H, c.page_size, dtype=torch.float64, device="cuda")
    t_out, t_lse, t_grow = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(grow)
    for b, length in enumerate(lens):
        if not length:
            continue
        page, off = rows(cache, b, length)
        k, v = (x[page, :, off].double().transpose(0, 1) for x in (cache.k_pages, cache.v_pages))      # [H][len][D]
        qq = q[b].double().view(H, G, D)
        x = torch.einsum("hgd,hld->hgl", qq, k) * scale
        d = torch.einsum("hgd,hld->hgl", qq.abs(), k.abs()) * scale * ((D / 16 + 4) * 2.0 ** -22)
        z = torch.logsumexp(x, -1)
        p = torch.exp(x - z[..., None])
        rel = 2 * (d.amax(-1) + 2.0 ** -20 + 2.0 ** -21 + (length / 64 + 340) * 2.0 ** -24)               # [H][G]
        out[b] = torch.einsum("hgl,hld->hgd", p, v).reshape(H * G, D)
        t_out[b] = (torch.einsum("hgl,hld->hgd", p, v.abs()) * rel[..., None]).reshape(H * G, D)
        lse[b] = z.reshape(-1)
        t_lse[b] = (rel + 2.0 ** -22 * z.abs()).reshape(-1)
        grow[page, :, off] = p.sum(1).T
        t_grow[page, :, off] = (p * (rel[..., None] + d)).sum(1).T
    return out, lse, grow, t_out, t_lse, t_grow


def check_attention(cache, q, *, out_dtype=None, accumulate=False, scale=None, softmax_scale=0.0):
    want, lse64, grow, t_out, t_lse, t_grow = attention64(cache, q, scale)
    before = None if cache.weights is None else cache.weights.clone()
    out = None if out_dtype is None else torch.full(q.shape, math.nan, dtype=out_dtype, device="cuda")
    lse = torch.full(q.shape[:2], math.nan, dtype=torch.float32, device="cuda")
    out = cache.laser_kv_paged_attention(q, softmax_scale=softmax_scale, accumulate=accumulate, out=out, lse=lse)
    cache.laser_kv_paged_poll_status()
    tol = t_out + torch.finfo(out.dtype).eps / 2 * (want.abs() + t_out) + torch.finfo(out.dtype).smallest_normal * torch.finfo(out.dtype).eps
    err = (out.double() - want).abs()
    assert bool((err <= tol).all()), ((err - tol).max().item(), (err / tol.clamp(min=1e-30)).max().item())
    empty = torch.isinf(lse64)
    assert bool((lse[empty] == -math.inf).all()) and bool((out[empty] == 0).all())
    assert bool(((lse.double() - lse64).abs()[~empty] <= t_lse[~empty]).all())
    if accumulate:
        w = before.double() + grow
        assert bool(((cache.weights.double() - w).abs() <= t_grow + 2.0 ** -24 * w.abs()).all())
        assert torch.equal(cache.weights[grow == 0], before[grow == 0])
    elif before is not None:
        assert torch.equal(cache.weights, before)
    return out


def snapshot(cache):
    """Everything that calls may change, on the host; rows as bits."""
    bits = lambda x: x.contiguous().view(torch.int16).cpu().numpy().copy()
    return dict(k=bits(cache.k_pages), v=bits(cache.v_pages), pos=cache.pos.cpu().numpy().copy(), state=cache.state.cpu().numpy().copy(),
                w=None if cache.weights is None else cache.weights.cpu().numpy().copy(), table=cache.page_table.cpu().numpy().copy())


def same(a, b):
    for x in ("k", "v", "pos", "state", "w"):
        if a[x] is None:
            assert b[x] is None
            continue
        x_a, x_b = (y.view(np.int32) if y.dtype == np.float32 else y for y in (a[x], b[x]))
        assert np.array_equal(x_a, x_b), (x, np.argwhere(x_a != x_b)[:4].tolist())


def append_plain(s, page_size, k, v, counts, w=None, pos=None):
    """The snapshot after an append; k, v [n][H][m][D] as bits."""
    n, H = k.shape[:2]
    for b in range(n):
        held, seen = s["state"][:, b]
        for i in range(counts[b]):
            page, off = s["table"][b, (held + i) // page_size], (held + i) % page_size
            s["k"][page, :, off], s["v"][page, :, off] = k[b, :, i], v[b, :, i]
            s["pos"][page, :, off] = seen + i if pos is None else pos[b, :, i]
            if s["w"] is not None:
                s["w"][page, :, off] = 0 if w is None else w[b, :, i]
        s["state"][0, b] += counts[b]
        if pos is None:
            s["state"][1, b] += counts[b]
    return s


def evict_plain(s, page_size, keep, anchors, recent):
    n, H = s["table"].shape[0], s["pos"].shape[1]
    for b in range(n):
        length, seen = (int(x) for x in s["state"][:, b])
        if length <= keep:
            continue
        j = np.arange(length)
        page, off = s["table"][b, j // page_size], j % page_size
        for h in range(H):
            w, pos = s["w"][page, h, off].astype(np.float64), s["pos"][page, h, off]
            w[np.isnan(w)] = -np.inf
            w[(pos < anchors) | (pos >= seen - recent)] = np.inf
            stay = np.zeros(length, dtype=bool)
            stay[np.argsort(-w, kind="stable")[:keep]] = True
            holes, movers = np.flatnonzero(~stay[:keep]), np.flatnonzero(stay[keep:])[::-1] + keep
            assert len(holes) == len(movers)
            for x in ("k", "v", "w", "pos"):
                s[x][page[holes], h, off[holes]] = s[x][page[movers], h, off[movers]]
        s["state"][0, b] = keep
    return s
