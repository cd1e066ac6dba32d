"""The operators of a paged key-value cache, as cases that can be timed and compared.

A paged cache keeps the entries of many sequences in one pool of pages, `page_size` entries of every KV head each; a
table names each sequence's pages. Next to an entry's key and value stand its position and, where wanted, the attention
weight it has received so far. Three kinds of case, told apart by `kind`:

  attention  one new token per sequence against the entries of its pages; with `weights` every entry's accumulated
             weight grows by what the group's query heads give it
  append     new entries behind each sequence's last one (a token of every sequence, or prompts)
  evict      new entries are appended, then every (sequence, KV head) is brought back to `keep` entries: those of the
             first `anchors` positions, of the last `recent` ones, and the ones of the largest accumulated weight. The
             last kept entry behind `keep` goes to the first slot that an evicted one left, and so on

The lengths of a case's sequences are spread evenly over the logarithm from `shortest` to `longest`; the seed deals them
out. Slots that no sequence holds keep what earlier sequences left there.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _attention(name, **kw):
    c = dict(name=name, kind="attention", dtype="bf16", out="fp32", n_seqs=1, n_kv_heads=8, group=4, head_dim=128, page_size=16,
             shortest=1637, longest=1637, empty=0, weights=False, token_major=False)
    c.update(kw)
    return c


def _append(name, **kw):
    c = dict(name=name, kind="append", dtype="bf16", n_seqs=1, n_kv_heads=8, group=4, head_dim=128, page_size=16, shortest=512,
             longest=512, n_new=1, ragged=False, seeded=False, token_major=False)
    c.update(kw)
    return c


def _evict(name, **kw):
    c = dict(name=name, kind="evict", dtype="bf16", n_seqs=1, n_kv_heads=8, group=4, head_dim=128, page_size=16, keep=2048, n_new=1,
             anchors=4, recent=256, token_major=False)
    c.update(kw)
    return c


def listed():
    return [
        # a token of one conversation whose 4k-token prompt was compressed: the smallest call, launch and latency count
        _attention("attn_short"),
        # a serving batch of mixed lengths in small pages, two of its rows not in use; fp16, results in the model's type
        _attention("attn_ragged", n_seqs=32, shortest=1, longest=16001, empty=2, dtype="fp16", out="fp16"),
        # one long document, uncompressed, in large pages
        _attention("attn_long", page_size=64, shortest=131071, longest=131071, out="bf16"),
        # narrow heads, sixteen query heads to a KV head, pages as a projection leaves them (token after token)
        _attention("attn_wide_group", n_seqs=24, n_kv_heads=2, group=16, head_dim=64, page_size=32, shortest=700, longest=9000,
                   token_major=True, out="bf16"),
        # a full serving batch of long contexts: the largest call
        _attention("attn_large", n_seqs=64, page_size=32, shortest=4000, longest=24000, out="bf16"),
        # decoding with accumulated weights over caches held at a budget
        _attention("attn_weights", n_seqs=16, shortest=2049, longest=2049, weights=True),
        # the same over long caches, groups of seven
        _attention("attn_weights_long", n_seqs=4, n_kv_heads=4, group=7, page_size=64, dtype="fp16", shortest=20000, longest=48000,
                   weights=True, out="fp16"),
        # a decoded token of every sequence of a batch
        _append("append_token", n_seqs=64, shortest=100, longest=16000),
        # prompts of different lengths behind what is cached already, weights from the observation window
        _append("append_prompts", n_seqs=6, shortest=1, longest=4000, n_new=16000, ragged=True, seeded=True, token_major=True),
        # decoding at a budget: one entry in, one entry out
        _evict("evict_step", n_seqs=16),
        # blockwise prefill at a budget: a block of 4096 in, down to 8192 again
        _evict("evict_block", keep=8192, n_new=4096, anchors=1024, recent=1024, page_size=64),
        # a batch of long contexts
        _evict("evict_large", n_seqs=8, keep=32768, n_new=8192, anchors=4096, recent=4096, page_size=64, dtype="fp16"),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "append", "evict"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "fp16"]), n_kv_heads=rng.choice([1, 2, 4, 5, 8]), head_dim=rng.choice([64, 128, 128, 256]),
             page_size=rng.choice([8, 16, 32, 64, 128]), token_major=rng.random() < 0.3)
    if kind == "attention":
        c["group"] = rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16, 20])
        c["n_seqs"] = _spread(rng, 1, 96)
        most = min(131072, (96 << 20) // (c["n_seqs"] * c["n_kv_heads"] * c["head_dim"] // 8))
        c["longest"] = _spread(rng, 1, most)
        c["shortest"] = _spread(rng, 1, c["longest"])
        c["empty"] = rng.choice([0, 0, 1]) if c["n_seqs"] > 1 else 0
        c["weights"] = rng.random() < 0.5
        c["out"] = rng.choice(["fp32", c["dtype"]])
    elif kind == "append":
        c["group"] = 1
        c["n_seqs"] = _spread(rng, 1, 96)
        c["n_new"] = _spread(rng, 1, max(1, 60000 // c["n_seqs"]))
        c["longest"] = _spread(rng, 1, 20000)
        c["shortest"] = _spread(rng, 1, c["longest"])
        c["ragged"] = rng.random() < 0.5
        c["seeded"] = rng.random() < 0.5
    else:
        c["group"] = 1
        c["n_seqs"] = _spread(rng, 1, 24)
        c["keep"] = _spread(rng, 16, 200000 // c["n_seqs"])
        c["n_new"] = _spread(rng, 1, max(1, c["keep"]))
        c["recent"] = rng.randint(0, c["keep"] // 2)
        c["anchors"] = rng.randint(0, c["keep"] // 4)
    return c


def _lengths(case):
    if case["kind"] == "evict":
        return [case["keep"]] * case["n_seqs"]
    lo, hi, n = case["shortest"], case["longest"], case["n_seqs"]
    got = [hi if n == 1 else max(1, round(lo * (hi / lo) ** (i / (n - 1)))) for i in range(n)]
    return [0] * case.get("empty", 0) + got[case.get("empty", 0):]


def _counts(case):
    n, most = case["n_seqs"], case["n_new"]
    if not case.get("ragged"):
        return [most] * n
    return [max(1, round(most * (i + 1) / n)) for i in range(n)]


def _pool(gen, case, n_pages, scale, gains):
    """One side of the pool, [n_pages][H][page_size][d] as a view whose rows lie as the case says."""
    h, p, d = case["n_kv_heads"], case["page_size"], case["head_dim"]
    shape = (n_pages, p, h, d) if case["token_major"] else (n_pages, h, p, d)
    x = torch.empty(shape, dtype=TYPES[case["dtype"]], device="cuda").normal_(0.0, scale, generator=gen)
    x = x.transpose(1, 2) if case["token_major"] else x
    return x.mul_(gains[None, :, None, :].to(x.dtype))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dev, n, h, d, p = "cuda", case["n_seqs"], case["n_kv_heads"], case["head_dim"], case["page_size"]
    dtype = TYPES[case["dtype"]]
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device=dev)
    deal = torch.randperm(n, generator=gen, device=dev)
    lens = lens[deal]
    n_new = case.get("n_new", 0)
    longest = max(_lengths(case)) + n_new
    max_pages = -(-longest // p)
    # attention reads the pages that hold entries and no others; the rows that grow own every page of their table
    need = -(-lens // p) if case["kind"] == "attention" else torch.full_like(lens, max_pages)
    n_pages = sum(-(-x // p) for x in _lengths(case)) if case["kind"] == "attention" else n * max_pages
    n_pages += 3
    order = torch.randperm(n_pages, generator=gen, device=dev).to(torch.int32)
    first = torch.cumsum(need, 0) - need
    at = torch.arange(max_pages, device=dev)
    table = torch.where(at < need[:, None], order[(first[:, None] + at).clamp(max=n_pages - 1)], -1).to(torch.int32).contiguous()
    gains = torch.exp(0.3 * torch.randn(h, d, generator=gen, device=dev))
    s = dict(case=case, dtype=dtype, table=table, k=_pool(gen, case, n_pages, 1.0, gains), v=_pool(gen, case, n_pages, 1.0, gains.flip(0)),
             state=torch.stack([lens, lens]).contiguous(), longest=longest)
    # positions as if nothing had been evicted; weights of the entries: most are small, one in twenty was never attended to
    j = torch.arange(max_pages * p, device=dev)
    owned = (j[None, :] // p) < need[:, None]
    page, off = table.clamp(min=0)[:, j // p].long(), (j % p).expand(n, -1)
    s["pos"] = torch.full((n_pages, h, p), -1, dtype=torch.int32, device=dev)
    s["pos"].transpose(1, 2)[page[owned], off[owned]] = j.to(torch.int32).expand(n, -1)[owned][:, None].expand(-1, h)
    w = torch.exp(2.0 * torch.randn(n_pages, h, p, generator=gen, device=dev) - 4.0)
    w[torch.rand(n_pages, h, p, generator=gen, device=dev) < 0.05] = 0.0
    s["weights"] = w if case["kind"] != "attention" or case["weights"] else None
    if case["kind"] == "attention":
        s["q"] = (2.5 * torch.randn(n, h * case["group"], d, generator=gen, device=dev) / gains.repeat_interleave(case["group"], 0)).to(dtype)
        # unused slots hold what is left there: not even numbers
        held = torch.zeros(n_pages, p, dtype=torch.bool, device=dev)
        valid = j[None, :] < lens[:, None]
        held[page[valid], off[valid]] = True
        s["k"].transpose(1, 2)[~held] = math.nan
        s["v"].transpose(1, 2)[~held] = math.nan
    else:
        shape = (n, n_new, h, d)
        s["k_new"] = torch.randn(shape, generator=gen, device=dev).to(dtype).transpose(1, 2)
        s["v_new"] = torch.randn(shape, generator=gen, device=dev).to(dtype).transpose(1, 2)
        seeded = case["kind"] == "evict" or case["seeded"]
        s["w_new"] = torch.exp(2.0 * torch.randn(n, h, n_new, generator=gen, device=dev) - 4.0) if seeded else None
        s["counts"] = torch.tensor(_counts(case), dtype=torch.int32, device=dev)[deal] if case.get("ragged") else None
        s["state_before"] = s["state"].clone()
    if case["kind"] == "attention":
        s["out"] = torch.empty(s["q"].shape, dtype=TYPES[case["out"]], device=dev)
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=dev)
    if own:
        from paper_2602_02199_b200 import binding
        s["cache"] = binding.PagedKV(s["k"], s["v"], table, n_q_heads=h * case["group"], weights=s["weights"], pos=s["pos"], state=s["state"])
    return s


# ---- the plain form ------------------------------------------------------------------------------
def _slots(s, j):
    """Pages and places in them of entries j [n][m] of every sequence."""
    p = s["case"]["page_size"]
    return torch.gather(s["table"].clamp(min=0), 1, j // p).long(), j % p


def _plain_attention(s):
    c, lens = s["case"], s["state"][0]
    n, h, g, d = c["n_seqs"], c["n_kv_heads"], c["group"], c["head_dim"]
    j = torch.arange(max(s["longest"], 1), device=lens.device).expand(n, -1)
    valid = j < lens[:, None]
    page, off = _slots(s, j.clamp(max=s["table"].shape[1] * c["page_size"] - 1))
    k = s["k"].transpose(1, 2)[page, off].float().masked_fill_(~valid[:, :, None, None], 0.0)      # [n][L][H][d]
    x = torch.matmul(s["q"].float().view(n, h, g, d), k.permute(0, 2, 3, 1)) / math.sqrt(d)
    del k
    x.masked_fill_(~valid[:, None, None, :], -math.inf)
    top = x.amax(-1, keepdim=True).masked_fill_((lens == 0)[:, None, None, None], 0.0)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    v = s["v"].transpose(1, 2)[page, off].float().masked_fill_(~valid[:, :, None, None], 0.0)
    some = (lens > 0)[:, None, None, None]
    out = torch.where(some, torch.matmul(e, v.permute(0, 2, 1, 3)) / total, 0.0).view(n, h * g, d)
    got = dict(out=out.to(TYPES[c["out"]]), lse=torch.where(some, top + torch.log(total), -math.inf).view(n, h * g))
    if c["weights"]:
        add = torch.where(some, e / total, 0.0).sum(2).transpose(1, 2)                                  # [n][L][H]
        s["weights"].transpose(1, 2).index_put_((page, off), add, accumulate=True)
        got["weights"] = s["weights"]
    return got


def _plain_append(s):
    c, lens, seen = s["case"], s["state"][0], s["state"][1]
    n, h, m = c["n_seqs"], c["n_kv_heads"], c["n_new"]
    counts = s["counts"] if s["counts"] is not None else torch.full_like(lens, m)
    i = torch.minimum(torch.arange(m, device=lens.device).expand(n, -1), counts[:, None].long() - 1)   # past the end: the last one again
    page, off = _slots(s, lens[:, None].long() + i)
    rows = torch.arange(n, device=lens.device)[:, None]
    s["k"].transpose(1, 2)[page, off] = s["k_new"].transpose(1, 2)[rows, i]
    s["v"].transpose(1, 2)[page, off] = s["v_new"].transpose(1, 2)[rows, i]
    s["pos"].transpose(1, 2)[page, off] = (seen[:, None] + i)[:, :, None].to(torch.int32).expand(-1, -1, h)
    if s["w_new"] is None:
        s["weights"].transpose(1, 2)[page, off] = 0.0
    else:
        s["weights"].transpose(1, 2)[page, off] = s["w_new"].transpose(1, 2)[rows, i]
    s["state"] += counts


def _plain_evict(s):
    c, lens, seen = s["case"], s["state"][0], s["state"][1]
    n, h, keep = c["n_seqs"], c["n_kv_heads"], c["keep"]
    j = torch.arange(s["longest"], device=lens.device).expand(n, -1)
    page, off = _slots(s, j)
    pos = s["pos"].transpose(1, 2)[page, off].transpose(1, 2)                                           # [n][H][L]
    w = s["weights"].transpose(1, 2)[page, off].transpose(1, 2)
    w = torch.where(torch.isnan(w), -math.inf, w)
    w = torch.where((pos < c["anchors"]) | (pos >= (seen[:, None, None] - c["recent"])), math.inf, w)
    w = torch.where(j[:, None, :] < lens[:, None, None], w, -math.inf)
    order = torch.argsort(w, dim=-1, descending=True, stable=True)
    kept = torch.zeros_like(w, dtype=torch.bool).scatter_(2, order[..., :keep], True) & (j[:, None, :] < lens[:, None, None])
    behind = kept & (j[:, None, :] >= keep)
    # the r-th kept entry from the end, and for every slot left before `keep` the one that goes there
    rank = torch.where(behind, behind.sum(-1, keepdim=True) - torch.cumsum(behind, -1), s["longest"])
    source = torch.zeros(n, h, s["longest"] + 1, dtype=torch.int64, device=w.device).scatter_(2, rank, j[:, None, :].expand(-1, h, -1))
    left = ~kept[..., :keep] & (lens > keep)[:, None, None]
    place = j[:, None, :keep].expand(-1, h, -1)
    come = torch.where(left, torch.gather(source, 2, (torch.cumsum(left, -1) - 1).clamp(min=0)), place)  # [n][H][keep]
    heads = torch.arange(h, device=w.device)[None, :, None]
    to = _slots(s, place.reshape(n, -1))
    to = to[0].view(n, h, keep), heads, to[1].view(n, h, keep)
    fr = _slots(s, come.reshape(n, -1))
    fr = fr[0].view(n, h, keep), heads, fr[1].view(n, h, keep)
    for x in (s["k"], s["v"], s["weights"], s["pos"]):
        x[to] = x[fr]
    lens.clamp_(max=keep)


def run(state):
    s, kind = state, state["case"]["kind"]
    if kind == "attention":
        if not own:
            return _plain_attention(s)
        got = dict(out=s["out"], lse=s["lse"])
        s["cache"].laser_kv_paged_attention(s["q"], accumulate=s["case"]["weights"], **got)
        return dict(got, weights=s["weights"]) if s["case"]["weights"] else got
    if kind == "append":
        s["state"].copy_(s["state_before"])          # the sequences are as long as before: the tokens of the last pass are taken back
    if own:
        s["cache"].laser_kv_paged_append(s["k_new"], s["v_new"], counts=s["counts"], weights=s["w_new"])
        if kind == "evict":
            s["cache"].laser_kv_paged_evict(s["case"]["keep"], anchors=s["case"]["anchors"], recent=s["case"]["recent"])
    else:
        _plain_append(s)
        if kind == "evict":
            _plain_evict(s)
    return dict(k=s["k"], v=s["v"], weights=s["weights"], pos=s["pos"], lens=s["state"][0], seen=s["state"][1])


# ---- what one pass cannot do without ------------------------------------------------------------
def work(case):
    lens, h, g, d, p = _lengths(case), case["n_kv_heads"], case["group"], case["head_dim"], case["page_size"]
    n, row = len(lens), 4 * case["head_dim"]                          # a key and a value, two bytes an element
    if case["kind"] == "attention":
        size = 4 if case["out"] == "fp32" else 2
        table = sum(-(-x // p) for x in lens) * 4
        # keys and values, queries, results and their normalisers, lengths and tables; with weights they are read and written
        b = sum(lens) * h * (row + (8 if case["weights"] else 0)) + n * h * g * (d * (2 + size) + 4) + 4 * n + table
        return {"bytes": b, "flops": 4 * sum(lens) * h * g * d}
    new = sum(_counts(case)) if case["kind"] == "append" else n * case["n_new"]
    seeded = case["kind"] == "evict" or case["seeded"]
    b = new * h * (2 * row + 4 + (8 if seeded else 4)) + 16 * n + new // p * 4
    if case["kind"] == "evict":
        # every entry's weight and position, and at least the new entries that have to stay move
        moved = min(case["n_new"], case["recent"])
        b += n * h * ((case["keep"] + case["n_new"]) * 8 + moved * (2 * row + 16))
    return {"bytes": b, "flops": 0}


# ---- the definition in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    n, h, g, d, p = case["n_seqs"], case["n_kv_heads"], case["group"], case["head_dim"], case["page_size"]
    lens, seen, table = s["state"][0].tolist(), s["state"][1].tolist(), s["table"].long()
    if case["kind"] == "attention":
        out = torch.zeros(n, h * g, d, dtype=torch.float64, device="cuda")
        lse = torch.full((n, h * g), -math.inf, dtype=torch.float64, device="cuda")
        weights = s["weights"].double() if case["weights"] else None
        for b, length in enumerate(lens):
            if length == 0:
                continue
            pages = table[b, :-(-length // p)]
            # [H][length][d], head after head and page after page
            k, v = (s[x][pages].transpose(0, 1).reshape(h, -1, d)[:, :length].double() for x in ("k", "v"))
            x = torch.einsum("hgd,hld->hgl", s["q"][b].double().view(h, g, d), k) * d ** -0.5
            z = torch.logsumexp(x, -1)
            prob = torch.exp(x - z[..., None])
            out[b] = torch.einsum("hgl,hld->hgd", prob, v).reshape(h * g, d)
            lse[b] = z.reshape(-1)
            if weights is not None:
                add = torch.zeros(h, pages.numel() * p, dtype=torch.float64, device="cuda")
                add[:, :length] = prob.sum(1)
                weights[pages] += add.view(h, -1, p).transpose(0, 1)
        return dict(out=out, lse=lse, weights=weights) if case["weights"] else dict(out=out, lse=lse)
    got = {x: s[x].double() for x in ("k", "v", "weights")}
    at = s["pos"].clone()
    counts = s["counts"].tolist() if s["counts"] is not None else [case["n_new"]] * n
    for b in range(n):
        slots = torch.arange(lens[b], lens[b] + counts[b], device="cuda")
        page, off = table[b, slots // p], slots % p
        for x in ("k", "v"):
            got[x][page, :, off] = s[x + "_new"][b, :, :counts[b]].transpose(0, 1).double()
        got["weights"][page, :, off] = 0.0 if s["w_new"] is None else s["w_new"][b, :, :counts[b]].T.double()
        at[page, :, off] = (seen[b] + torch.arange(counts[b], device="cuda", dtype=torch.int32))[:, None]
        length, keep = lens[b] + counts[b], case.get("keep", 1 << 30)
        if length <= keep:
            continue
        slots = torch.arange(length, device="cuda")
        page, off = table[b, slots // p], slots % p
        for i in range(h):
            w, q = got["weights"][page, i, off], at[page, i, off]
            w = torch.nan_to_num(w, nan=-math.inf, posinf=math.inf, neginf=-math.inf)
            w[(q < case["anchors"]) | (q >= seen[b] + counts[b] - case["recent"])] = math.inf
            stay = torch.sort(w, descending=True, stable=True).indices[:keep]
            gone = torch.ones(length, dtype=torch.bool, device="cuda")
            gone[stay] = False
            hole = torch.nonzero(gone[:keep]).flatten()
            mover = torch.nonzero(~gone[keep:]).flatten().flip(0) + keep
            for x in (got["k"], got["v"], got["weights"]):
                x[page[hole], i, off[hole]] = x[page[mover], i, off[mover]]
    return dict(k=got["k"], v=got["v"], weights=got["weights"], pos=None, lens=None, seen=None)
