"""The operators of a decode step over a paged KV cache, each as a user's program calls it: sizes,
inputs, a plain form in elementary torch operations and a 64-bit result.

Every case is one call (kind):
  page_map    block tables and slot maps from request lengths
  kv_append   new K and V rows written to their slots, with the key bounds of the pages they touch
  page_score  an upper bound on the logits of every page, from the page's key bounds
  page_select the pages of every KV head that a budget keeps
  decode      attention of one new token per sequence over its pages (all of them, or listed ones)
Fields: batch (sequences or requests), hq, hkv, page (tokens of a page), len (longest sequence, in
tokens), mix (0: every sequence has that length; otherwise lengths differ, and this number picks
them), and per kind: new (tokens of the longest request), fused (K and V are slices of one
projection), budget (pages kept), ties (scores repeat), listed (pages of a list, 0: all), lse.
"""
import math
import random

import torch

own = False

D = 128
_BASE = {"batch": 1, "hq": 32, "hkv": 8, "page": 64, "len": 4096, "mix": 0}


def _case(kind, name=None, **kw):
    extra = {"page_map": {"new": 1}, "kv_append": {"new": 1, "fused": False}, "page_score": {},
             "page_select": {"budget": 32, "ties": False}, "decode": {"listed": 0, "lse": False}}[kind]
    c = {"kind": kind, **_BASE, **extra, **kw}
    return {"name": name, **c} if name else c


def listed():
    return [
        # One decode step of a serving batch: every request adds a token, some of them a page.
        _case("page_map", "map_step_64", batch=64, len=20000, mix=1, new=1),
        # Prompts of different lengths enter an empty or partly filled cache, small pages.
        _case("page_map", "map_prompts_256", batch=256, len=2049, mix=2, new=1500, page=16),
        # A decode step writes its 64 tokens, from the rows of a fused projection.
        _case("kv_append", "append_step_64", batch=64, len=6000, mix=3, new=1, fused=True),
        # A chunk of prompts of uneven lengths is written, page after page.
        _case("kv_append", "append_prompts", batch=19, len=4097, mix=4, new=4097),
        # One sequence of 32K tokens: 256 pages, 8 KV heads.
        _case("page_score", "score_32k", len=32768, page=128),
        # A serving batch of long sequences with small pages: the most bounds that a step reads.
        _case("page_score", "score_batch_64", batch=64, len=131072, mix=5, page=32),
        # One sequence of 32K tokens keeps an eighth of its pages.
        _case("page_select", "select_32k", len=32768, page=128, budget=32),
        # The batch of long sequences, scores with ties, an odd group of query heads.
        _case("page_select", "select_batch_64", batch=64, hq=28, hkv=4, len=131072, mix=6, page=32, budget=129,
              ties=True),
        # The smallest call: one head, a short sequence; latency counts.
        _case("decode", "decode_one_head_1k", hq=1, hkv=1, len=1000, page=16, lse=True),
        # One sequence of 128K tokens on a 32-head, 8-KV-head layer: split over its length.
        _case("decode", "decode_128k", len=131072, page=64),
        # A serving batch of uneven sequences: the most bytes that a step reads.
        _case("decode", "decode_batch_64", batch=64, len=65536, mix=7, page=128),
        # The same kind of batch, 64 listed pages for each KV head, a wide group of query heads.
        _case("decode", "decode_listed_48", batch=48, hq=64, hkv=8, len=65536, mix=8, page=32, listed=64, lse=True),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng: random.Random):
    most = work(listed()[10])["bytes"]
    while True:
        kind = rng.choice(["page_map", "kv_append", "page_score", "page_select", "decode", "decode", "decode"])
        hkv = rng.choice([1, 2, 4, 5, 8])
        c = _case(kind, batch=_log(rng, 1, 256), hkv=hkv, hq=hkv * rng.choice([1, 2, 3, 4, 4, 6, 7, 8, 12, 16, 20]),
                  page=rng.choice([16, 32, 64, 128, 256]), mix=rng.choice([0] + [rng.randrange(1, 10 ** 6)] * 3))
        c["len"] = _log(rng, {"decode": 1, "page_select": 4 * c["page"]}.get(kind, 64), 131072)
        pages = -(-c["len"] // c["page"])
        if kind in ("page_map", "kv_append"):
            c["new"] = rng.choice([1, 1, min(c["len"], _log(rng, 2, 8192))])
            c["len"] = min(c["len"], 20000 if kind == "page_map" else 8192)
            c["new"] = min(c["new"], c["len"])
            c.update({"fused": rng.random() < 0.5} if kind == "kv_append" else {})
        elif kind == "page_select":
            c.update(budget=min(pages, _log(rng, 4, 512)), ties=rng.random() < 0.5)
        elif kind == "decode":
            c.update(listed=min(pages, _log(rng, 1, 256)) if rng.random() < 0.4 else 0, lse=rng.random() < 0.5)
        if work(c)["bytes"] <= 0.9 * most and _state_bytes(c) <= 6e9:
            return c


# ---- sizes

def _lens(c):
    """Tokens of every sequence, the new ones among them."""
    if not c["mix"]:
        return [c["len"]] * c["batch"]
    rng = random.Random(c["mix"])
    low = max(1, c["len"] // 32)
    return [c["len"]] + [_log(rng, low, c["len"]) for _ in range(c["batch"] - 1)]


def _new(c):
    """Of these, the tokens that the call adds."""
    if c["new"] == 1 or not c["mix"]:
        return [min(c["new"], n) for n in _lens(c)]
    rng = random.Random(c["mix"] + 1)
    return [min(n, c["new"] if i == 0 else rng.randrange(0, c["new"] + 1)) for i, n in enumerate(_lens(c))]


def _pages(c):
    return [-(-n // c["page"]) for n in _lens(c)]


def _touched(c):
    """(sequence, page) pairs that new tokens fall into, and those of them that held tokens before."""
    all_, old = 0, 0
    for n, w in zip(_lens(c), _new(c)):
        if w:
            first = (n - w) // c["page"]
            all_ += -(-n // c["page"]) - first
            old += (n - w) % c["page"] != 0
    return all_, old


def _list_tokens(c):
    """Tokens of every sequence's list: the last page is always listed and may be partly filled."""
    out = []
    for n, p in zip(_lens(c), _pages(c)):
        k = min(c["listed"], p)
        out.append(k * c["page"] - (p * c["page"] - n) if k else 0)
    return out


def _state_bytes(c):
    if c["kind"] in ("decode", "kv_append"):
        return sum(_pages(c)) * c["page"] * c["hkv"] * D * 4 * 1.3
    return sum(_pages(c)) * c["hkv"] * D * 4


def work(c):
    pages, row = sum(_pages(c)), c["hkv"] * D * 2
    if c["kind"] == "page_map":
        t, taken = sum(_new(c)), _touched(c)[0] - _touched(c)[1]
        return {"bytes": 8 * t + 8 * taken + 16 * c["batch"] + 4 * _touched(c)[1], "flops": 4 * t + 4 * c["batch"]}
    if c["kind"] == "kv_append":
        t, (all_, old) = sum(_new(c)), _touched(c)
        return {"bytes": 4 * t * row + 8 * t + (all_ + old) * 2 * row, "flops": 2 * t * c["hkv"] * D}
    if c["kind"] == "page_score":
        return {"bytes": pages * (2 * row + 4 + 4 * c["hq"]) + c["batch"] * c["hq"] * D * 2,
                "flops": 4 * D * c["hq"] * pages}
    if c["kind"] == "page_select":
        return {"bytes": 4 * c["hq"] * pages + 4 * c["batch"] * c["hkv"] * (c["budget"] + 1),
                "flops": 3 * c["hq"] * pages}
    t = sum(_list_tokens(c)) if c["listed"] else sum(_lens(c))
    return {"bytes": 2 * t * row + 4 * c["batch"] * c["hq"] * D + 4 * t // c["page"], "flops": 4 * D * c["hq"] * t}


# ---- inputs, made on the GPU from the seed alone

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _table(c, gen, spare):
    """int32 [batch, widest] page table of a cache with `spare` unused pages, and the unused ones; entries
    behind a sequence's last page are -1."""
    pages = _pages(c)
    n_pages = sum(pages) + spare
    perm = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((c["batch"], max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for n, p in enumerate(pages):
        table[n, :p] = perm[at:at + p]
        at += p
    return table, perm[at:].contiguous(), n_pages


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cache(c, gen, table, n_pages):
    """Keys with a direction per KV head that some of them share, attention sinks at the start of every sequence."""
    k = torch.empty(n_pages, c["hkv"], c["page"], D, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    u = torch.randn(c["hkv"], 1, D, generator=gen, device="cuda")
    u = 3.0 * u / u.norm(dim=2, keepdim=True)
    step = max(1, 2 ** 27 // (c["hkv"] * c["page"] * D))
    for a in range(0, n_pages, step):
        shape = k[a:a + step].shape
        x = torch.randn(shape, generator=gen, device="cuda")
        x += (torch.rand(shape[:3] + (1,), generator=gen, device="cuda") < 0.01) * u
        k[a:a + step] = x
        v[a:a + step] = torch.randn(shape, generator=gen, device="cuda")
    first = table[:, 0].long()
    k[first, :, :4] *= 4.0
    return k, v, u


def _queries(c, gen, u):
    g = c["hq"] // c["hkv"]
    q = torch.randn(c["batch"], c["hkv"], g, D, generator=gen, device="cuda")
    q += (torch.rand(c["batch"], c["hkv"], g, 1, generator=gen, device="cuda") < 0.3) * u
    return q.reshape(c["batch"], c["hq"], D).to(torch.bfloat16)


def _inputs(c, seed):
    gen = _gen(seed)
    st = {"case": c, "lens": _lens(c)}
    if c["kind"] == "page_map":
        cached = [n - w for n, w in zip(_lens(c), _new(c))]
        table, spare, n_pages = _table(c, gen, 7)
        # the pages that the call takes are not in the table yet
        held = torch.arange(table.shape[1], device="cuda")[None] < _i32([-(-x // c["page"]) for x in cached])[:, None]
        taken = table[~held & (table >= 0)]
        st.update(table=torch.where(held, table, -1), free=torch.cat([taken, spare]), cached=_i32(cached),
                  new=_i32(_new(c)), n_new=sum(_new(c)) + 5)
        st["n_free"] = _i32([st["free"].numel()])
    elif c["kind"] == "kv_append":
        table, _, n_pages = _table(c, gen, 3)
        k, v, _ = _cache(c, gen, table, n_pages)
        t = sum(_new(c))
        heads = c["hq"] + 2 * c["hkv"] if c["fused"] else 2 * c["hkv"]
        qkv = torch.randn(t, heads, D, generator=gen, device="cuda").to(torch.bfloat16)
        slots, host = torch.empty(t, dtype=torch.int64, device="cuda"), 0
        for n, (size, w) in enumerate(zip(_lens(c), _new(c))):
            pos = torch.arange(size - w, size, device="cuda")
            slots[host:host + w] = table[n].long()[pos // c["page"]] * c["page"] + pos % c["page"]
            host += w
        # the bounds of the tokens that are there already: all in front of a page's first new one
        first = torch.full((n_pages,), c["page"], dtype=torch.int64, device="cuda")
        for n, (size, w) in enumerate(zip(_lens(c), _new(c))):
            if w:
                first[table[n].long()[(size - w) // c["page"]]] = (size - w) % c["page"]
        bounds = torch.zeros(n_pages, c["hkv"], 2, D, dtype=torch.bfloat16, device="cuda")
        step = max(1, 2 ** 27 // (c["hkv"] * c["page"] * D))
        for a in range(0, n_pages, step):
            there = (torch.arange(c["page"], device="cuda")[None] < first[a:a + step, None])[:, None, :, None]
            x = k[a:a + step]
            bounds[a:a + step, :, 0] = torch.where(there, x, torch.inf).amin(2)
            bounds[a:a + step, :, 1] = torch.where(there, x, -torch.inf).amax(2)
        st.update(k_cache=k, v_cache=v, bounds=bounds, slots=slots, n_pages=n_pages, tokens=t)
        if c["fused"]:
            st.update(k=qkv[:, c["hq"]:c["hq"] + c["hkv"]], v=qkv[:, c["hq"] + c["hkv"]:])
        else:
            st.update(k=qkv[:, :c["hkv"]].contiguous(), v=qkv[:, c["hkv"]:].contiguous())
    elif c["kind"] == "page_score":
        table, _, n_pages = _table(c, gen, 3)
        # extremes of a page's keys: about sqrt(2 ln page) deviations on either side, and a page's own offset
        wide = math.sqrt(2.0 * math.log(c["page"]))
        bounds = torch.empty(n_pages, c["hkv"], 2, D, dtype=torch.bfloat16, device="cuda")
        for a in range(0, n_pages, 8192):
            shape = bounds[a:a + 8192, :, 0].shape
            shift = 0.3 * torch.randn(shape, generator=gen, device="cuda")
            for i, sign in ((0, -1.0), (1, 1.0)):
                ext = (wide + 0.4 * torch.randn(shape, generator=gen, device="cuda")).clamp_min(0.1)
                bounds[a:a + 8192, :, i] = sign * ext + shift
        st.update(table=table, n_pages=n_pages, bounds=bounds, q=_queries(c, gen, torch.zeros(c["hkv"], 1, D, device="cuda")))
    elif c["kind"] == "page_select":
        wide = max(_pages(c))
        score = 12.0 + 1.5 * torch.randn(c["batch"], c["hq"], wide, generator=gen, device="cuda")
        score += torch.randn(c["batch"], c["hq"], 1, generator=gen, device="cuda")
        st["score"] = (8 * score).round() / 8 if c["ties"] else score
        st["wide"] = wide
    else:
        table, _, n_pages = _table(c, gen, 3)
        k, v, u = _cache(c, gen, table, n_pages)
        st.update(table=table, n_pages=n_pages, k_cache=k, v_cache=v, q=_queries(c, gen, u))
        if c["listed"]:
            # every KV head's list: random pages in ascending order, the last page among them
            wide = min(c["listed"], table.shape[1])
            rank = torch.rand(c["batch"], c["hkv"], table.shape[1], generator=gen, device="cuda")
            at = torch.arange(table.shape[1], device="cuda")
            have = _i32(_pages(c))[:, None, None]
            rank = torch.where(at < have, rank, 2.0)
            rank = torch.where(at == have - 1, -1.0, rank)
            kept = have.clamp_max(wide)
            chosen = rank.argsort(2).argsort(2) < kept
            order = torch.where(chosen, at, table.shape[1]).sort(2).values[..., :wide]
            st["pages"] = torch.where(order < table.shape[1], order, -1).to(torch.int32).contiguous()
            st["count"] = kept[..., 0].expand(-1, c["hkv"]).to(torch.int32).contiguous()
    return st


def prepare(case, seed):
    c, st = case, _inputs(case, seed)
    dev = {"device": "cuda"}
    if c["kind"] == "page_map":
        st.update(seq_lens=torch.zeros(c["batch"], dtype=torch.int32, **dev),
                  cu_new=torch.zeros(c["batch"] + 1, dtype=torch.int32, **dev),
                  slots=torch.zeros(st["n_new"], dtype=torch.int64, **dev), n_taken=torch.zeros(1, dtype=torch.int32, **dev))
    else:
        st["seq_lens"] = _i32(_lens(c))
    if c["kind"] == "page_score":
        st["score"] = torch.zeros(c["batch"], c["hq"], st["table"].shape[1], **dev)
    elif c["kind"] == "page_select":
        st.update(pages=torch.zeros(c["batch"], c["hkv"], c["budget"], dtype=torch.int32, **dev),
                  count=torch.zeros(c["batch"], c["hkv"], dtype=torch.int32, **dev))
    elif c["kind"] == "decode":
        st["o"] = torch.zeros_like(st["q"])
        st["lse"] = torch.zeros(c["batch"], c["hq"], **dev) if c["lse"] else None
    if not own:
        return st
    from paper_2607_25291_amd import binding as B
    if c["kind"] in ("page_score", "page_select", "decode"):
        wide = st["wide"] if c["kind"] == "page_select" else st["table"].shape[1]
        st["p"] = B.DecodeProblem(c["batch"], c["hq"], c["hkv"], wide)
    if c["kind"] == "page_select":
        st["budget"] = B.page_budget(max_pages=c["budget"], min_pages=c["budget"], sink_pages=1, recent_pages=2)
    elif c["kind"] == "page_score":
        st["kv"] = B.paged_kv(None, None, st["table"], c["page"], st["n_pages"])
    elif c["kind"] == "decode":
        st["kv"] = B.paged_kv(st["k_cache"], st["v_cache"], st["table"], c["page"], st["n_pages"])
        st["ws_bytes"] = B.cosa_decode_workspace_bytes(st["p"])
        st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, **dev)
    return st


# ---- one pass

def _run_own(st):
    from paper_2607_25291_amd import binding as B
    c = st["case"]
    if c["kind"] == "page_map":
        B.cosa_page_map(c["batch"], c["page"], st["table"].shape[1], st["cached"], st["new"], st["free"],
                        st["free"].numel(), st["n_free"], st["table"], st["seq_lens"], st["cu_new"], st["slots"],
                        st["n_new"], st["n_taken"])
    elif c["kind"] == "kv_append":
        B.cosa_kv_append(c["hkv"], D, c["page"], st["n_pages"], st["k_cache"], st["v_cache"], st["bounds"],
                         st["tokens"], st["k"], st["v"], st["slots"])
    elif c["kind"] == "page_score":
        B.cosa_page_score(st["p"], st["q"], st["kv"], st["bounds"], st["seq_lens"], st["score"])
    elif c["kind"] == "page_select":
        B.cosa_page_select(st["p"], c["page"], st["seq_lens"], st["score"], st["budget"], st["pages"], st["count"])
    elif c["listed"]:
        B.cosa_decode_attention_listed(st["p"], st["q"], st["kv"], st["seq_lens"], st["pages"], st["count"],
                                       st["pages"].shape[2], st["ws"], st["ws_bytes"], st["o"], st["lse"])
    else:
        B.cosa_decode_attention(st["p"], st["q"], st["kv"], st["seq_lens"], st["ws"], st["ws_bytes"], st["o"], st["lse"])


def _plain_map(st):
    c, page = st["case"], st["case"]["page"]
    cached, new = st["cached"].long(), st["new"].long()
    wide = st["table"].shape[1]
    have = (cached + page - 1) // page
    need = (cached + new + page - 1) // page - have
    base = torch.cumsum(need, 0) - need
    at = torch.arange(wide, device="cuda")[None]
    fresh = (at >= have[:, None]) & (at < (have + need)[:, None])
    pick = (base[:, None] + at - have[:, None]).clamp(0, st["free"].numel() - 1)
    st["table"].copy_(torch.where(fresh, st["free"][pick], st["table"]))
    end = torch.cumsum(new, 0)
    t = torch.arange(st["n_new"], device="cuda")
    r = (t[:, None] >= end[None]).sum(1)
    real = r < c["batch"]
    r = r.clamp_max(c["batch"] - 1)
    pos = cached[r] + t - (end - new)[r]
    entry = st["table"][r, torch.where(real, pos // page, 0)].long()
    st["slots"].copy_(torch.where(real, entry * page + pos % page, -1))
    st["seq_lens"].copy_(cached + new)
    st["cu_new"][0] = 0
    st["cu_new"][1:] = end
    st["n_taken"][0] = need.sum()


def _plain_append(st):
    page = st["case"]["page"]
    p, off = st["slots"] // page, st["slots"] % page
    st["k_cache"][p, :, off] = st["k"]
    st["v_cache"][p, :, off] = st["v"]
    last = torch.full((st["n_pages"],), -1, dtype=torch.int64, device="cuda").scatter_reduce(0, p, off, "amax")
    step = max(1, 2 ** 27 // (st["k_cache"].shape[1] * page * D))
    for a in range(0, st["n_pages"], step):
        e = last[a:a + step]
        there = (torch.arange(page, device="cuda")[None] <= e[:, None])[:, None, :, None]
        x, old, hit = st["k_cache"][a:a + step], st["bounds"][a:a + step], (e >= 0)[:, None, None]
        lo = torch.where(there, x, torch.inf).amin(2)
        hi = torch.where(there, x, -torch.inf).amax(2)
        old.copy_(torch.stack([torch.where(hit, lo, old[:, :, 0]), torch.where(hit, hi, old[:, :, 1])], 2))


def _plain_score(st):
    c, g = st["case"], st["case"]["hq"] // st["case"]["hkv"]
    for n, p in enumerate(_pages(c)):
        b = st["bounds"][st["table"][n, :p].long()].float()
        q = st["q"][n].float().view(c["hkv"], g, D)
        up = torch.matmul(q.clamp_min(0), b[:, :, 1].permute(1, 2, 0)) + torch.matmul(q.clamp_max(0), b[:, :, 0].permute(1, 2, 0))
        st["score"][n, :, :p] = (up / math.sqrt(D)).reshape(c["hq"], p)


def _plain_select(st):
    c, wide = st["case"], st["wide"]
    at = torch.arange(wide, device="cuda")
    have = -(-st["seq_lens"].long() // c["page"])[:, None, None]
    s = torch.where(at < have, st["score"], -torch.inf)
    s = (s - s.amax(2, keepdim=True)).view(c["batch"], c["hkv"], -1, wide).amax(2)
    s = torch.where((at < 1) | (at >= have - 2), torch.inf, s)
    s = torch.where(at < have, s, -torch.inf)
    kept = have.clamp_max(c["budget"])
    by = torch.sort(s, dim=2, descending=True, stable=True).indices[..., :c["budget"]]
    by = torch.where(at[:c["budget"]] < kept, by, wide).sort(2).values
    st["pages"].copy_(torch.where(by < wide, by, -1))
    st["count"].copy_(kept[..., 0].expand(-1, c["hkv"]))


def _rows(st, n, length):
    """Keys and values [hkv, tokens, D] of sequence n that its heads attend to."""
    c = st["case"]
    if not c["listed"]:
        at = st["table"][n, :-(-length // c["page"])].long()
        k, v = (x[at].transpose(0, 1).reshape(c["hkv"], -1, D)[:, :length] for x in (st["k_cache"], st["v_cache"]))
        return k, v
    keep = min(c["listed"], -(-length // c["page"]))
    tokens = keep * c["page"] - (-length % c["page"])
    lists = st["table"][n].long()[st["pages"][n, :, :keep].long()]
    head = torch.arange(c["hkv"], device="cuda")[:, None]
    return tuple(x[lists, head].reshape(c["hkv"], -1, D)[:, :tokens] for x in (st["k_cache"], st["v_cache"]))


def _plain_decode(st):
    c, g = st["case"], st["case"]["hq"] // st["case"]["hkv"]
    for n, length in enumerate(st["lens"]):
        k, v = _rows(st, n, length)
        q = st["q"][n].float().view(c["hkv"], g, D)
        s = torch.matmul(q, k.float().transpose(1, 2).contiguous()) / math.sqrt(D)
        m = s.amax(2, keepdim=True)
        p = torch.exp(s - m)
        total = p.sum(2, keepdim=True)
        st["o"][n] = (torch.matmul(p, v.float()) / total).reshape(c["hq"], D)
        if c["lse"]:
            st["lse"][n] = (m + torch.log(total)).reshape(-1)


def run(st):
    kind = st["case"]["kind"]
    if own:
        _run_own(st)
    else:
        {"page_map": _plain_map, "kv_append": _plain_append, "page_score": _plain_score,
         "page_select": _plain_select, "decode": _plain_decode}[kind](st)
    names = {"page_map": ["table", "seq_lens", "cu_new", "slots", "n_taken"], "kv_append": ["k_cache", "v_cache", "bounds"],
             "page_score": ["score"], "page_select": ["pages", "count"],
             "decode": ["o", "lse"] if st["case"].get("lse") else ["o"]}[kind]
    return {x: st[x] for x in names}


# ---- the 64-bit results

def exact(case, seed):
    c = case
    if c["kind"] in ("page_map", "page_select"):  # whole numbers
        return None
    if c["kind"] == "kv_append" and _touched(c)[0] > 20000:
        return None
    st = _inputs(case, seed)
    f64 = {"dtype": torch.float64, "device": "cuda"}
    if c["kind"] == "kv_append":
        # a page's bounds: over its old tokens, which the old bounds stand for, and the rows that fall into it
        out = st["bounds"].double()
        off, at = 0, st["slots"] // c["page"]
        for w in _new(c):
            for p in torch.unique(at[off:off + w]).tolist():
                rows = torch.nonzero(at[off:off + w] == p).flatten() + off
                fresh = int((st["slots"][rows] % c["page"]).min()) == 0
                x = st["k"][rows].double()
                lo, hi = x.min(0).values, x.max(0).values
                out[p, :, 0] = lo if fresh else torch.minimum(out[p, :, 0], lo)
                out[p, :, 1] = hi if fresh else torch.maximum(out[p, :, 1], hi)
            off += w
        return {"k_cache": None, "v_cache": None, "bounds": out}
    g = c["hq"] // c["hkv"]
    if c["kind"] == "page_score":
        out = torch.zeros(c["batch"], c["hq"], st["table"].shape[1], **f64)
        for n, p in enumerate(_pages(c)):
            at = st["table"][n, :p].long()
            for h in range(c["hq"]):
                b, q = st["bounds"][at, h // g].double(), st["q"][n, h].double()
                out[n, h, :p] = torch.maximum(q * b[:, 0], q * b[:, 1]).sum(1) * D ** -0.5
        return {"score": out}
    o, lse = torch.zeros(c["batch"], c["hq"], D, **f64), torch.zeros(c["batch"], c["hq"], **f64)
    for n, length in enumerate(_lens(c)):
        pos = torch.arange(length, device="cuda")
        for h in range(c["hkv"]):
            if c["listed"]:
                mark = torch.zeros(-(-length // c["page"]), dtype=torch.bool, device="cuda")
                mark[st["pages"][n, h, :int(st["count"][n, h])].long()] = True
                pos = torch.nonzero(mark[torch.arange(length, device="cuda") // c["page"]]).flatten()
            p, r = st["table"][n].long()[pos // c["page"]], pos % c["page"]
            k, v = st["k_cache"][p, h, r].double(), st["v_cache"][p, h, r].double()
            s = st["q"][n, h * g:(h + 1) * g].double() @ k.T * D ** -0.5
            o[n, h * g:(h + 1) * g] = torch.softmax(s, 1) @ v
            lse[n, h * g:(h + 1) * g] = torch.logsumexp(s, 1)
    return {"o": o, "lse": lse} if c["lse"] else {"o": o}
