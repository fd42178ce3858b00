"""The operators of serving over a paged KV cache beside a decode step: attention of chunks of new tokens, and
the cache's pages (forked, copied, released, compacted). Each as a user's program calls it: sizes, inputs, a plain
form in elementary torch operations and, for the attention, a 64-bit result.

Every case is one call (kind):
  chunk    attention of every sequence's new tokens over its pages, causal from the sequence's end
  fork     block tables of children that share their parents' pages
  copy     pages (or their first rows) of K, V and the key bounds to other pages
  release  pages that no row holds any more go back to the free list
  compact  pages move to the lowest numbers: the moves, the new block tables and the free list
Fields: batch (sequences or rows), hq, hkv, page (tokens of a page), len (longest sequence in tokens), mix (0:
every sequence has that length; otherwise lengths differ, and this number picks them), and per kind: new (most new
tokens of a sequence), ones (share of the sequences that add one token), lse, fused (queries are slices of
one projection), children (rows of the new table), pairs, whole (whole pages), gone (share of the rows
that end), fill (share of the cache in use), moves (limit of a compaction, 0: none).
"""
import math
import random

import torch

own = False

D = 128
_BASE = {"batch": 1, "hq": 32, "hkv": 8, "page": 64, "len": 4096, "mix": 0}
_EXTRA = {"chunk": {"new": 512, "ones": 0.0, "lse": False, "fused": False}, "fork": {"children": 8, "all": False},
          "copy": {"pairs": 64, "whole": True, "bounds": True}, "release": {"gone": 0.2},
          "compact": {"fill": 0.5, "moves": 0}}


def _case(kind, name=None, **kw):
    c = {"kind": kind, **_BASE, **_EXTRA[kind], **kw}
    return {"name": name, **c} if name else c


def listed():
    return [
        # The smallest: 16 drafted tokens of one short sequence are verified, one group of heads; latency counts.
        _case("chunk", "chunk_verify_16", hq=4, hkv=1, page=16, len=1000, new=16, lse=True),
        # A mixed serving step: one request brings a chunk of its prompt, the others a token each.
        _case("chunk", "chunk_mixed_48", batch=48, len=16384, mix=1, new=1024, ones=0.9, fused=True),
        # Prompts of uneven lengths without a cached part, small pages, an odd group of query heads.
        _case("chunk", "chunk_prompts_19", batch=19, hq=28, hkv=4, page=16, len=4097, mix=2, new=4097),
        # A chunk of a long prompt behind what is cached of it: the most arithmetic.
        _case("chunk", "chunk_4k_over_64k", len=65536, new=4096, lse=True),
        # One prompt of 8K tokens is sampled 8 times.
        _case("fork", "fork_8_samples", len=8001, children=8),
        # A beam search over a large batch goes on from the rows that it keeps.
        _case("fork", "fork_beams_512", batch=512, len=65536, mix=3, page=16, children=512),
        # The partly filled pages of a fork's children, one layer.
        _case("copy", "copy_fork_64", pairs=64, whole=False),
        # The pages that a compaction moves, one layer.
        _case("copy", "copy_pages_2k", pairs=2048, page=128),
        # A few requests of a step end.
        _case("release", "release_step_64", batch=64, len=20000, mix=4, gone=0.05),
        # Many rows of long contexts with small pages, half of them end.
        _case("release", "release_512", batch=512, len=65536, mix=5, page=16, gone=0.5),
        # A small cache is compacted.
        _case("compact", "compact_64", batch=64, len=20000, mix=6),
        # A large one, a third in use.
        _case("compact", "compact_512", batch=512, len=65536, mix=7, page=16, fill=0.34),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng: random.Random):
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = [max(a, b) for a, b in zip(most.get(c["kind"], [0, 0]), [w["bytes"], w["flops"]])]
    while True:
        kind = rng.choice(["chunk", "chunk", "chunk", "chunk", "fork", "copy", "release", "compact"])
        hkv = rng.choice([1, 2, 4, 5, 8])
        c = _case(kind, batch=_log(rng, 1, 128 if kind == "chunk" else 512), hkv=hkv,
                  hq=hkv * rng.choice([1, 2, 3, 4, 4, 6, 7, 8, 12, 16, 20]), page=rng.choice([16, 32, 64, 128, 256]),
                  mix=rng.choice([0] + [rng.randrange(1, 10 ** 6)] * 3), len=_log(rng, 1, 65536))
        if kind == "chunk":
            c.update(new=min(c["len"], _log(rng, 1, 8192)), ones=rng.choice([0.0, 0.0, 0.5, 0.9]), lse=rng.random() < 0.5,
                     fused=rng.random() < 0.3)
        elif kind == "fork":
            c.update(children=_log(rng, 1, 512), all=rng.random() < 0.3)
        elif kind == "copy":
            c.update(pairs=_log(rng, 1, 4096), whole=rng.random() < 0.5, bounds=rng.random() < 0.7)
        elif kind == "release":
            c.update(gone=rng.choice([0.02, 0.2, 0.5, 1.0]))
        else:
            c.update(fill=rng.uniform(0.05, 1.0), moves=rng.choice([0, 0, _log(rng, 1, 4096)]))
        w = work(c)
        # a pass in the plain form over many short sequences is bound by its launches
        if w["bytes"] <= max(most[kind][0], most["copy"][0] if kind == "chunk" else 0) and w["flops"] <= most[kind][1]:
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
    """Of these, the tokens whose queries a chunk call has."""
    rng = random.Random(c["mix"] + 1)
    out = []
    for i, n in enumerate(_lens(c)):
        one = rng.random() < c["ones"] and i > 0
        w = c["new"] if i == 0 or not c["mix"] else rng.randrange(0, c["new"] + 1)
        out.append(min(n, 1 if one else n if c["new"] >= c["len"] else w))
    return out


def _pages(c):
    return [-(-n // c["page"]) for n in _lens(c)]


def _shared(c):
    """Leading pages that row n shares with the row in front of it (rows that were forked some time ago)."""
    rng, pages = random.Random(c["mix"] + 2), _pages(c)
    out = [0]
    for n in range(1, c["batch"]):
        most = min(min(_lens(c)[n], _lens(c)[n - 1]) // c["page"], pages[n])
        out.append(rng.randrange(0, most + 1) if rng.random() < 0.3 else 0)
    return out


def _used(c):
    return sum(_pages(c)) - sum(_shared(c))


def _n_pages(c):
    if c["kind"] == "copy":
        return 2 * c["pairs"] + 3
    if c["kind"] == "compact":
        return max(_used(c), int(_used(c) / c["fill"]))
    return _used(c) + (c["children"] if c["kind"] == "fork" else 0) + max(7, _used(c) // 8)


def _ends(c):
    rng = random.Random(c["mix"] + 3)
    return [rng.random() < c["gone"] for _ in range(c["batch"])]


def _parents(c):
    """Rows that the children continue; some rows have none, some many, and some children start empty."""
    rng = random.Random(c["mix"] + 4)
    return [rng.randrange(0, c["batch"]) if rng.random() < 0.97 else -1 for _ in range(c["children"])]


def _copy_rows(c):
    rng = random.Random(c["mix"] + 5)
    return [c["page"] if c["whole"] else rng.randrange(1, c["page"]) for _ in range(c["pairs"])]


def work(c):
    row = c["hkv"] * D * 2
    if c["kind"] == "chunk":
        seen = sum((n - w) * w + w * (w + 1) // 2 for n, w in zip(_lens(c), _new(c)))
        t = sum(_new(c))
        read = sum(n for n, w in zip(_lens(c), _new(c)) if w)
        return {"bytes": 2 * read * row + 4 * t * c["hq"] * D + 4 * read // c["page"] + (4 * t * c["hq"] if c["lse"] else 0),
                "flops": 4 * D * c["hq"] * seen}
    if c["kind"] == "copy":
        return {"bytes": 4 * sum(_copy_rows(c)) * row + (4 * c["pairs"] * row if c["bounds"] else 0) + 12 * c["pairs"],
                "flops": c["pairs"]}
    if c["kind"] == "fork":
        pages, kids = _pages(c), [p for p in _parents(c) if p >= 0]
        read, written = sum(pages[p] for p in set(kids)), sum(pages[p] for p in kids)
        return {"bytes": 4 * (read + written) + 12 * c["children"], "flops": written}
    if c["kind"] == "release":
        held, left = sum(_pages(c)), sum(p for p, e in zip(_pages(c), _ends(c)) if not e)
        return {"bytes": 4 * (held + left) + 8 * (_n_pages(c) - _used(c)) + 4 * (held - left) + 8 * c["batch"],
                "flops": held + left}
    entries, n = c["batch"] * max(_pages(c)), _n_pages(c)
    moved = min(n - _used(c), _used(c))
    return {"bytes": 8 * entries + 4 * (n - _used(c)) + 8 * min(moved, c["moves"] or moved) + 4 * c["batch"],
            "flops": entries + n}


# ---- inputs, made on the GPU from the seed alone

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _table(c, gen, shared):
    """int32 [batch, widest] page table, -1 behind a sequence's last page, and the unused pages, in random order."""
    pages = _pages(c)
    n_pages = _n_pages(c) if c["kind"] != "chunk" else sum(pages) + 3
    perm = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((c["batch"], max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for n, p in enumerate(pages):
        k = shared[n] if shared else 0
        if k:
            table[n, :k] = table[n - 1, :k]
        table[n, k:p] = perm[at:at + p - k]
        at += p - k
    return table, perm[at:].contiguous(), n_pages


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
    if table is not None:
        k[table[:, 0].long(), :, :4] *= 4.0
    return k, v, u


def _inputs(c, seed):
    gen = _gen(seed)
    st = {"case": c}
    if c["kind"] == "chunk":
        table, _, n_pages = _table(c, gen, None)
        k, v, u = _cache(c, gen, table, n_pages)
        t, g = sum(_new(c)), c["hq"] // c["hkv"]
        q = torch.randn(t, c["hkv"], g, D, generator=gen, device="cuda")
        q += (torch.rand(t, c["hkv"], g, 1, generator=gen, device="cuda") < 0.3) * u
        q = q.reshape(t, c["hq"], D).to(torch.bfloat16)
        if c["fused"]:
            wide = torch.randn(t, c["hq"] + 2 * c["hkv"], D, generator=gen, device="cuda").to(torch.bfloat16)
            wide[:, :c["hq"]] = q
            q = wide[:, :c["hq"]]
        cu = [0]
        for w in _new(c):
            cu.append(cu[-1] + w)
        st.update(table=table, n_pages=n_pages, k_cache=k, v_cache=v, q=q, seq_lens=_i32(_lens(c)), cu_new=_i32(cu),
                  lens=_lens(c), new=_new(c), rows=t)
        return st
    if c["kind"] == "copy":
        n_pages = _n_pages(c)
        k, v, _ = _cache(c, gen, None, n_pages)
        bounds = torch.randn(n_pages, c["hkv"], 2, D, generator=gen, device="cuda").to(torch.bfloat16)
        perm = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        st.update(n_pages=n_pages, k_cache=k, v_cache=v, bounds=bounds if c["bounds"] else None,
                  src=perm[:c["pairs"]].contiguous(), dst=perm[c["pairs"]:2 * c["pairs"]].contiguous(),
                  n_pairs=_i32([c["pairs"]]), rows=None if c["whole"] else _i32(_copy_rows(c)))
        return st
    table, free, n_pages = _table(c, gen, _shared(c))
    st.update(table=table, free=free, n_free=_i32([free.numel()]), n_pages=n_pages, seq_lens=_i32(_lens(c)))
    if c["kind"] == "fork":
        st["parent"] = _i32(_parents(c))
    elif c["kind"] == "release":
        st.update(new_lens=_i32([0 if e else n for n, e in zip(_lens(c), _ends(c))]),
                  n_taken=_i32([min(c["batch"] // 8, free.numel())]))
    return st


def prepare(case, seed):
    c, st = case, _inputs(case, seed)
    zeros = lambda *s, dt=torch.int32: torch.zeros(*s, dtype=dt, device="cuda")
    if c["kind"] == "chunk":
        st["o"] = zeros(st["rows"], c["hq"], D, dt=torch.bfloat16)
        st["lse"] = zeros(st["rows"], c["hq"], dt=torch.float32) if c["lse"] else None
    elif c["kind"] == "fork":
        n = c["children"]
        st.update(new_table=torch.full((n, st["table"].shape[1]), -1, dtype=torch.int32, device="cuda"), new_lens=zeros(n),
                  src=zeros(n), dst=zeros(n), rows=zeros(n), n_taken=zeros(1))
    elif c["kind"] == "release":
        st.update(free_out=zeros(st["n_pages"]), n_free_out=zeros(1))
    elif c["kind"] == "compact":
        st["max_moves"] = c["moves"] or st["n_pages"]
        st.update(new_table=torch.zeros_like(st["table"]), src=zeros(st["max_moves"]), dst=zeros(st["max_moves"]),
                  n_moves=zeros(1), free_out=zeros(st["n_pages"]), n_free_out=zeros(1))
    if not own:
        return st
    from paper_2607_25291_amd import binding as B
    if c["kind"] == "chunk":
        st["p"] = B.ChunkProblem(c["batch"], c["hq"], c["hkv"], st["table"].shape[1], st["rows"])
        st["kv"] = B.paged_kv(st["k_cache"], st["v_cache"], st["table"], c["page"], st["n_pages"])
        st["ws_bytes"] = B.cosa_chunk_workspace_bytes(st["p"])
    elif c["kind"] in ("release", "compact"):
        st["ws_bytes"] = B.cosa_page_workspace_bytes(st["n_pages"])
    if "ws_bytes" in st:
        st["ws"] = torch.empty(st["ws_bytes"], dtype=torch.uint8, device="cuda")
    return st


# ---- one pass

def _run_own(st):
    from paper_2607_25291_amd import binding as B
    c = st["case"]
    if c["kind"] == "chunk":
        B.cosa_chunk_attention(st["p"], st["q"], st["kv"], st["seq_lens"], st["cu_new"], st["ws"], st["ws_bytes"], st["o"],
                               st["lse"])
    elif c["kind"] == "fork":
        B.cosa_page_fork(c["batch"], c["children"], c["page"], st["table"].shape[1], st["parent"], st["table"], st["seq_lens"],
                         int(c["all"]), st["free"], st["free"].numel(), st["n_free"], st["new_table"], st["new_lens"],
                         st["src"], st["dst"], st["rows"], st["n_taken"])
    elif c["kind"] == "copy":
        B.cosa_page_copy(c["hkv"], D, c["page"], st["n_pages"], st["k_cache"], st["v_cache"], st["bounds"], st["src"],
                         st["dst"], st["rows"], c["pairs"], st["n_pairs"])
    elif c["kind"] == "release":
        B.cosa_page_release(c["page"], st["table"].shape[1], st["n_pages"], c["batch"], st["table"], st["seq_lens"],
                            c["batch"], st["table"], st["new_lens"], st["free"], st["free"].numel(), st["n_free"],
                            st["n_taken"], st["free_out"], st["n_pages"], st["n_free_out"], st["ws"], st["ws_bytes"])
    else:
        B.cosa_page_compact(c["batch"], c["page"], st["table"].shape[1], st["n_pages"], st["table"], st["seq_lens"],
                            st["max_moves"], st["new_table"], st["src"], st["dst"], st["n_moves"], st["free_out"],
                            st["n_pages"], st["n_free_out"], st["ws"], st["ws_bytes"])


def _plain_chunk(st):
    c, g = st["case"], st["case"]["hq"] // st["case"]["hkv"]
    row = 0
    for n, (length, w) in enumerate(zip(st["lens"], st["new"])):
        if not w:
            continue
        at = st["table"][n, :-(-length // c["page"])].long()
        k, v = (x[at].transpose(0, 1).reshape(c["hkv"], -1, D)[:, :length].float() for x in (st["k_cache"], st["v_cache"]))
        kt = k.transpose(1, 2).contiguous()
        t = torch.arange(length, device="cuda")
        step = max(1, 2 ** 28 // (c["hq"] * length))
        for a in range(0, w, step):
            b = min(w, a + step)
            q = st["q"][row + a:row + b].float().view(b - a, c["hkv"], g, D).transpose(0, 1).reshape(c["hkv"], -1, D)
            s = (torch.matmul(q, kt) / math.sqrt(D)).view(c["hkv"], b - a, g, length)
            pos = torch.arange(length - w + a, length - w + b, device="cuda")
            s = torch.where((t[None] <= pos[:, None])[None, :, None], s, -torch.inf)
            m = s.amax(3, keepdim=True)
            p = torch.exp(s - m)
            total = p.sum(3, keepdim=True)
            o = torch.matmul(p.view(c["hkv"], -1, length), v).view(c["hkv"], b - a, g, D) / total
            st["o"][row + a:row + b] = o.transpose(0, 1).reshape(b - a, c["hq"], D)
            if c["lse"]:
                st["lse"][row + a:row + b] = (m + torch.log(total)).transpose(0, 1).reshape(b - a, c["hq"])
        row += w


def _held(st, lens):
    have = -(-lens.long() // st["case"]["page"])
    return torch.arange(st["table"].shape[1], device="cuda")[None] < have[:, None]


def _mark(st, held):
    used = torch.zeros(st["n_pages"] + 1, dtype=torch.bool, device="cuda")
    used[torch.where(held, st["table"].long(), st["n_pages"])] = True
    return used[:-1]


def _put(out, keep, at, values):
    """out[at] = values where keep holds."""
    wide = torch.cat([out, out[:1]])
    wide[torch.where(keep, at, out.numel())] = values.to(out.dtype)
    out.copy_(wide[:-1])


def _plain_fork(st):
    c, page, n = st["case"], st["case"]["page"], st["case"]["children"]
    real = st["parent"] >= 0
    parent = st["parent"].long().clamp_min(0)
    length = torch.where(real, st["seq_lens"].long()[parent], 0)
    at = torch.arange(n, device="cuda")
    first = torch.full((c["batch"],), n, device="cuda").scatter_reduce(0, parent, torch.where(real, at, n), "amin")
    need = (length % page != 0) & ((first[parent] != at) | c["all"])
    rank = torch.cumsum(need, 0) - 1
    got = need & (rank < st["n_free"])
    length = torch.where(need & ~got, 0, length)
    j = torch.arange(st["table"].shape[1], device="cuda")[None]
    rows = st["table"][parent]
    fresh = st["free"][rank.clamp(0, st["free"].numel() - 1)]
    last = (length // page)[:, None]
    src = rows.gather(1, last.clamp_max(rows.shape[1] - 1))[:, 0]
    rows = torch.where(got[:, None] & (j == last), fresh[:, None], rows)
    st["new_table"].copy_(torch.where(j < -(-length // page)[:, None], rows, st["new_table"]))
    st["new_lens"].copy_(length)
    for name, x in (("src", src), ("dst", fresh), ("rows", length % page)):
        _put(st[name], got, rank, x)
    st["n_taken"][0] = got.sum()


def _plain_copy(st):
    c = st["case"]
    src, dst = st["src"].long(), st["dst"].long()
    step = max(1, 2 ** 28 // (c["hkv"] * c["page"] * D))
    for a in range(0, c["pairs"], step):
        s, d = src[a:a + step], dst[a:a + step]
        for x in (st["k_cache"], st["v_cache"]):
            if c["whole"]:
                x[d] = x[s]
            else:
                keep = torch.arange(c["page"], device="cuda")[None] < st["rows"][a:a + step, None]
                x[d] = torch.where(keep[:, None, :, None], x[s], x[d])
    if c["bounds"]:
        st["bounds"][dst] = st["bounds"][src]


def _plain_release(st):
    i = torch.arange(st["n_pages"], device="cuda")
    k = torch.arange(st["free"].numel(), device="cuda")
    old, new = _mark(st, _held(st, st["seq_lens"])), _mark(st, _held(st, st["new_lens"]))
    taken, n_free = st["n_taken"], st["n_free"]
    left = (k >= taken) & (k < n_free)
    listed_ = torch.zeros(st["n_pages"] + 1, dtype=torch.bool, device="cuda")
    listed_[torch.where(left, st["free"].long(), st["n_pages"])] = True
    gone = old & ~new & ~listed_[:-1]
    _put(st["free_out"], left, k - taken, st["free"])
    _put(st["free_out"], gone, torch.cumsum(gone, 0) - 1 + n_free - taken, i)
    st["n_free_out"].copy_(n_free - taken + gone.sum())


def _plain_compact(st):
    i = torch.arange(st["n_pages"], device="cuda")
    held = _held(st, st["seq_lens"])
    used = _mark(st, held)
    count = torch.cumsum(used, 0)
    total = count[-1]
    hole = ~used & (i < total)
    from_top, from_low = total - count, i - count
    moves = hole.sum().clamp_max(st["max_moves"])
    goes, filled = used & (i >= total) & (from_top < moves), hole & (from_low < moves)
    _put(st["src"], goes, from_top, i)
    _put(st["dst"], filled, from_low, i)
    to = torch.where(goes, st["dst"][from_top.clamp(0, st["max_moves"] - 1)], i)
    table = st["table"]
    st["new_table"].copy_(torch.where(held, to[table.long().clamp_min(0)], table))
    st["n_moves"][0] = moves
    free = (~used & ~filled) | goes
    _put(st["free_out"], free, torch.cumsum(free, 0) - 1, i)
    st["n_free_out"][0] = free.sum()


def run(st):
    kind = st["case"]["kind"]
    if own:
        _run_own(st)
    else:
        {"chunk": _plain_chunk, "fork": _plain_fork, "copy": _plain_copy, "release": _plain_release,
         "compact": _plain_compact}[kind](st)
    names = {"chunk": ["o", "lse"] if st["case"].get("lse") else ["o"],
             "fork": ["new_table", "new_lens", "src", "dst", "rows", "n_taken"],
             "copy": ["k_cache", "v_cache", "bounds"] if st["case"].get("bounds") else ["k_cache", "v_cache"],
             "release": ["free_out", "n_free_out"],
             "compact": ["new_table", "src", "dst", "n_moves", "free_out", "n_free_out"]}[kind]
    return {x: st[x] for x in names}


# ---- the 64-bit results

def exact(case, seed):
    c = case
    if c["kind"] != "chunk":  # whole numbers and copies
        return None
    if work(c)["flops"] > 6e12:
        return None
    st = _inputs(case, seed)
    f64 = {"dtype": torch.float64, "device": "cuda"}
    g, row = c["hq"] // c["hkv"], 0
    o, lse = torch.zeros(st["rows"], c["hq"], D, **f64), torch.zeros(st["rows"], c["hq"], **f64)
    for n, (length, w) in enumerate(zip(st["lens"], st["new"])):
        t = torch.arange(length, device="cuda")
        at, r = st["table"][n].long()[t // c["page"]], t % c["page"]
        step = max(1, 2 ** 26 // length)
        for h in range(c["hkv"] if w else 0):
            k, v = st["k_cache"][at, h, r].double(), st["v_cache"][at, h, r].double()
            for hh in range(h * g, (h + 1) * g):
                for a in range(0, w, step):
                    b = min(w, a + step)
                    s = st["q"][row + a:row + b, hh].double() @ k.T * D ** -0.5
                    last = length - w + torch.arange(a, b, device="cuda")
                    s.masked_fill_(t[None] > last[:, None], -torch.inf)
                    lse[row + a:row + b, hh] = torch.logsumexp(s, 1)
                    o[row + a:row + b, hh] = torch.softmax(s, 1) @ v
        row += w
    return {"o": o, "lse": lse} if c["lse"] else {"o": o}
