"""Performance cases of the key/value cache and the attention that reads it.

listed() names the cases, draw() gives further ones of the same ranges, prepare() makes what a program has in hand before a
call (a cache with its page table, queries, new keys and values), run() is one pass through an operator, exact() the same
outputs from the definition in 64 bits, work() the bytes and operations that one pass cannot do without.  With `own` false
run() computes the plain form, elementary torch operations in 32 bits rounded once at the end; with `own` true it makes the
calls of the library.

The cache: pool [layers][pages][K, V][kv_heads][page][D], 16 bits; table [rows][max_pages] page numbers, -1 where there is
none; lengths [rows] tokens held; refs [pages] how many rows hold a page.

Kinds of case
  attend   attention of the newest tokens of every sequence over the sequence's tokens in the cache, causal; the first
           `shared` tokens lie in the same pages for all sequences
  append   the keys and values of the newest tokens of every sequence written into the pages of one layer
  admit    the rows of finished sequences are freed, new prompts get pages, and their keys and values are written
  fork     the rows of dropped samples are freed and as many new samples forked from the parents: full pages shared, the last
           partial page copied in all layers
  compact  live pages moved to the low end of the pool in all layers, the table rewritten
"""
from __future__ import annotations

import math

import torch

own = False


# ------------------------------------------------------------------ the cases

def _attend(name, dtype, B, heads, kv_heads, D, page, shared, ctx, nq, ragged, fused):
    return {"name": name, "kind": "attend", "dtype": dtype, "B": B, "heads": heads, "kv_heads": kv_heads, "D": D, "page": page,
            "shared": shared, "ctx": ctx, "nq": nq, "ragged": ragged, "fused": fused}


def listed():
    return [
        # the smallest call: one sequence just begun, one token through the heads of a 4096-wide layer
        _attend("attend_b1_33", "f16", 1, 32, 32, 128, 16, 0, 33, 1, False, False),
        # sixteen sequences decoded together, ragged contexts around a thousand tokens, q a slice of a fused projection
        _attend("attend_b16_1000", "f16", 16, 32, 32, 128, 16, 0, 1000, 1, True, True),
        # one sequence with a long context, an 8192-wide layer with eight key/value heads: split along the context
        _attend("attend_b1_65537_gqa", "bf16", 1, 64, 8, 128, 64, 0, 65537, 1, False, False),
        # eight samples of one prompt, 4096-wide layer: the prompt's pages are shared, each sample has its own tail
        _attend("shared_b8_2048", "f16", 8, 32, 32, 128, 16, 2048, 100, 1, True, False),
        # many users behind one long system prompt, 8192-wide layer with grouped heads
        _attend("shared_b64_16384_gqa", "bf16", 64, 64, 8, 128, 32, 16384, 400, 1, True, False),
        # prompt pass of one sequence, 4096-wide layer
        _attend("prompt_b1_2048", "f16", 1, 32, 32, 128, 16, 0, 2048, 2048, False, False),
        # pieces of three prompts behind what the cache already holds, heads of 80, grouped, ragged
        _attend("chunk_b3_6000_d80", "bf16", 3, 32, 8, 80, 32, 0, 6000, 1000, True, True),
        # one decode step's keys and values of sixteen sequences
        {"name": "append_b16", "kind": "append", "dtype": "f16", "B": 16, "kv_heads": 32, "D": 128, "page": 16, "n": 1, "before": 1000, "layers": 1},
        # four prompts admitted in place of four that finished, two layers' keys and values written
        {"name": "admit_b4_1000", "kind": "admit", "dtype": "f16", "B": 4, "kv_heads": 32, "D": 128, "page": 16, "n": 1000, "before": 2000, "layers": 2},
        # sixteen samples forked from two prompts, four layers
        {"name": "fork_2x8", "kind": "fork", "dtype": "f16", "parents": 2, "children": 8, "ctx": 1500, "kv_heads": 8, "D": 128, "page": 16, "layers": 4},
        # sixty-four samples forked from eight prompts, all layers of a deep stack
        {"name": "fork_8x8_32_layers", "kind": "fork", "dtype": "bf16", "parents": 8, "children": 8, "ctx": 700, "kv_heads": 8, "D": 128, "page": 32, "layers": 32},
        # a pool of a thousand pages, three quarters of them live, squeezed to its low end
        {"name": "compact_1024_16_layers", "kind": "compact", "dtype": "f16", "pages": 1024, "fill": 0.75, "rows": 24, "kv_heads": 8, "D": 128, "page": 16, "layers": 16},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["attend", "append", "admit", "fork", "compact"], [7, 1, 1, 2, 2])[0]
    dtype = rng.choice(["f16", "bf16"])
    page = rng.choice([16, 16, 32, 64, 128])
    D = rng.choice([64, 80, 96, 128, 128, 128, 256])
    kv = rng.choice([1, 2, 4, 8, 8, 16, 32])
    while kind == "attend":
        heads = kv * rng.choice([1, 1, 2, 4, 5, 8])
        B, ctx = _log_int(rng, 1, 96), _log_int(rng, 1, 40000)
        shared = rng.choice([0, 0, page * _log_int(rng, 1, max(1, 16384 // page))])
        nq = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 2048)])
        ctx = max(ctx, nq)
        c = {"kind": kind, "dtype": dtype, "B": B, "heads": heads, "kv_heads": kv, "D": D, "page": page, "shared": shared, "ctx": ctx,
             "nq": nq, "ragged": rng.random() < 0.6 and B > 1, "fused": rng.random() < 0.4}
        room = B * nq * heads * (shared + 1.75 * ctx + page) * 4                # the plain form's scores, bytes
        held = B * (1.75 * ctx + page) * kv * D * 8 + shared * kv * D * 8       # ... and keys and values in 32 bits
        if heads <= 64 and room < 4e9 and held < 4e9 and work(c)["flops"] < 7e10 and work(c)["bytes"] < 2.6e8:
            return c
    if kind == "append":
        return {"kind": kind, "dtype": dtype, "B": _log_int(rng, 1, 128), "kv_heads": kv, "D": D, "page": page, "n": rng.choice([1, 1, 2, 4]),
                "before": _log_int(rng, 1, 2000), "layers": 1}
    while kind == "admit":
        c = {"kind": kind, "dtype": dtype, "B": _log_int(rng, 1, 32), "kv_heads": kv, "D": D, "page": page, "n": _log_int(rng, 1, 4000),
             "before": _log_int(rng, 1, 2000), "layers": rng.randint(1, 4)}
        if work(c)["bytes"] < 2.6e8:
            return c
    while kind == "fork":
        c = {"kind": kind, "dtype": dtype, "parents": _log_int(rng, 1, 8), "children": _log_int(rng, 1, 16), "ctx": _log_int(rng, 1, 3000),
             "kv_heads": kv, "D": D, "page": page, "layers": _log_int(rng, 1, 32)}
        if work(c)["bytes"] < 2.6e8 and _fork_pages(c) * _page_bytes(c) * c["layers"] < 1.5e9:
            return c
    while kind == "compact":
        c = {"kind": kind, "dtype": dtype, "pages": _log_int(rng, 20, 8000), "fill": round(rng.uniform(0.2, 0.95), 2), "rows": rng.randint(1, 40),
             "kv_heads": kv, "D": D, "page": page, "layers": _log_int(rng, 1, 32)}
        if work(c)["bytes"] < 4e8 and c["pages"] * _page_bytes(c) * c["layers"] < 1.5e9:
            return c


# ------------------------------------------------------------------ sizes that a case fixes

def _frac(x):
    return x - math.floor(x)


def _sizes(c):
    """Tokens that each sequence holds (shared ones among them) and new ones of them, ragged by a fixed rule."""
    n, nq = [], []
    for b in range(c["B"]):
        q = max(1, int(c["nq"] * (0.3 + 0.7 * _frac(0.4142 * (b + 1))))) if c["ragged"] else c["nq"]
        k = int(c["ctx"] * (0.25 + 1.5 * _frac(0.6180 * (b + 1)))) if c["ragged"] else c["ctx"]
        n.append(c["shared"] + max(q, k))
        nq.append(q)
    return n, nq


def _counts(c):
    """New tokens of each sequence of an append or admit case: equal where they are few, ragged where they are many."""
    return [c["n"] if c["n"] <= 4 else max(1, int(c["n"] * (0.25 + 1.5 * _frac(0.6180 * (b + 1))))) for b in range(c["B"])]


def _pages(tokens, page):
    return (tokens + page - 1) // page


def _page_bytes(c):
    return 2 * c["kv_heads"] * c["page"] * c["D"] * 2


def _fork_ctx(c, i):
    return max(1, int(c["ctx"] * (0.5 + _frac(0.6180 * (i + 1)))))


def _fork_pages(c):
    return sum(_pages(_fork_ctx(c, i), c["page"]) for i in range(c["parents"])) + c["parents"] * c["children"] + 16


def _holes(c):
    live = max(1, int(c["pages"] * c["fill"]))
    return live, min(int(live * (1 - c["fill"])), c["pages"] - live)


def work(case):
    c = case
    row = c["kv_heads"] * c["D"] * 2                                            # bytes of one token's keys, or values
    if c["kind"] == "attend":
        n, nq = _sizes(c)
        keys = c["shared"] + sum(x - c["shared"] for x in n)
        seen = sum(q * x - q * (q - 1) // 2 for x, q in zip(n, nq))             # (row, key) pairs of a head
        return {"bytes": 2 * row * keys + 4 * sum(nq) * c["heads"] * c["D"], "flops": 4 * c["D"] * c["heads"] * seen}
    if c["kind"] in ("append", "admit"):
        return {"bytes": 2 * 2 * row * sum(_counts(c)) * c["layers"], "flops": 0}
    if c["kind"] == "fork":
        pairs = sum(c["children"] for i in range(c["parents"]) if _fork_ctx(c, i) % c["page"])
        return {"bytes": 2 * pairs * _page_bytes(c) * c["layers"] + 8 * _fork_pages(c), "flops": 0}
    return {"bytes": 2 * _holes(c)[1] * _page_bytes(c) * c["layers"] + 8 * c["pages"], "flops": 0}


# ------------------------------------------------------------------ inputs, from the seed alone

def _type(c):
    return {"f16": torch.float16, "bf16": torch.bfloat16}[c["dtype"]]


def _normal(c, g, *shape):
    return torch.randn(*shape, device="cuda", generator=g, dtype=torch.float32).to(_type(c)) if math.prod(shape) < 1 << 26 else \
        torch.empty(*shape, device="cuda", dtype=_type(c)).normal_(generator=g)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(rows, width):
    return _ints([r + [-1] * (width - len(r)) for r in rows])


def _refs(rows, pages):
    n = [0] * pages
    for r in rows:
        for p in r:
            n[p] += 1
    return _ints(n)


def _cache(c, g, layers, pages, rows, width, lengths):
    return {"pool": _normal(c, g, layers, pages, 2, c["kv_heads"], c["page"], c["D"]), "table": _table(rows, width),
            "lengths": _ints(lengths), "refs": _refs(rows, pages)}


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 % (1 << 62))
    order = torch.Generator()
    order.manual_seed(int(seed) * 1000003 % (1 << 62))
    s = {"case": c}
    if c["kind"] == "attend":
        n, nq = _sizes(c)
        sh = c["shared"] // c["page"]
        own_pages = [_pages(x, c["page"]) - sh for x in n]
        pages = sh + sum(own_pages) + 3
        ids = torch.randperm(pages, generator=order).tolist()
        rows, at = [], sh
        for k in own_pages:
            rows.append(ids[:sh] + ids[at:at + k])
            at += k
        s.update(_cache(c, g, 1, pages, rows, max(len(r) for r in rows), n))
        s["shared"] = s["table"][0, :sh].clone() if sh else None
        T, Hq, D = sum(nq), c["heads"], c["D"]
        wide = _normal(c, g, T, Hq + (2 * c["kv_heads"] if c["fused"] else 0), D)
        s["q"] = (wide * 2)[:, :Hq]                                             # of a fused projection: rows lie further apart
        s["q_start"] = _ints([sum(nq[:b]) for b in range(c["B"] + 1)]) if c["nq"] > 1 else None
        s["scale"] = 1.0 / math.sqrt(D)
    elif c["kind"] in ("append", "admit"):
        count = _counts(c)
        after = [c["before"] + k for k in count] if c["kind"] == "append" else count
        # admit: one row more holds a resident sequence, pages all over the pool
        held = [_pages(x, c["page"]) for x in after]
        pages = sum(held) + _pages(c["before"], c["page"]) + 8
        ids = torch.randperm(pages, generator=order).tolist()
        if c["kind"] == "append":
            rows, at = [], 0
            for k in held:
                rows.append(ids[at:at + k])
                at += k
            s.update(_cache(c, g, c["layers"], pages, rows, max(held), after))
            s["start"] = _ints([c["before"]] * c["B"])
        else:
            rows = [[] for _ in held] + [ids[:_pages(c["before"], c["page"])]]
            s.update(_cache(c, g, c["layers"], pages, rows, max(held + [len(rows[-1])]), [0] * c["B"] + [c["before"]]))
            s["rows"], s["count"] = _ints(list(range(c["B"]))), _ints(count + [0])
        T = sum(count)
        s["k"] = [_normal(c, g, T, c["kv_heads"], c["D"]) for _ in range(c["layers"])]
        s["v"] = [_normal(c, g, T, c["kv_heads"], c["D"]) for _ in range(c["layers"])]
        edges = [sum(count[:b]) for b in range(c["B"] + 1)]
        s["q_start"] = _ints(edges if c["kind"] == "append" else edges + [T]) if max(count) > 1 or c["kind"] == "admit" else None
    elif c["kind"] == "fork":
        pages, at, rows, n = _fork_pages(c), 0, [], []
        ids = torch.randperm(pages, generator=order).tolist()
        for i in range(c["parents"]):
            n.append(_fork_ctx(c, i))
            rows.append(ids[at:at + _pages(n[-1], c["page"])])
            at += len(rows[-1])
        kids = c["parents"] * c["children"]
        s.update(_cache(c, g, c["layers"], pages, rows + [[] for _ in range(kids)], max(len(r) for r in rows) + 2, n + [0] * kids))
        s["parent"] = _ints([i for i in range(c["parents"]) for _ in range(c["children"])])
        s["child"] = _ints(list(range(c["parents"], c["parents"] + kids)))
    else:
        live, holes = _holes(c)
        low, high = torch.randperm(live, generator=order), live + torch.randperm(c["pages"] - live, generator=order)
        ids = torch.cat([low[holes:], high[:holes]])
        ids = ids[torch.randperm(live, generator=order)].tolist()
        rows = [ids[i::c["rows"]] for i in range(c["rows"])]
        s.update(_cache(c, g, c["layers"], c["pages"], rows, max(len(r) for r in rows) + 1, [len(r) * c["page"] for r in rows]))
    return s


# ------------------------------------------------------------------ the library's calls

def _run_own(s):
    import paper_2501_16385_amd as fbq
    c = s["case"]
    if "cache" not in s:                                                        # the handle, buffers and workspace that a program keeps
        s["cache"] = fbq.Cache(s["pool"], s["table"], s["lengths"], s["refs"])
        if c["kind"] == "attend":
            s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
            s["workspace"] = fbq.attention_workspace(s["cache"], s["q"], max_q=c["nq"], shared=s["shared"])
        if c["kind"] == "compact":
            s["new"] = fbq.Cache(s["pool"], torch.empty_like(s["table"]), s["lengths"], torch.empty_like(s["refs"]))
            s["info"] = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache = s["cache"]
    if c["kind"] == "attend":
        return fbq.attention(cache, 0, s["q"], q_start=s["q_start"], max_q=c["nq"], shared=s["shared"], scale=s["scale"], out=s["out"],
                             workspace=s["workspace"])
    if c["kind"] in ("append", "admit"):
        start = s.get("start")
        if c["kind"] == "admit":
            fbq.cache_free(cache, s["rows"])
            start = fbq.cache_reserve(cache, s["count"])
        for layer in range(c["layers"]):
            fbq.cache_append(cache, layer, s["k"][layer], s["v"][layer], start, q_start=s["q_start"])
        return {"pool": s["pool"], "table": s["table"], "lengths": s["lengths"], "refs": s["refs"], "start": start}
    if c["kind"] == "fork":
        fbq.cache_free(cache, s["child"])
        fbq.cache_fork(cache, s["parent"], s["child"])
        return {"pool": s["pool"], "table": s["table"], "lengths": s["lengths"], "refs": s["refs"]}
    fbq.cache_compact(cache, out=s["new"], info=s["info"])
    return {"pool": s["pool"], "table": s["new"].table, "refs": s["new"].refs, "live": s["info"][0]}


# ------------------------------------------------------------------ plain forms

def _plain_attend(s):
    c, pool, table = s["case"], s["pool"][0], s["table"].long().clamp(min=0)
    B, Hq, Hk, D, page, nq = c["B"], c["heads"], c["kv_heads"], c["D"], c["page"], c["nq"]
    g, sh = Hq // Hk, c["shared"]
    q, n = s["q"], s["lengths"].long()
    T = q.shape[0]
    edge = s["q_start"].long() if s["q_start"] is not None else torch.arange(B + 1, device="cuda")
    i = torch.arange(nq, device="cuda")
    count = edge[1:] - edge[:-1]
    sees = n[:, None] - count[:, None] + i + 1                                  # keys before which a new token's row ends
    sees = torch.where(i < count[:, None], sees, 0)
    rows = q[(edge[:-1, None] + i).clamp(max=T - 1)].float() * s["scale"]       # [B, nq, Hq, D]
    rows = rows.view(B, nq, Hk, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hk, nq * g, D)
    ends = sees[:, None, :, None].expand(B, 1, nq, g).reshape(B, 1, nq * g, 1)
    own_kv = pool[table[:, sh // page:]].float()                                # [B, pages, 2, Hk, page, D]
    m = own_kv.shape[1] * page
    k, v = own_kv.permute(2, 0, 3, 1, 4, 5).reshape(2, B, Hk, m, D)
    p = torch.matmul(rows, k.transpose(2, 3).contiguous())                      # [B, Hk, nq g, m]
    p.masked_fill_(sh + torch.arange(m, device="cuda") >= ends, -math.inf)
    top = p.amax(3, keepdim=True)
    if sh:                                                                      # the shared tokens once, for the rows of all sequences
        kv = pool[s["shared"].long()].float().permute(1, 2, 0, 3, 4).reshape(2, Hk, sh, D)
        flat = rows.permute(1, 0, 2, 3).reshape(Hk, B * nq * g, D)
        p_sh = torch.matmul(flat, kv[0].transpose(1, 2).contiguous()).view(Hk, B, nq * g, sh)
        p_sh.masked_fill_(torch.arange(sh, device="cuda") >= ends.permute(1, 0, 2, 3), -math.inf)
        top = torch.maximum(top, p_sh.amax(3, keepdim=True).permute(1, 0, 2, 3))
    top = top.clamp(min=-3e38)
    p = p.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v)
    if sh:
        p_sh = p_sh.sub_(top.permute(1, 0, 2, 3)).exp_()
        total = total + p_sh.sum(3, keepdim=True).permute(1, 0, 2, 3)
        o = o + torch.matmul(p_sh.view(Hk, B * nq * g, sh), kv[1]).view(Hk, B, nq * g, D).permute(1, 0, 2, 3)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.view(B, Hk, nq, g, D).permute(0, 2, 1, 3, 4).reshape(B * nq, Hq, D)
    return o[(i < count[:, None]).reshape(-1)].to(q.dtype) if c["nq"] > 1 else o.to(q.dtype)


def _plain_free(s, rows):
    rows = rows.long()
    held = s["table"][rows]
    held = held[held >= 0].long()
    s["refs"].sub_(torch.bincount(held, minlength=s["refs"].numel()).to(torch.int32))
    s["table"][rows] = -1
    s["lengths"][rows] = 0


def _plain_take(s, need):
    """Pages for `need` of each asker, lowest first: (page numbers, who gets them); who comes after the last free page gets none."""
    free = (s["refs"] == 0).nonzero()[:, 0]
    end = need.cumsum(0)
    ok = (end <= free.numel()) | (need == 0)
    who = torch.repeat_interleave(torch.arange(need.numel(), device="cuda"), torch.where(ok, need, 0))
    ids = free[:who.numel()].to(torch.int32)
    s["refs"][ids.long()] = 1
    return ids, who, end - need, ok


def _plain_reserve(s, count):
    page, count, n = s["case"]["page"], count.long(), s["lengths"].long()
    old, new = (n + page - 1) // page, (n + count + page - 1) // page
    fits = new <= s["table"].shape[1]
    need = torch.where(fits, new - old, 0)
    ids, who, first, ok = _plain_take(s, need)
    ok = ok & fits
    s["table"][who, old[who] + torch.arange(who.numel(), device="cuda") - first[who]] = ids
    s["lengths"].copy_(torch.where(ok, n + count, n))
    return torch.where(ok, n, -1).to(torch.int32)


def _plain_append(s, layer, start):
    k, v, page = s["k"][layer], s["v"][layer], s["case"]["page"]
    T = k.shape[0]
    t = torch.arange(T, device="cuda")
    if s["q_start"] is None:
        b, i = t, torch.zeros_like(t)
    else:
        edge = s["q_start"].long()
        b = torch.searchsorted(edge, t, right=True) - 1
        i = t - edge[b]
    pos = start.long()[b] + i
    at, slot = s["table"][b, pos // page].long(), pos % page
    s["pool"][layer, at, 0, :, slot] = k
    s["pool"][layer, at, 1, :, slot] = v


def _plain_fork(s):
    page, parent, child = s["case"]["page"], s["parent"].long(), s["child"].long()
    n = s["lengths"].long()[parent]
    full, part = n // page, (n % page > 0).long()
    ids, who, _, ok = _plain_take(s, part)
    n, full = torch.where(ok, n, 0), torch.where(ok, full, 0)
    at = torch.arange(s["table"].shape[1], device="cuda")
    src = s["table"][parent]
    keep = at < full[:, None]
    s["refs"].add_(torch.bincount(src[keep].long(), minlength=s["refs"].numel()).to(torch.int32))
    s["table"][child] = torch.where(keep, src, -1)
    s["table"][child[who], full[who]] = ids
    s["lengths"][child] = n.to(torch.int32)
    s["pool"][:, ids.long()] = s["pool"][:, src[who, full[who]].long()]


def _plain_compact(s):
    live = s["refs"] > 0
    n = live.sum()
    at = torch.arange(live.numel(), device="cuda")
    holes, movers = (~live & (at < n)).nonzero()[:, 0], (live & (at >= n)).nonzero()[:, 0]
    to = at.clone()
    to[movers] = holes
    s["pool"][:, holes] = s["pool"][:, movers]
    table = torch.where(s["table"] >= 0, to[s["table"].long().clamp(min=0)], -1).to(torch.int32)
    refs = s["refs"].clone()
    refs[holes] = s["refs"][movers]
    refs[movers] = 0
    return {"pool": s["pool"], "table": table, "refs": refs, "live": n.to(torch.int32)}


def run(state):
    if own:
        return _run_own(state)
    s, kind = state, state["case"]["kind"]
    if kind == "attend":
        return _plain_attend(s)
    if kind == "compact":
        return _plain_compact(s)
    start = s.get("start")
    if kind == "fork":
        _plain_free(s, s["child"])
        _plain_fork(s)
        return {"pool": s["pool"], "table": s["table"], "lengths": s["lengths"], "refs": s["refs"]}
    if kind == "admit":
        _plain_free(s, s["rows"])
        start = _plain_reserve(s, s["count"])
    for layer in range(s["case"]["layers"]):
        _plain_append(s, layer, start)
    return {"pool": s["pool"], "table": s["table"], "lengths": s["lengths"], "refs": s["refs"], "start": start}


# ------------------------------------------------------------------ 64 bits, from the definitions

def _exact_attend(s):
    """Token by token and head by head: softmax over the keys the token sees, in the order that the table gives them."""
    c = s["case"]
    n, nq = _sizes(c)
    group = c["heads"] // c["kv_heads"]
    pool, table = s["pool"][0], s["table"].tolist()
    out, at = torch.zeros(sum(nq), c["heads"], c["D"], dtype=torch.float64, device="cuda"), 0
    for b, (tokens, new) in enumerate(zip(n, nq)):
        where = torch.tensor([table[b][j // c["page"]] * c["page"] + j % c["page"] for j in range(tokens)], device="cuda")
        see = torch.arange(tokens, device="cuda")[None, :] <= torch.arange(tokens - new, tokens, device="cuda")[:, None]
        for h in range(c["kv_heads"]):
            k, v = (pool[:, x, h].reshape(-1, c["D"])[where].double() for x in (0, 1))
            for j in range(group):
                z = s["q"][at:at + new, h * group + j].double() @ k.T * s["scale"]
                z[~see] = -math.inf
                out[at:at + new, h * group + j] = torch.exp(z - torch.logsumexp(z, 1, keepdim=True)) @ v
        at += new
    return out


def _exact_pages(s):
    """The page operations with lists, one page after another; the pool in 64 bits."""
    c = s["case"]
    page = c["page"]
    table, lengths, refs = s["table"].tolist(), s["lengths"].tolist(), s["refs"].tolist()
    pool = s["pool"].double()

    def lowest():
        return next((p for p, r in enumerate(refs) if r == 0), None)

    if c["kind"] == "compact":
        live = [p for p, r in enumerate(refs) if r > 0]
        holes = [p for p in range(len(live)) if refs[p] == 0]
        moved = dict(zip([p for p in live if p >= len(live)], holes))
        for a, b in moved.items():
            pool[:, b] = pool[:, a].clone()
        return {"pool": pool, "table": None, "refs": None, "live": None}
    if c["kind"] == "fork":
        for a, b in zip(s["parent"].tolist(), s["child"].tolist()):
            lengths[b] = lengths[a]
            if lengths[a] % page:
                p = lowest()
                refs[p] = 1
                pool[:, p] = pool[:, table[a][lengths[a] // page]]
        return {"pool": pool, "table": None, "lengths": None, "refs": None}
    count = _counts(c)
    start = [0] * c["B"] if c["kind"] == "admit" else s["start"].tolist()
    if c["kind"] == "admit":
        for b, k in enumerate(count):
            for j in range(_pages(k, page)):
                table[b][j] = lowest()
                refs[table[b][j]] = 1
    at = 0
    for b, k in enumerate(count):
        for j in range(0, k):
            p = start[b] + j
            for layer in range(c["layers"]):
                pool[layer, table[b][p // page], 0, :, p % page] = s["k"][layer][at + j].double()
                pool[layer, table[b][p // page], 1, :, p % page] = s["v"][layer][at + j].double()
        at += k
    return {"pool": pool, "table": None, "lengths": None, "refs": None, "start": None}


def exact(case, seed):
    if case["kind"] in ("append", "admit") and sum(_counts(case)) * case["layers"] > 20000:
        return None
    if case["kind"] == "attend" and sum(_sizes(case)[0]) * case["heads"] > 100000000:
        return None
    s = prepare(case, seed)
    return _exact_attend(s) if case["kind"] == "attend" else _exact_pages(s)
