"""Performance cases of the key/value cache held in 4 bits, of attention over it, and of eviction by accumulated attention weight.

listed() names the cases, draw() gives further ones of the same ranges, prepare() makes what a program has in hand before a
call, run() is one pass through an operator, exact() the same outputs from the definition in 64 bits, work() the bytes and
operations that one pass cannot do without.  With `own` false run() computes the plain form, elementary torch operations in
32 bits rounded once at the end; with `own` true it makes the calls of the library.

A cache of 16 bits: pool [layers][pages][K, V][kv_heads][page][D].  One of 4 bits: pool [layers][pages][K, V][kv_heads][page][bytes
a token], in groups of 64 features of a token's head with a scale s and a lowest value m, value = m + s code; its layout is
below (_maps).  table [rows][max_pages] page numbers, -1 where there is none; lengths [rows] tokens held; refs [pages] how
many rows hold a page.

Kinds of case
  attend   attention of the newest tokens of every sequence over the sequence's tokens in a cache of 4 bits, causal; the
           first `shared` tokens lie in the same pages for all sequences
  append   keys and values of new tokens quantized into a cache of 4 bits, and the tokens read back as the values they stand for
  weigh    the attention weights of the newest tokens added up, key by key and key/value head by key/value head, over a
           cache of 16 or 4 bits; sums of earlier calls fade by a factor, new tokens begin at nothing
  evict    a step's tokens get pages, and every row is cut back to `keep` tokens in all layers: the first and the most recent
           ones, and those of the others with the largest weights, ties to the earlier one
"""
from __future__ import annotations

import math

import torch

own = False


# ------------------------------------------------------------------ the cases

def _attend(name, dtype, B, heads, kv_heads, D, page, shared, ctx, nq, ragged, fused):
    return {"name": name, "kind": "attend", "bits": 4, "dtype": dtype, "B": B, "heads": heads, "kv_heads": kv_heads, "D": D, "page": page,
            "shared": shared, "ctx": ctx, "nq": nq, "ragged": ragged, "fused": fused}


def _append(name, dtype, B, kv_heads, D, page, n, before):
    return {"name": name, "kind": "append", "bits": 4, "dtype": dtype, "B": B, "kv_heads": kv_heads, "D": D, "page": page, "n": n, "before": before}


def _weigh(name, bits, dtype, B, heads, kv_heads, D, page, ctx, nq, ragged, decay):
    return {"name": name, "kind": "weigh", "bits": bits, "dtype": dtype, "B": B, "heads": heads, "kv_heads": kv_heads, "D": D, "page": page,
            "shared": 0, "ctx": ctx, "nq": nq, "ragged": ragged, "fused": False, "decay": decay}


def _evict(name, dtype, B, kv_heads, D, page, layers, keep, drop, first, recent):
    return {"name": name, "kind": "evict", "bits": 16, "dtype": dtype, "B": B, "kv_heads": kv_heads, "D": D, "page": page, "layers": layers,
            "keep": keep, "drop": drop, "first": first, "recent": recent}


def listed():
    return [
        # the smallest call: one sequence just begun, one token through the heads of a 4096-wide layer
        _attend("attend4_b1_33", "f16", 1, 32, 32, 128, 16, 0, 33, 1, False, False),
        # sixteen sequences decoded together, ragged contexts around a thousand tokens, q a slice of a fused projection
        _attend("attend4_b16_1000", "f16", 16, 32, 32, 128, 16, 0, 1000, 1, True, True),
        # one sequence with a long context, an 8192-wide layer with eight key/value heads: split along the context
        _attend("attend4_b1_65537_gqa", "bf16", 1, 64, 8, 128, 64, 0, 65537, 1, False, False),
        # samples of one long prompt, its pages shared, grouped heads
        _attend("attend4_shared_b24_8192", "bf16", 24, 64, 8, 128, 32, 8192, 300, 1, True, False),
        # pieces of three prompts behind what the cache already holds, heads of 80, grouped, ragged
        _attend("attend4_chunk_b3_6000_d80", "f16", 3, 32, 8, 80, 32, 0, 6000, 1000, True, True),
        # one decode step's keys and values of sixteen sequences
        _append("append4_b16", "f16", 16, 32, 128, 16, 1, 1000),
        # four prompts of about a thousand tokens written behind a few that are there, ragged
        _append("append4_b4_1000", "bf16", 4, 32, 128, 16, 1000, 21),
        # the weights of a decode step of sixteen sequences
        _weigh("weigh_b16_1000", 16, "f16", 16, 32, 32, 128, 16, 1000, 1, True, 1.0),
        # the weights of a prompt's last piece over all of it, 4-bit cache, grouped heads
        _weigh("weigh4_b2_4000_gqa", 4, "bf16", 2, 32, 8, 128, 32, 4000, 512, False, 0.5),
        # one sequence over its budget
        _evict("evict_b1_512", "f16", 1, 32, 128, 16, 2, 512, 64, 4, 64),
        # sixteen sequences cut back together, all of a stack's layers that one call has
        _evict("evict_b16_1024", "f16", 16, 8, 128, 16, 4, 1024, 256, 16, 128),
        # long contexts, heads of 80
        _evict("evict_b3_6000_d80", "bf16", 3, 8, 80, 32, 4, 6000, 2500, 0, 500),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["attend", "append", "weigh", "evict"], [6, 2, 3, 3])[0]
    c = {"kind": kind, "bits": 4, "dtype": rng.choice(["f16", "bf16"]), "page": rng.choice([16, 16, 32, 64, 128]),
         "D": rng.choice([64, 80, 96, 128, 128, 128, 256]), "kv_heads": rng.choice([1, 2, 4, 8, 8, 16, 32])}
    while True:
        if kind in ("attend", "weigh"):
            B, ctx = _log_int(rng, 1, 64), _log_int(rng, 1, 40000)
            nq = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 1024)])
            c.update(heads=c["kv_heads"] * rng.choice([1, 1, 2, 4, 5, 8]), B=B, ctx=max(ctx, nq), nq=nq, ragged=rng.random() < 0.6 and B > 1, shared=0, fused=False)
            if kind == "attend":
                c.update(shared=rng.choice([0, 0, c["page"] * _log_int(rng, 1, max(1, 8192 // c["page"]))]), fused=rng.random() < 0.4)
            else:
                c.update(bits=rng.choice([4, 16]), decay=rng.choice([1.0, 1.0, 0.9, 0.0]))
            room = B * nq * c["heads"] * (c["shared"] + 1.75 * ctx + c["page"]) * 4                     # the plain form's scores, bytes
            held = (B * (1.75 * ctx + c["page"]) + c["shared"]) * c["kv_heads"] * c["D"] * 8            # ... and keys and values in 32 bits
            if c["heads"] <= 64 and room < 3e9 and held < 3e9 and work(c)["flops"] < 3.5e10 and work(c)["bytes"] < 1.0e8:
                return c
        elif kind == "append":
            c.update(B=_log_int(rng, 1, 64), n=rng.choice([1, 1, 2, 4, _log_int(rng, 5, 3000)]), before=_log_int(rng, 1, 2000))
            if work(c)["bytes"] < 2.5e8:
                return c
        else:
            keep = _log_int(rng, 32, 8000)
            c.update(bits=16, B=_log_int(rng, 1, 32), layers=_log_int(rng, 1, 16), keep=keep, drop=max(1, int(keep * rng.uniform(0.02, 1.0))),
                     first=rng.choice([0, 4, keep // 8]), recent=rng.choice([1, keep // 8, keep // 4]))
            if work(c)["bytes"] < 5e8:
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
    """New tokens of each sequence of an append case: equal where they are few, ragged where they are many."""
    return [c["n"] if c["n"] <= 4 else max(1, int(c["n"] * (0.25 + 1.5 * _frac(0.6180 * (b + 1))))) for b in range(c["B"])]


def _drops(c):
    """Tokens by which each row of an evict case is over its budget."""
    return [max(1, int(c["drop"] * (0.5 + 0.5 * _frac(0.6180 * (b + 1))))) for b in range(c["B"])]


def _pages(tokens, page):
    return (tokens + page - 1) // page


def _row_bytes(c, bits):
    """Bytes of one token's keys, or values: codes, and a scale and a lowest value for 64 features."""
    return c["kv_heads"] * (2 * c["D"] if bits == 16 else c["D"] // 2 + 4 * ((c["D"] + 63) // 64))


def work(case):
    c = case
    row = _row_bytes(c, c["bits"])
    if c["kind"] in ("attend", "weigh"):
        n, nq = _sizes(c)
        keys = c["shared"] + sum(x - c["shared"] for x in n)
        seen = sum(q * x - q * (q - 1) // 2 for x, q in zip(n, nq))             # (row, key) pairs of a head
        if c["kind"] == "attend":
            return {"bytes": 2 * row * keys + 4 * sum(nq) * c["heads"] * c["D"], "flops": 4 * c["D"] * c["heads"] * seen}
        return {"bytes": (row + 8 * c["kv_heads"]) * keys + sum(nq) * c["heads"] * (2 * c["D"] + 4), "flops": 2 * c["D"] * c["heads"] * seen}
    if c["kind"] == "append":
        tokens = sum(_counts(c))
        return {"bytes": tokens * (2 * _row_bytes(c, 16) + 2 * 2 * row + 2 * 4 * c["kv_heads"] * c["D"]), "flops": 0}
    # the weights once, and each token that stays, but for the first ones, read and written
    return {"bytes": c["layers"] * sum(2 * 2 * row * (c["keep"] - c["first"]) + 4 * c["kv_heads"] * (2 * c["keep"] + k) for k in _drops(c)), "flops": 0}


# ------------------------------------------------------------------ a cache of 4 bits

def _padded(D):
    return next(x for x in (64, 96, 128, 192, 256) if x >= D)


_known = {}


def _maps(page, D):
    """Where the codes of a head's keys, and values, lie in a page: (nibble of [token][feature] for keys, the same for values, and both the other way round).

    DS = 64, 96, 128, 192 or 256 features, the least that holds D; the codes of 16 tokens are one piece of 8 DS bytes, and behind a page's codes lie its
    scales: [token][DS / 64 groups, rounded up] words, m in the lower 16 bits and s in the upper.  Nibble n of a word is bits 4 n ..
    Keys    words [token][g < 4][w < DS / 32]: features 32 w + 8 g + e, e the number n with its three bits in reverse.
    Values  words [g < 4][r < 16][x < DS / 32]: tokens 4 g + k, and features 64 y + z r + j of product 2 x + f = 4 y + j, where z is 4, or 2 in a last half
            group; f is the lowest bit of n and k the others in reverse."""
    if (page, D) not in _known:
        DS, reverse = _padded(D), (0, 4, 2, 6, 1, 5, 3, 7)
        keys, values = torch.zeros(page, DS, dtype=torch.long), torch.zeros(page, DS, dtype=torch.long)
        for block in range(page // 16):
            at = block * 16 * DS
            for g in range(4):
                for w in range(DS // 32):
                    for n in range(8):
                        for t in range(16):
                            keys[16 * block + t, 32 * w + 8 * g + reverse[n]] = at + ((t * 4 + g) * (DS // 32) + w) * 8 + n
                        product = 2 * w + (n & 1)
                        y, j = product // 4, product % 4
                        z = min(4, DS // 16 - 4 * y)
                        k = (n >> 2 & 1) + 2 * (n >> 1 & 1)
                        for r in range(16):
                            values[16 * block + 4 * g + k, 64 * y + z * r + j] = at + ((g * 16 + r) * (DS // 32) + w) * 8 + n
        turned = [torch.empty_like(m.flatten()).index_copy_(0, m.flatten(), torch.arange(m.numel())) for m in (keys, values)]
        _known[page, D] = tuple(m.cuda() for m in (keys[:, :D].flatten(), values[:, :D].flatten(), *turned))
    return _known[page, D]


def _token_bytes(D):
    return _padded(D) // 2 + 4 * ((_padded(D) + 63) // 64)


def _largest(dtype):
    return torch.finfo(dtype).max


def _quantized(x):
    """x [.., D] of 16 bits -> (codes [.., D], scales and lowest values [.., groups] of x's type) for groups of 64 features, in 32 bits.

    m is the group's least value; s the least number of the type with 15 s >= largest - m, or the one before it if m + 15 s were beyond the
    type; a code is (x - m) / s to the nearest, ties to even.  All halved first, so that differences stay in range."""
    D, f = x.shape[-1], x.float() * 0.5
    codes, scales, lows = [], [], []
    for a in range(0, D, 64):
        v = f[..., a:a + 64]
        low, d = v.amin(-1, keepdim=True), v.amax(-1, keepdim=True) - v.amin(-1, keepdim=True)
        s = (d / 7.5).to(x.dtype)
        zero = torch.zeros_like(s)
        up = (s.view(torch.int16) + 1).view(x.dtype)
        s = torch.where(s.float() * 7.5 < d, up, s)
        down = torch.where(s == 0, zero, (s.view(torch.int16) - 1).view(x.dtype))
        s = torch.where(low * 2 + s.float() * 15 > _largest(x.dtype), down, s)
        half = s.float() * 0.5
        q = torch.where(half > 0, (v - low) / half, 0.0)
        codes.append(torch.round(q).clamp(0, 15).to(torch.uint8))
        scales.append(s)
        lows.append((low * 2).to(x.dtype))
    return torch.cat(codes, -1), torch.cat(scales, -1), torch.cat(lows, -1)


def _packed(c, x):
    """[.., 2, kv_heads, page, D] of 16 bits -> the pool's bytes [.., 2, kv_heads, page, bytes a token]."""
    page, D, DS = c["page"], c["D"], _padded(c["D"])
    codes, s, m = _quantized(x)
    codes = torch.nn.functional.pad(codes, (0, DS - D)).flatten(-2)
    turned = _maps(page, D)[2:]
    nibbles = torch.stack([codes[..., i, :, :].index_select(-1, turned[i]) for i in (0, 1)], -3)
    low, high = nibbles[..., 0::2], nibbles[..., 1::2]
    sm = torch.stack([m, s], -1)
    groups = (DS + 63) // 64
    sm = torch.nn.functional.pad(sm.flatten(-2), (0, 2 * (groups - s.shape[-1]))).flatten(-2).contiguous().view(torch.uint8)
    return torch.cat([low | high << 4, sm], -1).view(*x.shape[:-1], _token_bytes(D))


def _values(c, pages, x):
    """The pages' bytes [.., kv_heads, page, bytes a token] of keys (x = 0) or values (1) as the numbers that they stand for, 32 bits [.., kv_heads, page, D]."""
    page, D, DS = c["page"], c["D"], _padded(c["D"])
    flat = pages.flatten(-2)
    at = _maps(page, D)[x]
    codes = flat.index_select(-1, at >> 1) >> (at & 1) * 4 & 15
    codes = codes.view(*flat.shape[:-1], page, D).float()
    sm = flat[..., page * DS // 2:].contiguous().view(_type(c)).view(*flat.shape[:-1], page, -1, 2).float()
    groups = (D + 63) // 64
    m, s = (sm[..., :groups, i].repeat_interleave(64, -1)[..., :D] for i in (0, 1))
    return m + s * codes


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


def _pool(c, g, layers, pages):
    """Normal keys and values in 16 or 4 bits, a thousand pages at a time."""
    parts = []
    for a in range(0, pages, 1024):
        x = _normal(c, g, layers, min(1024, pages - a), 2, c["kv_heads"], c["page"], c["D"])
        parts.append(_packed(c, x) if c["bits"] == 4 else x)
    return torch.cat(parts, 1) if len(parts) > 1 else parts[0]


def _cache(c, g, layers, pages, rows, width, lengths):
    return {"pool": _pool(c, g, layers, pages), "table": _table(rows, width), "lengths": _ints(lengths), "refs": _refs(rows, pages)}


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 % (1 << 62))
    order = torch.Generator()
    order.manual_seed(int(seed) * 1000003 % (1 << 62))
    s = {"case": c}
    if c["kind"] in ("attend", "weigh"):
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
        if c["kind"] == "weigh":
            width = s["table"].shape[1] * c["page"]
            s["lse"] = _lse(s)                                                  # as the attention of the same step left it
            s["weights"] = torch.rand(c["B"], c["kv_heads"], width, device="cuda", generator=g).pow_(6) * 4
            s["out"] = torch.zeros_like(s["weights"])
    elif c["kind"] == "append":
        count = _counts(c)
        held = [_pages(c["before"] + k, c["page"]) for k in count]
        ids = torch.randperm(sum(held) + 8, generator=order).tolist()
        rows, at = [], 0
        for k in held:
            rows.append(ids[at:at + k])
            at += k
        s.update(_cache(c, g, 1, sum(held) + 8, rows, max(held), [c["before"] + k for k in count]))
        s["start"] = _ints([c["before"]] * c["B"])
        T = sum(count)
        s["k"], s["v"] = (_normal(c, g, T, c["kv_heads"], c["D"]) for _ in range(2))
        s["q_start"] = _ints([sum(count[:b]) for b in range(c["B"] + 1)]) if max(count) > 1 else None
    else:
        drop, held = _drops(c), _pages(c["keep"], c["page"])
        most = _pages(c["keep"] + max(drop), c["page"])
        pages = sum(_pages(c["keep"] + k, c["page"]) for k in drop) + 5
        ids = torch.randperm(pages, generator=order).tolist()
        rows = [ids[i * held:(i + 1) * held] for i in range(c["B"])]
        s.update(_cache(c, g, c["layers"], pages, rows, most, [c["keep"]] * c["B"]))
        s["count"], s["keep"] = _ints(drop), _ints([c["keep"]] * c["B"])
        width = most * c["page"]
        w = torch.randn(c["layers"], c["B"], c["kv_heads"], width, device="cuda", generator=g).mul_(2).exp_()
        s["weights"] = torch.where(w < 0.3, 0.0, w)                             # what small weights add up to is nothing: many alike
        s["out"] = torch.zeros_like(w)
    return s


# ------------------------------------------------------------------ the library's calls

def _run_own(s):
    import paper_2501_16385_amd as fbq
    c = s["case"]
    if "cache" not in s:                                                        # the handle, buffers and workspace that a program keeps
        s["cache"] = fbq.Cache(s["pool"], s["table"], s["lengths"], s["refs"], **({"dtype": _type(c), "dim": c["D"]} if c["bits"] == 4 else {}))
        if c["kind"] == "attend":
            s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
            s["workspace"] = fbq.attention_workspace(s["cache"], s["q"], max_q=c["nq"], shared=s["shared"])
        if c["kind"] == "append":
            s["read"] = [torch.empty(s["k"].shape, dtype=torch.float32, device="cuda") for _ in range(2)]
        if c["kind"] == "evict":
            s["workspace"] = fbq.cache_evict_workspace(s["cache"], s["weights"])
    cache = s["cache"]
    if c["kind"] == "attend":
        return fbq.attention(cache, 0, s["q"], q_start=s["q_start"], max_q=c["nq"], shared=s["shared"], scale=s["scale"], out=s["out"], workspace=s["workspace"])
    if c["kind"] == "append":
        fbq.cache_append(cache, 0, s["k"], s["v"], s["start"], q_start=s["q_start"])
        return fbq.cache_read(cache, 0, s["k"].shape[0], s["start"], q_start=s["q_start"], k=s["read"][0], v=s["read"][1])
    if c["kind"] == "weigh":
        return fbq.attention_weights(cache, 0, s["q"], s["lse"], s["weights"], q_start=s["q_start"], max_q=c["nq"], scale=s["scale"], decay=c["decay"], out=s["out"])
    start = fbq.cache_reserve(cache, s["count"])
    fbq.cache_evict(cache, s["weights"], s["keep"], first=c["first"], recent=c["recent"], out=s["out"], workspace=s["workspace"])
    return {"pool": s["pool"], "table": s["table"], "lengths": s["lengths"], "refs": s["refs"], "weights": s["out"], "start": start}


# ------------------------------------------------------------------ plain forms

def _held(s, first, which):
    """Keys (which = 0) or values of every row from page `first` of its table on, 32 bits [B, kv_heads, tokens, D]."""
    c = s["case"]
    pages = s["pool"][0, :, which][s["table"].long().clamp(min=0)[:, first:]]   # [B, pages, kv_heads, page, ..]
    x = _values(c, pages, which) if c["bits"] == 4 else pages.float()
    return x.permute(0, 2, 1, 3, 4).reshape(x.shape[0], c["kv_heads"], -1, c["D"])


def _query_rows(s):
    """(queries [B, kv_heads, nq group, D] in 32 bits, scaled; where each one's sight ends [B, 1, nq group, 1]; new tokens a row [B]; their places in q [B, nq])."""
    c = s["case"]
    B, Hk, nq, g = c["B"], c["kv_heads"], c["nq"], c["heads"] // c["kv_heads"]
    n = s["lengths"].long()
    edge = s["q_start"].long() if s["q_start"] is not None else torch.arange(B + 1, device="cuda")
    i = torch.arange(nq, device="cuda")
    count = edge[1:] - edge[:-1]
    sees = torch.where(i < count[:, None], n[:, None] - count[:, None] + i + 1, 0)
    place = (edge[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    rows = (s["q"].float() * s["scale"])[place].view(B, nq, Hk, g, c["D"]).permute(0, 2, 1, 3, 4).reshape(B, Hk, nq * g, c["D"])
    return rows, sees[:, None, :, None].expand(B, 1, nq, g).reshape(B, 1, nq * g, 1), count, place


def _scores(rows, ends, k, at):
    z = torch.matmul(rows, k.transpose(2, 3).contiguous())
    return z.masked_fill_(at + torch.arange(k.shape[2], device="cuda") >= ends, -math.inf)


def _lse(s):
    """ln of the softmax's sums [T, heads], of the keys in 32 bits."""
    c = s["case"]
    rows, ends, count, place = _query_rows(s)
    z = _scores(rows, ends, _held(s, 0, 0), 0)
    top = z.amax(3, keepdim=True).clamp(min=-3e38)
    lse = (top + z.sub_(top).exp_().sum(3, keepdim=True).log()).view(c["B"], c["kv_heads"], c["nq"], -1).permute(0, 2, 1, 3).reshape(c["B"] * c["nq"], c["heads"])
    return lse[(torch.arange(c["nq"], device="cuda") < count[:, None]).reshape(-1)].contiguous()


def _plain_attend(s):
    c = s["case"]
    B, Hq, Hk, D, nq, sh = c["B"], c["heads"], c["kv_heads"], c["D"], c["nq"], c["shared"]
    g = Hq // Hk
    rows, ends, count, _ = _query_rows(s)
    p = _scores(rows, ends, _held(s, sh // c["page"], 0), sh)
    top = p.amax(3, keepdim=True)
    if sh:                                                                      # the shared tokens once, for the rows of all sequences
        k, v = (_values(c, s["pool"][0, :, x][s["shared"].long()], x).permute(1, 0, 2, 3).reshape(Hk, sh, D) for x in (0, 1))
        flat = rows.permute(1, 0, 2, 3).reshape(Hk, B * nq * g, D)
        p_sh = torch.matmul(flat, k.transpose(1, 2).contiguous()).view(Hk, B, nq * g, sh)
        p_sh.masked_fill_(torch.arange(sh, device="cuda") >= ends.permute(1, 0, 2, 3), -math.inf)
        top = torch.maximum(top, p_sh.amax(3, keepdim=True).permute(1, 0, 2, 3))
    top = top.clamp(min=-3e38)
    p = p.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, _held(s, sh // c["page"], 1))
    if sh:
        p_sh = p_sh.sub_(top.permute(1, 0, 2, 3)).exp_()
        total = total + p_sh.sum(3, keepdim=True).permute(1, 0, 2, 3)
        o = o + torch.matmul(p_sh.view(Hk, B * nq * g, sh), v).view(Hk, B, nq * g, D).permute(1, 0, 2, 3)
    o = torch.where(total > 0, o / total, 0.0)
    o = o.view(B, Hk, nq, g, D).permute(0, 2, 1, 3, 4).reshape(B * nq, Hq, D)
    return o[(torch.arange(nq, device="cuda") < count[:, None]).reshape(-1)].to(s["q"].dtype)


def _places(s):
    """Row and position of every new token of an append case."""
    T = s["k"].shape[0]
    t = torch.arange(T, device="cuda")
    if s["q_start"] is None:
        return t, s["start"].long()
    edge = s["q_start"].long()
    b = torch.searchsorted(edge, t, right=True) - 1
    return b, s["start"].long()[b] + t - edge[b]


def _plain_append(s):
    """Codes and scales into the bytes of the pages' heads that get tokens, and the tokens' values out of them again."""
    c = s["case"]
    page, D, DS = c["page"], c["D"], _padded(c["D"])
    b, pos = _places(s)
    at, slot = s["table"][b, pos // page].long(), pos % page
    touched, which = torch.unique(at, return_inverse=True)
    read = []
    for x, new in ((0, s["k"]), (1, s["v"])):
        old = s["pool"][0, touched, x].flatten(-2)                              # [pages, kv_heads, page * bytes]
        codes, sc, lo = _quantized(new)
        nibbles = torch.stack([old & 15, old >> 4], -1).flatten(-2)
        place = _maps(page, D)[x].view(page, D)[slot]                           # [T, D]
        heads = torch.arange(c["kv_heads"], device="cuda")
        nibbles[which[:, None, None], heads[None, :, None], place[:, None, :]] = codes
        held = nibbles[..., 0::2] | nibbles[..., 1::2] << 4
        sm = torch.stack([lo, sc], -1).flatten(-2).contiguous().view(torch.uint8)       # [T, kv_heads, 4 groups]
        where = page * DS // 2 + slot[:, None] * 4 * ((DS + 63) // 64) + torch.arange(sm.shape[-1], device="cuda")
        held[which[:, None, None], heads[None, :, None], where[:, None, :]] = sm
        held = held.view(touched.numel(), c["kv_heads"], page, _token_bytes(D))
        s["pool"][0, touched, x] = held
        read.append(_values(c, held, x)[which, :, slot])
    return tuple(read)


def _plain_weigh(s):
    c = s["case"]
    rows, ends, count, place = _query_rows(s)
    B, Hk, g = c["B"], c["kv_heads"], c["heads"] // c["kv_heads"]
    z = _scores(rows, ends, _held(s, 0, 0), 0)
    lse = s["lse"][place].view(B, c["nq"], Hk, g).permute(0, 2, 1, 3).reshape(B, Hk, -1, 1)
    new = z.sub_(lse).exp_().sum(2)                                             # [B, kv_heads, tokens]
    j, n = torch.arange(new.shape[2], device="cuda"), s["lengths"].long()
    old = torch.where(j < (n - count)[:, None, None], s["weights"] * c["decay"], 0.0)
    s["out"].copy_(torch.where(j < n[:, None, None], old + new, s["out"]))
    return s["out"]


def _plain_reserve(s):
    page, count, n = s["case"]["page"], s["count"].long(), s["lengths"].long()
    old, new = (n + page - 1) // page, (n + count + page - 1) // page
    free = (s["refs"] == 0).nonzero()[:, 0]
    need = new - old
    who = torch.repeat_interleave(torch.arange(need.numel(), device="cuda"), need)
    ids = free[:who.numel()]
    s["refs"][ids] = 1
    s["table"][who, old[who] + torch.arange(who.numel(), device="cuda") - (need.cumsum(0) - need)[who]] = ids.to(torch.int32)
    s["lengths"].copy_(n + count)
    return n.to(torch.int32)


def _plain_evict(s):
    c = s["case"]
    page, keep = c["page"], c["keep"]
    start = _plain_reserve(s)
    n = s["lengths"].long()
    w, j = s["weights"], torch.arange(s["weights"].shape[-1], device="cuda")
    held = j < n[:, None]                                                       # [rows, width]
    always = held & ((j < c["first"]) | (j >= n[:, None] - c["recent"]))
    key = torch.where(always[:, None], math.inf, torch.where(held[:, None], w, -1.0))
    best = torch.sort(key, dim=-1, descending=True, stable=True)[1][..., :keep]
    src = torch.sort(best, dim=-1)[0]                                           # [layers, rows, kv_heads, keep], ascending
    s["out"].copy_(torch.where(j < keep, torch.nn.functional.pad(torch.gather(w, 3, src), (0, w.shape[-1] - keep)), torch.where(held[:, None], 0.0, s["out"])))
    dst = torch.arange(keep, device="cuda")
    heads = torch.arange(c["kv_heads"], device="cuda")[:, None]
    for b in range(c["B"]):
        pages = s["table"][b].long()
        for layer in range(c["layers"]):
            from_page, from_slot = pages[src[layer, b] // page], src[layer, b] % page           # [kv_heads, keep]
            moved = s["pool"][layer, from_page, :, heads, from_slot]                            # [kv_heads, keep, 2, D]
            s["pool"][layer, pages[dst // page][None], :, heads, (dst % page)[None]] = moved
    at = torch.arange(s["table"].shape[1], device="cuda")
    gone = (at >= _pages(keep, page)) & (s["table"] >= 0)
    s["refs"].index_add_(0, s["table"][gone].long(), torch.full((int(gone.sum()),), -1, dtype=torch.int32, device="cuda"))
    s["table"][gone] = -1
    s["lengths"].copy_(torch.minimum(n, s["keep"].long()))
    return {"pool": s["pool"], "table": s["table"], "lengths": s["lengths"], "refs": s["refs"], "weights": s["out"], "start": start}


def run(state):
    if own:
        return _run_own(state)
    return {"attend": _plain_attend, "append": _plain_append, "weigh": _plain_weigh, "evict": _plain_evict}[state["case"]["kind"]](state)


# ------------------------------------------------------------------ 64 bits, from the definitions

def _decoded(s, which):
    """A layer's keys or values in 64 bits [pages, kv_heads, page, D], word by word as the layout says."""
    c = s["case"]
    pool = s["pool"][0, :, which]
    if c["bits"] == 16:
        return pool.double()
    page, D, DS = c["page"], c["D"], _padded(c["D"])
    P, H = pool.shape[:2]
    flat = pool.reshape(P, H, -1)
    words = flat[..., :page * DS // 2].contiguous().view(torch.int32).view(P, H, page // 16, 8 * DS // 4)
    code = torch.zeros(P, H, page // 16, 16, DS, dtype=torch.float64, device="cuda")
    for n in range(8):
        nibble = (words >> 4 * n & 15).double()
        if which == 0:
            e = (n & 1) * 4 + (n & 2) + (n >> 2)
            code.view(P, H, page // 16, 16, DS // 32, 4, 8)[..., e] = nibble.view(P, H, page // 16, 16, 4, DS // 32).transpose(-1, -2)
            continue
        k = (n >> 2) + (n & 2)
        nibble = nibble.view(P, H, page // 16, 4, 16, DS // 32)
        for x in range(DS // 32):
            y, j = divmod(2 * x + n % 2, 4)
            z = 4 if 64 * y + 64 <= DS else 2
            code[:, :, :, k::4, 64 * y + j:64 * y + 16 * z:z] = nibble[..., x]
    sm = flat[..., page * DS // 2:].contiguous().view(_type(c)).double().view(P, H, page, -1, 2)
    feature = torch.arange(D, device="cuda") // 64
    return sm[..., 0][..., feature] + sm[..., 1][..., feature] * code.view(P, H, page, DS)[..., :D]


def _exact_attend(s):
    """Token by token and head by head: softmax over the keys the token sees, in the order that the table gives them; weights or the values they weigh."""
    c = s["case"]
    n, nq = _sizes(c)
    group, page = c["heads"] // c["kv_heads"], c["page"]
    weigh = c["kind"] == "weigh"
    keys, values, table = _decoded(s, 0), None if weigh else _decoded(s, 1), s["table"].tolist()
    out, at = torch.zeros(sum(nq), c["heads"], c["D"], dtype=torch.float64, device="cuda"), 0
    total = s["out"].double() if weigh else None
    for b, (tokens, new) in enumerate(zip(n, nq)):
        pages = torch.tensor(table[b][:_pages(tokens, page)], device="cuda")
        see = torch.arange(tokens, device="cuda")[None, :] <= torch.arange(tokens - new, tokens, device="cuda")[:, None]
        for h in range(c["kv_heads"]):
            k = keys[pages, h].reshape(-1, c["D"])[:tokens]
            if weigh:
                total[b, h, :tokens] = s["weights"][b, h, :tokens].double() * c["decay"]
                total[b, h, tokens - new:tokens] = 0
            else:
                v = values[pages, h].reshape(-1, c["D"])[:tokens]
            for j in range(group):
                z = s["q"][at:at + new, h * group + j].double() @ k.T * s["scale"]
                z[~see] = -math.inf
                if weigh:
                    total[b, h, :tokens] += torch.exp(z - s["lse"][at:at + new, h * group + j, None].double()).sum(0)
                else:
                    out[at:at + new, h * group + j] = torch.exp(z - torch.logsumexp(z, 1, keepdim=True)) @ v
        at += new
    return total if weigh else out


def _exact_append(s):
    """Group by group in 64 bits: the scale by looking at the numbers of the type around (largest - least) / 15."""
    c = s["case"]
    dtype = _type(c)
    out = []
    for x in (s["k"], s["v"]):
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for a in range(0, c["D"], 64):
            v = x[..., a:a + 64].double()
            low, high = v.min(-1, keepdim=True)[0], v.max(-1, keepdim=True)[0]
            near = ((high - low) / 15).to(dtype).view(torch.int16)
            around = torch.stack([(near + i).clamp(min=0).view(dtype).double() for i in (-1, 0, 1)])
            s_ = torch.where(15 * around >= high - low, around, math.inf).amin(0)
            code = torch.where(s_ > 0, torch.round((v - low) / s_), 0.0)
            y[..., a:a + 64] = low + s_ * code
        out.append(y)
    return tuple(out)


def _exact_evict(s):
    """Row by row with sorted lists of (weight, place); the pool in 64 bits."""
    import numpy
    c = s["case"]
    page, keep = c["page"], c["keep"]
    table, refs = s["table"].tolist(), s["refs"].tolist()
    pool, weights, out = s["pool"].double(), s["weights"].cpu().numpy(), s["out"].double().cpu().numpy()
    for b, drop in enumerate(_drops(c)):
        tokens, row = keep + drop, [p for p in table[b] if p >= 0]
        while len(row) < _pages(tokens, page):
            row.append(refs.index(0))
            refs[row[-1]] = 1
        row = torch.tensor(row, device="cuda")
        for layer in range(c["layers"]):
            for h in range(c["kv_heads"]):
                w = weights[layer, b, h, :tokens]
                middle = numpy.arange(c["first"], tokens - c["recent"])
                by_weight = middle[numpy.lexsort((middle, -w[middle]))]
                stay = numpy.sort(numpy.concatenate([numpy.arange(c["first"]), by_weight[:keep - c["first"] - c["recent"]], numpy.arange(tokens - c["recent"], tokens)]))
                out[layer, b, h, :keep], out[layer, b, h, keep:tokens] = w[stay], 0
                stay = torch.from_numpy(stay).cuda()
                held = pool[layer, row, :, h].transpose(0, 1).reshape(2, -1, c["D"])
                held[:, :keep] = held[:, stay].clone()
                pool[layer, row, :, h] = held.view(2, -1, page, c["D"]).transpose(0, 1)
    return {"pool": pool, "table": None, "lengths": None, "refs": None, "weights": torch.from_numpy(out).cuda(), "start": None}


def exact(case, seed):
    if case["kind"] == "evict" and work(case)["bytes"] > 1.2e9:
        return None
    s = prepare(case, seed)
    return {"attend": _exact_attend, "weigh": _exact_attend, "append": _exact_append, "evict": _exact_evict}[case["kind"]](s)
