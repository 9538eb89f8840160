"""Caches for the attention and page tests: random contents, places that hold no token filled with NaN, and attention in 64 bits."""
import math

import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}       # unit roundoff


def make_cache(lengths, kv_heads, D, page, dtype, shared_pages=0, layers=1, spare=3, seed=0, width=None):
    """(pool, table, lengths, refs) on the CPU.  Rows begin with the same `shared_pages` pages; every place without a token is NaN."""
    g = torch.Generator().manual_seed(seed)
    own = [max(0, math.ceil(n / page) - shared_pages) for n in lengths]
    pages = shared_pages + sum(own) + spare
    ids = torch.randperm(pages, generator=g).tolist()
    width = width or max(1, max(shared_pages + k for k in own))
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32)
    pool = torch.full((layers, pages, 2, kv_heads, page, D), float("nan"), dtype=dtype)
    at = shared_pages
    for b, k in enumerate(own):
        row = ids[:shared_pages] + ids[at:at + k]
        at += k
        table[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
        for p in row:
            refs[p] += 1
        for i, p in enumerate(row):
            n = page if i < shared_pages else min(page, lengths[b] - i * page)
            if n > 0:
                pool[:, p, :, :, :n] = torch.randn(layers, 2, kv_heads, n, D, generator=g).to(dtype)
    return pool, table, torch.tensor(lengths, dtype=torch.int32), refs


def row_tokens(pool, table, layer, b, n):
    """Keys and values [n, kv_heads, D] of a row's first n tokens, in 64 bits."""
    page = pool.shape[4]
    pages = table[b, :math.ceil(n / page)].long()
    kv = pool[layer, pages].permute(1, 0, 3, 2, 4).reshape(2, -1, pool.shape[3], pool.shape[5])[:, :n]
    return kv[0].double(), kv[1].double()


def attention64(pool, table, lengths, layer, q, counts, scale):
    """(out, lse, bound of out, bound of lse) in 64 bits: what rounding the probabilities and the result to the type, and 32-bit scores, can move an element by.

    |o^ - o| <= sum_j p_j |v_j| (u + d) + u |o| + s, u the type's unit roundoff, d the relative error of a probability - twice the score's, D 2^-24 sum_d |q_d k_d| scale,
    and 2^-17 for exponential, sums and the join - and s what probabilities below fp16's normal numbers lose: 2^-25 each.  |lse^ - lse| <= d + 2^-20 |lse|."""
    T, Hq, D = q.shape
    kv_heads = pool.shape[3]
    u = UNIT[q.dtype]
    out, lse, bound = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64), torch.zeros(T, Hq, D, dtype=torch.float64)
    lse_bound = torch.zeros(T, Hq, dtype=torch.float64)
    t = 0
    for b, c in enumerate(counts):
        n = int(lengths[b])
        k, v = row_tokens(pool, table, layer, b, n)
        for i in range(c):
            sees = n - c + i + 1
            if sees > 0:
                for h in range(Hq):
                    kk, vv = k[:sees, h * kv_heads // Hq], v[:sees, h * kv_heads // Hq]
                    x = q[t, h].double()
                    z = kk @ x * scale
                    top = z.max()
                    p = torch.exp(z - top)
                    total = p.sum()
                    out[t, h] = p @ vv / total
                    lse[t, h] = top + torch.log(total)
                    d = 2 * D * 2.0 ** -24 * float((kk.abs() @ x.abs()).max() * abs(scale)) + 2.0 ** -17
                    lse_bound[t, h] = d + 2.0 ** -20 * abs(lse[t, h])
                    lost = sees * 2.0 ** -25 * vv.abs().amax(0) / total if q.dtype == torch.float16 else 0.0
                    bound[t, h] = p @ vv.abs() / total * (u + d) + u * out[t, h].abs() + lost + (2.0 ** -25 if q.dtype == torch.float16 else 1e-40)
            t += 1
    return out, lse, bound, lse_bound


def to_cache(fbq, pool, table, lengths, refs):
    return fbq.Cache(pool.cuda(), table.cuda(), lengths.cuda(), refs.cuda())


def starts(counts):
    edges = [0]
    for c in counts:
        edges.append(edges[-1] + c)
    return torch.tensor(edges, dtype=torch.int32)
