"""Caches in 4 bits for the tests: the layout one nibble at a time, the quantizer in 64 bits, and attention over what codes stand for in 64 bits with derived bounds."""
import math

import torch

from cache_cases import UNIT, make_cache

F16, BF16 = torch.float16, torch.bfloat16


def padded(D):
    return next(n for n in (64, 96, 128, 192, 256) if n >= D)


def groups(D):
    return -(-padded(D) // 64)


def token_bytes(D):
    return padded(D) // 2 + 4 * groups(D)


def nibble(page, D, values, token, feature):
    """Number of the nibble (of the head's bytes in a page) that has this token's code of this feature."""
    DS = padded(D)
    at = token // 16 * 16 * DS                                 # nibbles of 16 tokens
    t = token % 16
    reverse = lambda e: (e & 1) << 2 | (e & 2) | e >> 2
    if not values:
        w, g, e = feature // 32, feature // 8 % 4, feature % 8
        return at + ((t * 4 + g) * (DS // 32) + w) * 8 + reverse(e)
    y, f = feature // 64, feature % 64
    z = 4 if 64 * y + 64 <= DS else 2
    r, j = f // z, f % z
    g, k = t // 4, t % 4
    return at + ((g * 16 + r) * (DS // 32) + 2 * y + j // 2) * 8 + ((j & 1) | (k >> 1) << 1 | (k & 1) << 2)


_maps = {}


def nibbles(page, D, values):
    if (page, D, values) not in _maps:
        _maps[page, D, values] = torch.tensor([[nibble(page, D, values, t, d) for d in range(padded(D))] for t in range(page)])
    return _maps[page, D, values]


def quantize(x):
    """x [.., D] of 16 bits -> (codes, scales, lowest values), each group by the definition in 64 bits."""
    D, most = x.shape[-1], torch.finfo(x.dtype).max
    codes, ss, ms = [], [], []
    for a in range(0, D, 64):
        v = x[..., a:a + 64].double()
        lo, hi = v.amin(-1, keepdim=True) + 0.0, v.amax(-1, keepdim=True)             # (a zero without a sign)
        near = ((hi - lo) / 15).to(x.dtype).view(torch.int16).int()
        s = torch.full_like(lo, math.inf)
        for step in (1, 0, -1):                                # the least number of the type that is enough
            try_ = (near + step).clamp(min=0).short().view(x.dtype).double()
            s = torch.where(15 * try_ >= hi - lo, try_, s)
        below = (s.to(x.dtype).view(torch.int16).int() - 1).clamp(min=0).short().view(x.dtype).double()
        s = torch.where(lo + 15 * s > most, below, s)
        codes.append(torch.where(s > 0, torch.round((v - lo) / s), 0.0).clamp(0, 15))
        ss.append(s)
        ms.append(lo)
    return torch.cat(codes, -1).to(torch.uint8), torch.cat(ss, -1).to(x.dtype), torch.cat(ms, -1).to(x.dtype)


def pack(x, page, garbage=None):
    """x [.., 2, kv_heads, page, D] of 16 bits -> the pool's bytes; features from D on have codes of 0.  Places of x that are NaN have no token: there `garbage`, or codes of 15 and scales that are NaN."""
    D, DS, G = x.shape[-1], padded(x.shape[-1]), groups(x.shape[-1])
    held = ~torch.isnan(x[..., 0])                             # [.., 2, kv_heads, page]
    codes, s, m = quantize(torch.nan_to_num(x))
    codes = torch.nn.functional.pad(codes, (0, DS - D))
    out = torch.full((*x.shape[:-1], token_bytes(D)), 0xFF, dtype=torch.uint8).flatten(-2) if garbage is None else garbage.clone().flatten(-2)
    for i in (0, 1):
        flat = out[..., i, :, :]
        n = torch.stack([flat[..., :page * DS // 2] & 15, flat[..., :page * DS // 2] >> 4], -1).flatten(-2)
        at = nibbles(page, D, bool(i)).flatten()
        n[..., at] = torch.where(held[..., i, :, :, None].expand(*codes[..., i, :, :, :].shape).flatten(-2), codes[..., i, :, :, :].flatten(-2), n[..., at])
        flat[..., :page * DS // 2] = n[..., 0::2] | n[..., 1::2] << 4
        words = torch.zeros(*s[..., i, :, :, :1].shape[:-1], G, 2, dtype=x.dtype)
        words[..., 0], words[..., 1] = m[..., i, :, :, :], s[..., i, :, :, :]
        words = words.flatten(-2).contiguous().view(torch.uint8)
        old = flat[..., page * DS // 2:].unflatten(-1, (page, 4 * G))
        flat[..., page * DS // 2:] = torch.where(held[..., i, :, :, None], words, old).flatten(-2)
    return out.unflatten(-1, (x.shape[-2], token_bytes(D)))


def unpack(pool, dtype, D):
    """The numbers that a pool's bytes stand for, in 64 bits [.., 2, kv_heads, page, D]."""
    page, DS, G = pool.shape[-2], padded(D), groups(D)
    out = torch.empty(*pool.shape[:-1], D, dtype=torch.float64)
    for i in (0, 1):
        flat = pool[..., i, :, :, :].flatten(-2)
        n = torch.stack([flat[..., :page * DS // 2] & 15, flat[..., :page * DS // 2] >> 4], -1).flatten(-2)
        codes = n[..., nibbles(page, D, bool(i))[:, :D].flatten()].unflatten(-1, (page, D)).double()
        words = flat[..., page * DS // 2:].contiguous().view(dtype).double().unflatten(-1, (page, G, 2))
        of = torch.arange(D) // 64
        out[..., i, :, :, :] = words[..., 0][..., of] + words[..., 1][..., of] * codes
    return out


def make_cache4(lengths, kv_heads, D, page, dtype, **how):
    """(pool, table, lengths, refs, what the pool stands for in 64 bits) on the CPU; places without a token hold codes of 15 and scales that are NaN."""
    pool, table, n, refs = make_cache(lengths, kv_heads, D, page, dtype, **how)
    four = pack(pool, page)
    return four, table, n, refs, unpack(four, dtype, D)


def attention4_64(values, table, lengths, layer, q, counts, scale, few):
    """(out, lse, bound of out, bound of lse) in 64 bits, from what the codes stand for.

    few: scores are exact products and 32-bit sums: a probability is off by d = 2 (D + 8) 2^-24 sum_d |q_d| (|k_d| + 2 |m|) scale + 2^-17, |m| <= max |k|; p s is rounded to fp16, 2^-11, and what is
    below its normal numbers loses 2^-25 of 2^e each, at most the largest scale / 16, times a code of 15:  sum_j p_j (|v_j| + max |v|) (2^-11 + d) + u |o| + n 2^-25 max |v|.
    else k and v are rounded to the type as well: independent roundings of up to u |k_d| move a score by six standard deviations of them, 6 u sqrt(sum_d (q_d k_d)^2 / 3) scale, and
    fp16 loses 2^-25 of a p below its normal numbers."""
    T, Hq, D = q.shape
    kv_heads, page = values.shape[3], values.shape[4]
    u = UNIT[q.dtype]
    out, lse = torch.zeros(T, Hq, D, dtype=torch.float64), torch.full((T, Hq), -math.inf, dtype=torch.float64)
    bound, lse_bound = torch.zeros(T, Hq, D, dtype=torch.float64), torch.zeros(T, Hq, dtype=torch.float64)
    t = 0
    for b, c in enumerate(counts):
        n = int(lengths[b])
        pages = table[b, :math.ceil(n / page)].long()
        kv = values[layer, pages].permute(1, 0, 3, 2, 4).reshape(2, -1, kv_heads, D)[:, :n]
        for i in range(c):
            sees = n - c + i + 1
            if sees > 0:
                for h in range(Hq):
                    kk, vv = kv[0, :sees, h * kv_heads // Hq], kv[1, :sees, h * kv_heads // Hq]
                    x = q[t, h].double()
                    z = kk @ x * scale
                    top = z.max()
                    p = torch.exp(z - top)
                    total = p.sum()
                    p = p / total
                    out[t, h] = p @ vv
                    lse[t, h] = top + torch.log(total)
                    size = float((kk.abs() @ x.abs()).max() + 2 * kk.abs().max() * x.abs().sum()) * abs(scale)
                    d = 2 * (D + 8) * 2.0 ** -24 * size + 2.0 ** -17
                    most = vv.abs().amax()
                    if few:
                        lost = sees * 2.0 ** -25 * most / total
                        bound[t, h] = (p @ vv.abs() + most) * (2.0 ** -11 + d) + lost
                    else:
                        d += 6 * u * float((kk * x).pow(2).sum(1).max() / 3) ** 0.5 * abs(scale)
                        bound[t, h] = (p @ vv.abs()) * (2 * u + 2 * d) + (sees * 2.0 ** -25 * most / total if q.dtype == F16 else 0.0)
                    bound[t, h] += u * out[t, h].abs() + 2.0 ** -24
                    lse_bound[t, h] = d + 2.0 ** -20 * abs(lse[t, h])
            t += 1
    return out, lse, bound, lse_bound


def to_cache4(fbq, pool, table, lengths, refs, dtype, D):
    return fbq.Cache(pool.cuda(), table.cuda(), lengths.cuda(), refs.cuda(), dtype=dtype, dim=D)
