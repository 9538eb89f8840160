"""Attention weights added up over calls, and rows cut back by them, against plain implementations in 64 bits and Python lists, over caches of 16 and of 4 bits."""
import math

import pytest
import torch

from cache4_cases import BF16, F16, make_cache4, to_cache4
from cache_cases import make_cache, starts

pytestmark = pytest.mark.gpu


def any_cache(bits, lengths, kv_heads, D, page, dtype, **how):
    """(cache on the device, table, what the pool stands for in 64 bits)"""
    import paper_2501_16385_amd as fbq
    if bits == 4:
        pool, table, n, refs, values = make_cache4(lengths, kv_heads, D, page, dtype, **how)
        return to_cache4(fbq, pool, table, n, refs, dtype, D), table, values
    pool, table, n, refs = make_cache(lengths, kv_heads, D, page, dtype, **how)
    return fbq.Cache(pool.cuda(), table.cuda(), n.cuda(), refs.cuda()), table, pool.double()


def weights64(values, table, lengths, layer, q, lse, counts, scale, before, decay, out):
    """(what the call leaves in out, how far off each may be): a weight's exponent is off by D + 8 roundings of 32-bit sums over |q| (|k| + 2 max |k|) and of z and lse themselves."""
    T, Hq, D = q.shape
    kv_heads, page = values.shape[3], values.shape[4]
    want, bound = out.double().clone(), torch.zeros_like(out, dtype=torch.float64)
    width, t = out.shape[2], 0
    for b, c in enumerate(counts):
        if c == 0:                                             # (left as it is)
            continue
        n = int(lengths[b])
        m = min(n, width)
        k = values[layer, table[b, :math.ceil(n / page)].long(), 0].permute(1, 0, 2, 3).reshape(kv_heads, -1, D)[:, :n]
        want[b, :, :m] = before[b, :, :m].double() * decay if before is not None and decay else 0.0
        want[b, :, max(0, n - c):m] = 0.0
        bound[b, :, :m] = want[b, :, :m].abs() * 2.0 ** -22
        for i in range(c):
            sees = n - c + i + 1
            for h in range(Hq if sees > 0 else 0):
                hk = h * kv_heads // Hq
                x = q[t + i, h].double()
                z = k[hk, :sees] @ x * scale
                p = torch.exp(z - float(lse[t + i, h]))
                size = (k[hk, :sees].abs() @ x.abs() + 2 * k[hk, :sees].abs().max() * x.abs().sum()) * abs(scale)
                d = (D + 8) * 2.0 ** -24 * size + 2.0 ** -21 * (z.abs() + abs(float(lse[t + i, h])) + 1)
                m_ = min(sees, width)
                want[b, hk, :m_] += p[:m_]
                bound[b, hk, :m_] += (p * (d + (c * Hq // kv_heads + 8) * 2.0 ** -24))[:m_] + 1e-38
        t += c
    return want, bound


def check_weights(bits, lengths, counts, heads, kv_heads, D, page, dtype, seed=0, decay=1.0, width=None, layer=0, layers=1, fused=0, scale=None, fresh=False, token_form=None, apart=False):
    import paper_2501_16385_amd as fbq
    cache, table, values = any_cache(bits, lengths, kv_heads, D, page, dtype, seed=seed, layers=layers)
    T = sum(counts)
    g = torch.Generator().manual_seed(seed + 1)
    wide = (torch.randn(T, heads + fused, D, generator=g) * 2).to(dtype)
    q = wide.cuda()[:, :heads]
    single = all(c == 1 for c in counts) if token_form is None else token_form
    q_start = None if single else starts(counts).cuda()
    lse = torch.empty(T, heads, device="cuda")
    fbq.attention(cache, layer, q, q_start=q_start, max_q=max(counts), scale=scale, lse=lse)
    width = width or table.shape[1] * page
    before = torch.rand(len(lengths), kv_heads, width, generator=g)
    for b, n in enumerate(lengths):                            # where a new token begins lies anything
        before[b, :, max(0, n - counts[b]):] = math.nan
    out = torch.full_like(before, 77.0) if apart else before.clone()
    want, bound = weights64(values, table, lengths, layer, wide[:, :heads], lse.cpu(), counts, D ** -0.5 if scale is None else scale, None if fresh else before, decay, out)
    dev = before.cuda()
    got = fbq.attention_weights(cache, layer, q, lse, None if fresh else dev, q_start=q_start, max_q=max(counts), scale=scale, decay=decay, out=out.cuda() if apart or fresh else None)
    torch.cuda.synchronize()
    if not apart and not fresh:
        assert got is dev
    got = got.cpu()
    for b, n in enumerate(lengths):
        m = min(n, width)
        if counts[b] == 0:
            assert torch.equal(torch.nan_to_num(got[b], nan=-1.0), torch.nan_to_num(out[b], nan=-1.0))
            continue
        off = (got[b, :, :m].double() - want[b, :, :m]).abs()
        assert (off <= bound[b, :, :m]).all(), (b, float((off / bound[b, :, :m].clamp(min=1e-300)).max()))
        assert torch.equal(torch.nan_to_num(got[b, :, m:], nan=-1.0), torch.nan_to_num(out[b, :, m:], nan=-1.0))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 64, 80, 96, 128, 136, 192, 256])
def test_weights_of_single_tokens(D, dtype, bits):
    check_weights(bits, [1, 33, 0, 15, 16, 65, 300], [1] * 7, 4, 2, D, 16, dtype, seed=D)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("heads,kv_heads,max_count", [(4, 4, 5), (8, 1, 8), (6, 2, 9), (40, 1, 7), (3, 1, 100), (4, 2, 33)])
def test_weights_of_several_tokens(heads, kv_heads, max_count, bits):
    lengths, counts = [120, 40, 9, 333], [max_count, 1, min(3, max_count), 0]
    lengths = [max(n, c) for n, c in zip(lengths, counts)]
    check_weights(bits, lengths, counts, heads, kv_heads, 64, 16, F16, seed=heads, decay=0.5)
    check_weights(bits, lengths, counts, heads, kv_heads, 128, 32, BF16, seed=heads, apart=True)


@pytest.mark.parametrize("bits", [16, 4])
def test_weights_of_prompts_and_tokens_that_see_nothing(bits):
    check_weights(bits, [150, 64, 1], [150, 30, 1], 4, 2, 96, 16, BF16, seed=1)
    check_weights(bits, [3, 50, 0], [5, 2, 4], 4, 4, 64, 16, F16, seed=1)
    check_weights(bits, [30, 50, 0], [45, 40, 33], 4, 4, 64, 16, F16, seed=2, fresh=True)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("how", [dict(decay=0.0), dict(fresh=True), dict(width=100), dict(width=1), dict(layer=2, layers=3), dict(fused=3), dict(scale=0.0), dict(scale=-0.2), dict(token_form=False)])
def test_weights_forms(how, bits):
    check_weights(bits, [90, 257, 40], [1, 1, 1], 4, 2, 64, 16, F16, seed=5, **how)


@pytest.mark.parametrize("bits", [16, 4])
def test_weights_of_long_rows_and_many(bits):
    check_weights(bits, [9000, 5, 3001], [1] * 3, 2, 1, 64, 16, F16, seed=3)
    check_weights(bits, [7 * b for b in range(150)], [1] * 150, 2, 2, 16, 16, BF16, seed=4)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("rows", [16, 33])
@pytest.mark.parametrize("heads", [96, 128])
def test_weights_of_many_heads_and_tokens(heads, rows, bits):
    """Enough keys that two waves, or one, and not four, share 64 of them; 3 and 4 heads to one of the keys', so that a tile ends inside a token, and not."""
    check_weights(bits, [128, 100, 61] + [20 + b for b in range(rows - 3)], [40, 33, 17] + [2] * (rows - 3), heads, 32, 64, 16, BF16 if heads == 96 else F16, seed=rows, decay=0.25)


@pytest.mark.parametrize("bits", [16, 4])
def test_weights_sum_to_what_was_asked(bits):
    """Each query's weights are one in all: the sums over a row's keys are its queries times heads; equal calls give equal bits."""
    import paper_2501_16385_amd as fbq
    cache, table, _ = any_cache(bits, [200, 70], 2, 128, 16, F16)
    counts = [40, 3]
    q = torch.randn(43, 8, 128, generator=torch.Generator().manual_seed(3)).half().cuda()
    lse, qs = torch.empty(43, 8, device="cuda"), starts(counts).cuda()
    fbq.attention(cache, 0, q, q_start=qs, max_q=40, lse=lse)
    outs = [fbq.attention_weights(cache, 0, q, lse, None, q_start=qs, max_q=40, out=torch.zeros(2, 2, table.shape[1] * 16, device="cuda")) for _ in range(3)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    # 128-feature scores in half precision operands: attention's lse and these weights agree to 2^-9
    for b in (0, 1):
        assert ((outs[0][b].sum(1) - counts[b] * 4).abs() < counts[b] * 4 * 2.0 ** -9).all()


# ------------------------------------------------------------------ eviction

def evicted(values, table, refs, lengths, weights, keep, first, recent, page):
    """The same with lists: (pool, table, refs, lengths, weights, rows cut back, rows skipped)."""
    values, table, refs, lengths, weights = values.clone(), table.clone(), refs.clone(), list(lengths), weights.clone()
    layers, heads = values.shape[0], values.shape[3]
    held, done, skipped = refs.clone(), 0, 0
    for b, n in enumerate(lengths):
        k = keep[b]
        if k < 0 or k >= n:
            continue
        pages = [int(p) for p in table[b, :math.ceil(n / page)]]
        if k < first + recent or n > weights.shape[3] or any(p < 0 or p >= refs.numel() or int(held[p]) != 1 for p in pages[first // page:]):
            skipped += 1
            continue
        done += 1
        where = torch.tensor([pages[j // page] * page + j % page for j in range(n)])
        for layer in range(layers):
            for h in range(heads):
                w = weights[layer, b, h].numpy().copy()
                # (what is no number below everything)
                middle = sorted(range(first, n - recent), key=lambda j: (math.isnan(w[j]), -float(w[j]) if not math.isnan(w[j]) else 0.0, j))
                stay = sorted(list(range(first)) + middle[:k - first - recent] + list(range(n - recent, n)))
                for x in (0, 1):
                    flat = values[layer, :, x, h].reshape(-1, values.shape[5])
                    flat[where[:k]] = flat[where[torch.tensor(stay, dtype=torch.long)]].clone() if k else flat[where[:0]]
                    values[layer, :, x, h] = flat.view(values.shape[1], page, -1)
                weights[layer, b, h, :k] = torch.from_numpy(w[stay]) if k else weights[layer, b, h, :0]
                weights[layer, b, h, k:n] = 0
        for e in range(math.ceil(k / page), math.ceil(n / page)):
            refs[int(table[b, e])] -= 1
            table[b, e] = -1
        lengths[b] = k
    return values, table, refs, lengths, weights, done, skipped


def check_evict(bits, lengths, keep, first, recent, kv_heads, D, page, dtype, layers=2, seed=0, width=None, weights=None, apart=False, table_change=None, held=()):
    import paper_2501_16385_amd as fbq
    cache, table, values = any_cache(bits, lengths, kv_heads, D, page, dtype, seed=seed, layers=layers)
    g = torch.Generator().manual_seed(seed + 1)
    width = width or table.shape[1] * page
    w = torch.randn(layers, len(lengths), kv_heads, width, generator=g).exp() if weights is None else weights(torch.rand(layers, len(lengths), kv_heads, width, generator=g))
    if table_change is not None:
        table_change(table)
        cache.table.copy_(table)
    for p in held:
        cache.refs[int(table[p])] += 1
    refs = cache.refs.cpu()
    raw = cache.pool.cpu()
    want = evicted(values, table, refs, lengths, w, keep, first, recent, page)
    info, dev = torch.full((2,), 9, dtype=torch.int32, device="cuda"), w.cuda()
    workspace = fbq.cache_evict_workspace(cache, dev).fill_(0xFF)
    out = torch.full_like(dev, 5.0) if apart else None
    got = fbq.cache_evict(cache, dev, torch.tensor(keep, dtype=torch.int32, device="cuda"), first=first, recent=recent, out=out, info=info, workspace=workspace)
    torch.cuda.synchronize()
    assert info.tolist() == [want[5], want[6]]
    assert cache.lengths.tolist() == want[3] and torch.equal(cache.table.cpu(), want[1]) and torch.equal(cache.refs.cpu(), want[2])
    # every token that a row holds, and every byte that holds none of a row's
    if bits == 16:
        assert torch.equal(torch.nan_to_num(cache.pool.cpu().double(), nan=-9.0), torch.nan_to_num(want[0], nan=-9.0))
    else:
        from cache4_cases import unpack
        assert torch.equal(torch.nan_to_num(unpack(cache.pool.cpu(), dtype, D), nan=-9.0), torch.nan_to_num(want[0], nan=-9.0))
    same = (lambda a, b: torch.equal(torch.nan_to_num(a, nan=-9.0), torch.nan_to_num(b, nan=-9.0)))
    for b, n in enumerate(lengths):
        if want[3][b] != n or not apart:
            m = min(n, width)
            assert same(got.cpu()[:, b, :, :m], want[4][:, b, :, :m]), b
            assert same(got.cpu()[:, b, :, m:], (w if not apart else torch.full_like(w, 5.0))[:, b, :, m:])
        else:
            assert (got[:, b] == 5.0).all()                    # (a row that is left as it is: nothing written)
    return raw


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 40, 64, 80, 96, 128, 136, 192, 256])
def test_evict_every_head_size(D, dtype, bits):
    check_evict(bits, [100, 40, 77, 5], [64, 39, -1, 0], 0, 0, 2, D, 16, dtype, seed=D)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("first,recent", [(0, 0), (4, 8), (17, 0), (0, 33), (33, 17)])
def test_evict_first_and_recent(first, recent, page, bits):
    check_evict(bits, [300, 50, 51, 129], [150, 50, 50, 128], first, recent, 3, 64, page, F16, seed=page + first, apart=first == 4)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("keep", [1, 2, 3, 4, 5, 15, 16, 17, 255, 256, 257, 1023, 1024, 1500, 2046, 2047])
def test_evict_sizes(keep, bits):
    check_evict(bits, [2048, 7], [keep, 3], 0, min(1, keep), 1, 64, 32, F16, layers=1, seed=keep)


@pytest.mark.parametrize("bits", [16, 4])
def test_evict_ties_zeros_infinities_and_nan(bits):
    check_evict(bits, [400, 90], [100, 30], 2, 5, 2, 64, 16, F16, weights=lambda r: torch.zeros_like(r))
    check_evict(bits, [400, 90], [100, 30], 2, 5, 2, 64, 16, F16, weights=lambda r: (r * 4).floor())

    def odd(r):
        r = r - 0.3
        r[..., ::3], r[..., 1::7], r[..., 5::11], r[..., 2::13], r[..., 3::17] = -0.0, math.nan, math.inf, -math.inf, 1e-42
        return r
    for keep in (20, 100, 180, 350, 395):
        check_evict(bits, [400, 90], [keep, 30], 0, 0, 2, 64, 16, F16, weights=odd)


@pytest.mark.parametrize("bits", [16, 4])
def test_evict_long_rows_many_rows_and_layers(bits):
    check_evict(bits, [9000], [5000], 16, 100, 1, 64, 64, F16, layers=1)
    check_evict(bits, [20 + b for b in range(90)], [b % 33 for b in range(90)], 0, 0, 1, 16, 16, BF16, layers=5)


@pytest.mark.parametrize("bits", [16, 4])
def test_evict_skips_what_cannot_be_cut(bits):
    # more to stay than to keep; more tokens than weights; pages that others hold, from `first` on and before; page numbers outside the pool
    check_evict(bits, [100, 60], [10, 30], 6, 5, 2, 64, 16, F16)
    check_evict(bits, [100, 60], [10, 30], 0, 5, 2, 64, 16, F16, width=80)
    check_evict(bits, [100, 60, 80], [50, 30, 40], 32, 5, 2, 64, 16, F16, held=[(0, 3), (1, 0), (1, 1), (2, 2)])
    check_evict(bits, [100, 60], [50, 30], 0, 0, 2, 64, 16, F16, held=[(0, 6)])

    def change(t):
        t[0, 1], t[1, 3] = 1 << 20, -4
    check_evict(bits, [100, 60, 80], [50, 30, 40], 0, 5, 2, 64, 16, F16, table_change=change)


def test_evict_a_part_of_the_rows():
    """cache.rows() with a slice of the weights: the others' are not touched."""
    import paper_2501_16385_amd as fbq
    cache, table, values = any_cache(16, [90, 80, 70], 2, 64, 16, F16, layers=2)
    w = torch.rand(2, 3, 2, 96, generator=torch.Generator().manual_seed(1))
    want = evicted(values, table, cache.refs.cpu(), [90, 80, 70], w, [-1, 20, 30], 1, 2, 16)
    dev = w.cuda()
    fbq.cache_evict(cache.rows(1, 3), dev[:, 1:3], torch.tensor([20, 30], dtype=torch.int32, device="cuda"), first=1, recent=2)
    assert cache.lengths.tolist() == want[3] and torch.equal(cache.table.cpu(), want[1]) and torch.equal(dev.cpu(), want[4])
    assert torch.equal(torch.nan_to_num(cache.pool.cpu().double(), nan=-9.0), torch.nan_to_num(want[0], nan=-9.0))


@pytest.mark.parametrize("bits", [16, 4])
def test_a_captured_loop_under_a_budget(bits):
    """Reserve, append, attention, weights and eviction in one graph, replayed over steps, against the same calls one by one; rows never hold more than their budget."""
    import paper_2501_16385_amd as fbq
    D, rows, layers = 64, 3, 2
    sides = []
    g = torch.Generator().manual_seed(0)
    counts = [45, 20, 30]
    k0, v0 = (torch.randn(sum(counts), 2, D, generator=g).half().cuda() for _ in range(2))
    for _ in range(2):
        c = fbq.cache_create(layers, 30, 16, 2, D, rows, 8, bits=bits)
        c.pool.zero_()
        start = fbq.cache_reserve(c, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        for layer in range(layers):
            fbq.cache_append(c, layer, k0, v0, start, q_start=starts(counts).cuda())
        sides.append((c, torch.zeros(layers, rows, 2, 128, device="cuda")))
    one, keep = torch.ones(rows, dtype=torch.int32, device="cuda"), torch.tensor([40, -1, 31], dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros(rows, n, D, dtype=F16, device="cuda") for n in (8, 2, 2))
    start, info = torch.zeros_like(one), torch.zeros(2, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(rows, 8, device="cuda")
    ws, room = fbq.attention_workspace(sides[0][0], q), fbq.cache_evict_workspace(sides[0][0], sides[0][1])

    def step(c, w):
        fbq.cache_reserve(c, one, start=start)
        for layer in range(layers):
            fbq.cache_append(c, layer, k, v, start)
            fbq.attention(c, layer, q, out=out, lse=lse, workspace=ws)
            fbq.attention_weights(c, layer, q, lse, w[layer], decay=0.9)
        fbq.cache_evict(c, w, keep, first=2, recent=8, info=info, workspace=room)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(*sides[0])
    for i in range(12):
        g.manual_seed(i)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g).half())
        graph.replay()
        got = out.clone(), lse.clone(), info.tolist()
        step(*sides[1])
        assert torch.equal(got[0], out) and torch.equal(got[1], lse) and got[2] == info.tolist(), i
        for a, b in ((sides[0][0].table, sides[1][0].table), (sides[0][0].refs, sides[1][0].refs), (sides[0][1], sides[1][1]), (sides[0][0].pool, sides[1][0].pool)):
            assert torch.equal(a, b), i
    assert sides[0][0].lengths.tolist() == [40, 32, 31]
