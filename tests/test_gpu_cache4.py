"""A cache in 4 bits: append and read against the definition, every byte of the pool; the page operations on it."""
import math

import pytest
import torch

from cache4_cases import BF16, F16, make_cache4, pack, quantize, to_cache4, unpack
from cache_cases import make_cache, starts

pytestmark = pytest.mark.gpu


def appended(before, counts, kv_heads, D, page, dtype, seed=0, stride=0, start=None, change=None):
    """A call of cache_append against the pool that the definition makes of the old one and the new tokens; the pool, its cache and the new tokens."""
    import paper_2501_16385_amd as fbq
    g = torch.Generator().manual_seed(seed)
    after = [b + c for b, c in zip(before, counts)]
    x16, table, _, refs = make_cache(after, kv_heads, D, page, dtype, seed=seed, layers=2)
    T = sum(counts)
    k, v = ((torch.randn(T, kv_heads + stride, D, generator=g) * 1.7).to(dtype)[:, :kv_heads] for _ in range(2))
    if change is not None:
        change(k, v)
    old = x16.clone()                                          # nothing in the places that come
    new = x16.clone()
    at = 0
    for b, c in enumerate(counts):
        for i in range(c):
            pos = before[b] + i
            p, slot = int(table[b, pos // page]), pos % page
            old[:, p, :, :, slot] = float("nan")
            if start is None or start[b] >= 0:
                new[1, p, 0, :, slot], new[1, p, 1, :, slot] = k[at + i], v[at + i]
            else:
                new[1, p, :, :, slot] = float("nan")
        at += c
    new[0] = old[0]
    before4 = pack(old, page)
    want = pack(new, page, garbage=before4)
    cache = to_cache4(fbq, before4, table, torch.tensor(after, dtype=torch.int32), refs, dtype, D)
    first = torch.tensor(before if start is None else start, dtype=torch.int32).cuda()
    single = all(c == 1 for c in counts)
    fbq.cache_append(cache, 1, k.cuda() if not stride else torch.cat([k, k[:, :stride]], 1).cuda()[:, :kv_heads], v.cuda(), first, q_start=None if single else starts(counts).cuda())
    torch.cuda.synchronize()
    return cache, want, k, v, first


def check_append(*a, **how):
    cache, want, *_ = appended(*a, **how)
    got = cache.pool.cpu()
    assert torch.equal(got, want), f"{int((got != want).sum())} bytes of {got.numel()}"


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 40, 64, 72, 80, 96, 104, 128, 136, 192, 200, 256])
def test_append_every_head_size(D, dtype):
    check_append([5, 0, 16, 31], [1, 1, 1, 1], 3, D, 16, dtype, seed=D)
    check_append([5, 0, 14, 31], [40, 1, 3, 17], 2, D, 32, dtype, seed=D + 1)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("kv_heads,stride", [(1, 0), (4, 0), (5, 2), (9, 0)])
def test_append_heads_pages_and_rows_that_lie_apart(kv_heads, stride, page):
    check_append([0, 100, 37], [300, 2, 16], kv_heads, 64, page, F16, seed=page + kv_heads, stride=stride)


@pytest.mark.parametrize("offset", range(0, 18, 3))
@pytest.mark.parametrize("count", [1, 2, 3, 4, 5, 15, 16, 17, 33])
def test_append_where_tokens_begin_and_end_in_a_word(offset, count):
    check_append([offset, 2], [count, 1], 1, 64, 16, BF16, seed=offset)


def test_append_leaves_rows_without_pages_alone():
    check_append([5, 9, 3], [20, 4, 2], 2, 80, 16, F16, start=[5, -1, 3])


def test_append_of_special_numbers():
    """Constant groups, the type's least and largest numbers, ranges at its ends, ties, zeros of both signs."""
    def change(k, v):
        k[0], k[1, :, :64], v[2], v[3] = 0.0, 3.25, -0.0, 65504.0
        k[4, :, 0], k[4, :, 1] = -65504.0, 65504.0             # (m + 15 s beyond the type: the scale goes a step back)
        v[5] = torch.linspace(0, 7.5, 80).round(decimals=1).to(F16)                                     # many ties
        k[6] = torch.linspace(0, 15 * 2.0 ** -24, 80).to(F16)  # below the normal numbers
        v[7], v[7, :, 3] = 0.0, 2.0 ** -24
    check_append([0], [8], 2, 80, 16, F16, change=change)

    def change_b(k, v):
        k[0, :, 0], k[0, :, 1] = -3.0e38, 3.0e38
        k[1, :, 0] = -3.3895e38
        v[2] = 1e-39
        v[3], v[3, :, 5] = 0.0, 1e-40
    check_append([0], [8], 2, 80, 16, BF16, change=change_b)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_append_of_what_is_not_finite(dtype):
    """Such a token's head: its keys read as NaN, its values as 0; its other heads, and other tokens, as ever."""
    import paper_2501_16385_amd as fbq

    def change(k, v):
        k[2, 0, 5], v[4, 1, 70], k[6, 1, 0], v[7, 0, 3] = math.inf, -math.inf, math.nan, math.nan
    clean = appended([3], [9], 2, 80, 16, dtype)
    cache, _, _, _, first = appended([3], [9], 2, 80, 16, dtype, change=change)
    (k, v), (ck, cv) = (fbq.cache_read(c, 1, 9, f, q_start=starts([9]).cuda()) for c, f in ((cache, first), (clean[0], clean[4])))
    bad = torch.zeros(9, 2, dtype=torch.bool, device="cuda")
    bad[2, 0] = bad[4, 1] = bad[6, 1] = bad[7, 0] = True
    assert torch.isnan(k[bad]).all() and (v[bad] == 0).all()
    assert torch.equal(k[~bad], ck[~bad]) and torch.equal(v[~bad], cv[~bad])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 64, 80, 96, 128, 136, 256])
@pytest.mark.parametrize("bits", [4, 16])
def test_read(D, dtype, bits):
    import paper_2501_16385_amd as fbq
    lengths, page = [40, 7, 0, 33], 16
    if bits == 4:
        pool, table, n, refs, values = make_cache4(lengths, 3, D, page, dtype, layers=2, seed=D)
        cache = to_cache4(fbq, pool, table, n, refs, dtype, D)
    else:
        pool, table, n, refs = make_cache(lengths, 3, D, page, dtype, layers=2, seed=D)
        cache, values = fbq.Cache(pool.cuda(), table.cuda(), n.cuda(), refs.cuda()), pool.double()
    first, counts = [3, 0, 0, 30], [37, 7, 0, 3]
    start = torch.tensor([3, 0, -1, 30], dtype=torch.int32).cuda()
    k = torch.full((47, 3, D), 9.0, device="cuda")
    got = fbq.cache_read(cache, 1, 47, start, q_start=starts(counts).cuda(), k=k)
    assert got[0] is k
    t = 0
    for b, c in enumerate(counts):
        for i in range(c):
            p, slot = int(table[b, (first[b] + i) // page]), (first[b] + i) % page
            for x in (0, 1):
                assert torch.equal(got[x][t].cpu(), values[1, p, x, :, slot].float())
            t += 1
    start[1] = -1
    table_out = fbq.cache_read(cache, 0, 4, start, k=torch.full((4, 3, D), 8.0, device="cuda"), v=torch.full((4, 3, D), 8.0, device="cuda"))
    assert all((x[1] == 8).all() and (x[2] == 8).all() and torch.equal(x[3].cpu(), values[0, int(table[3, 1]), i, :, 14].float()) for i, x in enumerate(table_out))


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("counts", [[300, 0, 1, 83], [128], [127], [40, 216, 5]])
def test_read_of_many_tokens(counts, bits):
    """A hundred and more in one call are what calls of one token a row give."""
    import paper_2501_16385_amd as fbq
    before = [7 + b for b in range(len(counts))]
    pool, table, n, refs, _ = make_cache4([b + c for b, c in zip(before, counts)], 2, 72, 16, F16, seed=sum(counts))
    cache = to_cache4(fbq, pool, table, n, refs, F16, 72)
    if bits == 16:
        x, table, n, refs = make_cache([b + c for b, c in zip(before, counts)], 2, 72, 16, F16, seed=sum(counts))
        cache = fbq.Cache(x.cuda(), table.cuda(), n.cuda(), refs.cuda())
    start = torch.tensor(before, dtype=torch.int32).cuda()
    k, v = fbq.cache_read(cache, 0, sum(counts), start, q_start=starts(counts).cuda())
    at = 0
    for b, c in enumerate(counts):
        for i in range(c):
            ones = torch.full((len(counts),), -1, dtype=torch.int32)
            ones[b] = before[b] + i
            k1, v1 = fbq.cache_read(cache, 0, len(counts), ones.cuda())
            assert torch.equal(k1[b], k[at]) and torch.equal(v1[b], v[at]), (b, i)
            at += 1


def test_read_follows_no_page_outside_the_pool():
    import paper_2501_16385_amd as fbq
    pool, table, n, refs, _ = make_cache4([40, 20], 2, 64, 16, F16)
    table[0, 1], table[1, 0] = 1 << 20, -5
    cache = to_cache4(fbq, pool, table, n, refs, F16, 64)
    k, v = (torch.full((2, 2, 64), 8.0, device="cuda") for _ in range(2))
    fbq.cache_read(cache, 0, 2, torch.tensor([17, 3], dtype=torch.int32).cuda(), k=k, v=v)
    fbq.cache_read(cache, 0, 2, torch.tensor([1 << 30, 2147483647], dtype=torch.int32).cuda(), k=k, v=v)
    before = cache.pool.clone()
    fbq.cache_append(cache, 0, k.half(), v.half(), torch.tensor([17, 3], dtype=torch.int32).cuda())
    fbq.cache_append(cache, 0, k.half(), v.half(), torch.tensor([1 << 30, 2147483647], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert (k == 8).all() and (v == 8).all() and torch.equal(before, cache.pool)


@pytest.mark.parametrize("D,page", [(64, 16), (80, 32), (128, 64)])
def test_page_operations(D, page):
    """Reserve, append, fork, copy and compact of a cache in 4 bits: what the rows read back."""
    import paper_2501_16385_amd as fbq
    cache = fbq.cache_create(2, 40, page, 2, D, 6, 5, bits=4)
    cache.pool.fill_(0xFF)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    count = [3 * page + 5, 0, page, 0, 1, 0]
    g = torch.Generator().manual_seed(D)
    held = {b: [torch.randn(2, c, 2, D, generator=g).half() for _ in range(2)] for b, c in enumerate(count) if c}
    start = fbq.cache_reserve(cache, ints(*count))
    for layer in range(2):
        k, v = (torch.cat([held[b][x][layer] for b in held]).cuda() for x in (0, 1))
        fbq.cache_append(cache, layer, k, v, start, q_start=starts(count).cuda())

    def check(rows):
        for b, of in rows.items():
            n = count[of]
            assert int(cache.lengths[b]) == n
            edges = ints(*[0] * (b + 1), *[n] * (6 - b))
            for layer in range(2):
                got = fbq.cache_read(cache, layer, n, ints(*[0] * 6), q_start=edges)
                for x in (0, 1):
                    c, s, m = quantize(held[of][x][layer])
                    y = torch.arange(D) // 64
                    want = m.double()[..., y] + s.double()[..., y] * c.double()
                    assert torch.equal(got[x].cpu(), want.float())
    check({0: 0, 2: 2, 4: 4})
    fbq.cache_fork(cache, ints(0, 4, 0), ints(1, 3, 5))
    check({0: 0, 1: 0, 2: 2, 3: 4, 4: 4, 5: 0})
    fbq.cache_free(cache, ints(0, 4))
    info = ints(0, 0)
    fbq.cache_compact(cache, info=info)
    check({1: 0, 2: 2, 3: 4, 5: 0})
    assert info.tolist()[0] == 3 + 2 + 1 + 1
    a, b = int(cache.table[2, 0]), int(info[0]) + 3
    fbq.cache_copy(cache, ints(a), ints(b))
    assert torch.equal(cache.pool[:, a], cache.pool[:, b])


def test_append_of_equal_calls_is_equal_and_captured_ones_are():
    import paper_2501_16385_amd as fbq
    cache, want, k, v, first = appended([5, 30], [1, 1], 4, 128, 16, F16)
    k, v = k.cuda(), v.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fbq.cache_append(cache, 1, k, v, first)
        read = fbq.cache_read(cache, 1, 2, first)
    for i in range(3):
        k.copy_(torch.randn(k.shape, generator=torch.Generator().manual_seed(i)).half())
        graph.replay()
        torch.cuda.synchronize()
        c, s, m = quantize(k.cpu())
        y = torch.arange(128) // 64
        assert torch.equal(read[0].cpu(), (m.double()[..., y] + s.double()[..., y] * c.double()).float())
