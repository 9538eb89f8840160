"""Attention over a cache in 4 bits against the formula in 64 bits over what its codes stand for (tests/cache4_cases.py), element by element within derived bounds; every place of
the pool without a token holds scales that are NaN."""
import math

import pytest
import torch

from cache4_cases import BF16, F16, attention4_64, make_cache4, pack, to_cache4
from cache_cases import starts

pytestmark = pytest.mark.gpu


def check(lengths, counts, heads, kv_heads, D, page, dtype, shared_pages=0, fused=0, seed=0, scale=None, layers=1, layer=0, gain=2.0, token_form=None, width=None):
    """One call against the formula; token_form: whether q_start is left out (default: where every row has one token)."""
    import paper_2501_16385_amd as fbq
    pool, table, n, refs, values = make_cache4(lengths, kv_heads, D, page, dtype, shared_pages=shared_pages, layers=layers, seed=seed, width=width)
    T = sum(counts)
    g = torch.Generator().manual_seed(seed + 1)
    wide = (torch.randn(T, heads + fused, D, generator=g) * gain).to(dtype)
    scale = D ** -0.5 if scale is None else scale
    few = max(counts) * heads // kv_heads <= 16 and not shared_pages
    want, want_lse, bound, lse_bound = attention4_64(values, table, n, layer, wide[:, :heads], counts, scale, few)
    cache = to_cache4(fbq, pool, table, n, refs, dtype, D)
    q = wide.cuda()[:, :heads]
    lse = torch.full((T, heads), 77.0, device="cuda")
    out = torch.full((T, heads, D), 55.0, dtype=dtype, device="cuda")
    single = all(c == 1 for c in counts) if token_form is None else token_form
    shared = table[0, :shared_pages].contiguous().cuda() if shared_pages else None
    workspace = fbq.attention_workspace(cache, q, max_q=max(counts), shared=shared, q_start=None if single else starts(counts).cuda())
    workspace.fill_(0xFF)                                      # NaN wherever something is read that was not written
    go = lambda: fbq.attention(cache, layer, q, q_start=None if single else starts(counts).cuda(), max_q=max(counts), shared=shared, scale=scale, out=out, lse=lse, workspace=workspace)
    got = go()
    torch.cuda.synchronize()
    first = got.clone()
    got, lse_ = got.cpu().double(), lse.cpu().double()
    assert torch.isfinite(got).all()
    off = (got - want).abs()
    assert (off <= bound).all(), f"{(off / bound).max():.2f} times the bound, at {int((off / bound).argmax())} of {off.numel()}"
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse_), empty) and (lse_[empty] < 0).all()
    assert (got[empty] == 0).all()
    assert ((lse_ - want_lse)[~empty].abs() <= lse_bound[~empty]).all()
    assert torch.equal(go(), first)                            # equal calls, equal bits
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 40, 64, 72, 80, 96, 128, 136, 192, 200, 256])
def test_single_tokens_every_head_size(D, dtype):
    check([1, 33, 0, 15, 16, 17, 200], [1] * 7, 4, 2, D, 16, dtype, seed=D)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (8, 1), (16, 2), (15, 3), (16, 1)])
def test_single_tokens_head_layouts_and_pages(heads, kv_heads, page):
    check([300, 1, 64, 257, 31], [1] * 5, heads, kv_heads, 64, page, F16, seed=page + heads)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("lengths", [[1], [2], [31], [32], [33], [63, 64, 65], [0], [0, 5, 0], [1000, 0, 3], [2049], [1] * 70 + [500] + [0] * 70 + [40] * 3])
def test_single_tokens_lengths(lengths, dtype):
    check(lengths, [1] * len(lengths), 4, 2, 128, 16, dtype, seed=len(lengths))


@pytest.mark.parametrize("D", [64, 96, 256])
def test_single_tokens_one_long_row_among_short_ones(D):
    check([7, 20000, 100], [1] * 3, 2, 1, D, 32, BF16, seed=3)


@pytest.mark.parametrize("lengths", [[9000, 4000, 1, 12345], [0, 16000, 31, 16001, 64], [2500] * 20, [40 * b for b in range(60)]])
@pytest.mark.parametrize("heads,kv_heads,shared_pages", [(8, 8, 0), (3, 1, 0), (8, 8, 2)])
def test_single_tokens_more_steps_than_waves(lengths, heads, kv_heads, shared_pages):
    if shared_pages:
        lengths = [max(n, 32) for n in lengths]
    check(lengths, [1] * len(lengths), heads, kv_heads, 16, 16, F16, shared_pages=shared_pages, seed=sum(lengths) % 1000)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,kv_heads,max_count", [(4, 4, 5), (8, 4, 8), (8, 2, 4), (6, 2, 9), (32, 1, 3), (40, 1, 7), (3, 1, 100)])
def test_several_tokens_a_row(heads, kv_heads, max_count, dtype):
    lengths, counts = [120, 40, 9, 333], [max_count, 1, min(3, max_count), max(1, max_count - 1)]
    lengths = [max(n, c) for n, c in zip(lengths, counts)]
    check(lengths, counts, heads, kv_heads, 64, 16, dtype, seed=heads)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 64, 80, 96, 128, 136, 192, 200, 256])
def test_prompts(D, dtype):
    check([150, 64, 1, 129], [150, 30, 1, 129], 4, 2, D, 16, dtype, seed=D)


@pytest.mark.parametrize("count", [1, 2, 127, 128, 129, 300])
def test_prompt_lengths(count):
    check([count], [count], 2, 2, 128, 32, F16, seed=count, token_form=False)
    check([count + 77], [count], 4, 1, 64, 16, BF16, seed=count, token_form=False)


def test_a_long_prompt_cut_into_pieces():
    check([1100], [70], 2, 2, 128, 64, BF16, seed=1)
    check([5000, 90], [20, 30], 4, 2, 96, 16, F16, seed=2)


def test_rows_without_query_tokens_and_tokens_that_see_nothing():
    # row 0 has more new tokens than it holds: its first ones see nothing; rows 1 and 3 have none; row 4 holds nothing
    check([3, 50, 70, 20, 0], [5, 0, 2, 0, 4], 4, 4, 64, 16, F16, seed=1)
    check([30, 50, 70, 20, 0], [45, 0, 40, 0, 33], 4, 4, 64, 16, F16, seed=2)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,heads,kv_heads,own", [(4, 4, 4, 20), (24, 16, 2, 40), (3, 64, 2, 5)])
def test_shared_tokens(rows, heads, kv_heads, own, dtype):
    """Behind a prefix that is read apart (its bytes are enough) and one that is not."""
    for shared, D in ((4096, 128), (64, 64)):
        check([shared + own + b for b in range(rows)], [1] * rows, heads, kv_heads, D, 32, dtype, shared_pages=shared // 32, seed=rows)


def test_shared_tokens_are_read_apart_in_both_kernels():
    """Twelve rows of few queries behind 8192 tokens: 2 MiB and more of the 16-bit rule's bytes are saved."""
    check([8192 + 3 * b for b in range(12)], [1] * 12, 8, 8, 64, 64, F16, shared_pages=128, seed=5)
    check([8192 + 3 * b for b in range(40)], [1] * 40, 8, 4, 128, 64, BF16, shared_pages=128, seed=6)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,kv_heads,rows,count", [(64, 8, 18, 1), (80, 4, 30, 1), (128, 4, 18, 1), (192, 2, 24, 1), (64, 4, 34, 20), (136, 4, 18, 17)])
def test_shared_tokens_of_the_many_row_kernel(D, kv_heads, rows, count, dtype):
    """17 query rows and more of a head behind 8192 tokens, 256 MiB and more of the 16-bit rule's bytes: a launch with the rows' own tokens, or one of their own (192 features; 17 tokens and more)."""
    assert 4 * 8192 * kv_heads * D * (rows - 1) >= 256 << 20
    check([8192 + count + 7 * b for b in range(rows)], [count] + [1 + b % count for b in range(rows - 1)], kv_heads, kv_heads, D, 64, dtype, shared_pages=128, seed=D)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-8, 3.0])
def test_scales(scale):
    check([90, 40], [1, 1], 4, 2, 64, 16, F16, seed=1, scale=scale, gain=1.0)
    check([90, 40], [20, 30], 4, 2, 64, 16, BF16, seed=1, scale=scale, gain=1.0)


def test_strided_queries_layers_and_large_ones():
    check([100, 30], [1, 1], 4, 2, 80, 16, F16, fused=4, layers=3, layer=2, seed=4)
    check([100, 130], [50, 70], 4, 2, 80, 16, BF16, fused=4, layers=3, layer=1, seed=4)
    check([100, 300], [1, 1], 4, 2, 128, 16, BF16, gain=40.0, seed=5)


@pytest.mark.parametrize("dtype,size", [(F16, 3000.0), (F16, 1e-4), (BF16, 1e20), (BF16, 1e-20)])
@pytest.mark.parametrize("counts", [[1, 1], [60, 30]])
def test_values_of_any_size(dtype, size, counts):
    """Scales from near the type's largest to near its least, and one row in which they grow and shrink by a thousand from token to token."""
    import paper_2501_16385_amd as fbq
    from cache_cases import make_cache
    D, page = 64, 16
    x, table, n, refs = make_cache([200, 77], 2, D, page, dtype, seed=3)
    x[:, :, 1] = (x[:, :, 1].double() * size).to(dtype)
    x[0, table[1, 0].long(), 1, :, ::2] = (x[0, table[1, 0].long(), 1, :, ::2].double() / 1000).to(dtype)
    pool = pack(x, page)
    from cache4_cases import unpack
    values = unpack(pool, dtype, D)
    T = sum(counts)
    q = torch.randn(T, 4, D, generator=torch.Generator().manual_seed(9)).to(dtype)
    want, _, bound, _ = attention4_64(values, table, n, 0, q, counts, D ** -0.5, max(counts) == 1)
    cache = to_cache4(fbq, pool, table, n, refs, dtype, D)
    got = fbq.attention(cache, 0, q.cuda(), q_start=starts(counts).cuda(), max_q=max(counts)).cpu().double()
    # (bf16 at 1e-20: the bound's 2^-24 for results below fp16's normal numbers is nothing here)
    bound = bound - 2.0 ** -24 + (2.0 ** -24 if dtype == F16 else 1e-38)
    assert ((got - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("counts", [[4, 1], [40, 30]])
def test_what_a_token_does_not_see_does_not_reach_it(counts, dtype):
    """A NaN among the newest token's keys, or its values: that token's result is NaN in the head's queries, those before it are as without."""
    import paper_2501_16385_amd as fbq
    D, page, lengths = 128, 16, [90, 64]
    pool, table, n, refs, _ = make_cache4(lengths, 2, D, page, dtype, seed=2)
    q = torch.randn(sum(counts), 4, D, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    kv = torch.randn(2, counts[0], 2, D, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    results = []
    for which in (None, 0, 1):
        cache = to_cache4(fbq, pool, table, n, refs, dtype, D)
        new = kv.clone()
        if which is not None:
            new[which, -1, 1, 7] = math.nan if which else math.inf
        start = torch.tensor([lengths[0] - counts[0], -1], dtype=torch.int32, device="cuda")
        fbq.cache_append(cache, 0, new[0], new[1], start, q_start=torch.tensor([0, counts[0], counts[0]], dtype=torch.int32, device="cuda"))
        lse = torch.empty(sum(counts), 4, device="cuda")
        results.append((fbq.attention(cache, 0, q, q_start=starts(counts).cuda(), max_q=max(counts), lse=lse), lse))
    last = counts[0] - 1
    for out, lse in results[1:]:
        assert torch.isnan(out[last, 2:]).all() and torch.isnan(lse[last, 2:]).all()
        keep = torch.ones(sum(counts), 4, dtype=torch.bool, device="cuda")
        keep[last, 2:] = False
        assert torch.equal(out[keep], results[0][0][keep]) and torch.equal(lse[keep], results[0][1][keep])


@pytest.mark.parametrize("counts", [[1, 1], [30, 20]])
def test_page_numbers_outside_the_pool_read_zeros(counts):
    import paper_2501_16385_amd as fbq
    D, page = 64, 16
    pool, table, n, refs, values = make_cache4([100, 50], 2, D, page, F16, seed=2)
    gone = [int(table[0, 2]), int(table[1, 0])]
    wild = table.clone()
    wild[0, 2], wild[1, 0] = pool.shape[1], -7
    values[:, gone] = 0
    q = torch.randn(sum(counts), 4, D, generator=torch.Generator().manual_seed(1)).half()
    want, _, bound, _ = attention4_64(values, table, n, 0, q, counts, 0.125, max(counts) == 1)
    cache = to_cache4(fbq, pool, wild, n, refs, F16, D)
    got = fbq.attention(cache, 0, q.cuda(), q_start=starts(counts).cuda(), max_q=max(counts), scale=0.125).cpu().double()
    assert ((got - want).abs() <= bound).all()


def test_a_captured_call_follows_lengths_and_tables():
    """The graph of reserve, append and attention, replayed over steps, against the same steps called one by one."""
    import paper_2501_16385_amd as fbq
    D, rows = 128, 3
    caches = [fbq.cache_create(1, 30, 16, 2, D, rows, 8, bits=4) for _ in range(2)]
    g = torch.Generator().manual_seed(0)
    k0, v0 = (torch.randn(40, 2, D, generator=g).half().cuda() for _ in range(2))
    counts = [25, 1, 14]
    for c in caches:
        c.pool.fill_(0xFF)
        start = fbq.cache_reserve(c, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        fbq.cache_append(c, 0, k0, v0, start, q_start=starts(counts).cuda())
    one = torch.ones(rows, dtype=torch.int32, device="cuda")
    q, k, v = torch.zeros(rows, 8, D, dtype=F16, device="cuda"), torch.zeros(rows, 2, D, dtype=F16, device="cuda"), torch.zeros(rows, 2, D, dtype=F16, device="cuda")
    start, out = torch.zeros_like(one), torch.zeros_like(q)
    ws = fbq.attention_workspace(caches[0], q)

    def step(c):
        fbq.cache_reserve(c, one, start=start)
        fbq.cache_append(c, 0, k, v, start)
        return fbq.attention(c, 0, q, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(caches[0])
    for i in range(20):
        g.manual_seed(i)
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g).half())
        graph.replay()
        got = out.clone()
        assert torch.equal(got, step(caches[1])), i
    assert caches[0].lengths.tolist() == caches[1].lengths.tolist() == [45, 21, 34]


@pytest.mark.parametrize("k_size,v_size", [(1e-6, 1.0), (1.0, 1e-6), (1e5, 1.0), (1.0, 1e5), (1e-30, 1e30)])
def test_prompts_over_scales_that_fp16_operands_are_not_made_for(k_size, v_size):
    """bf16: a part of the rows has such keys or values, another has ordinary ones; constant groups and zeros among them."""
    import paper_2501_16385_amd as fbq
    from cache4_cases import unpack
    from cache_cases import make_cache
    D, page, counts = 128, 16, [60, 30, 50]
    x, table, n, refs = make_cache([200, 77, 130], 2, D, page, BF16, seed=3)
    for i, size in ((0, k_size), (1, v_size)):
        x[0, table[0].long().clamp(min=0)[:13], i] = (x[0, table[0].long().clamp(min=0)[:13], i].double() * size).to(BF16)
        x[0, table[2, :4].long(), i, :, :8] = 0.0 if size < 1 else 3.0
    pool = pack(x, page)
    values = unpack(pool, BF16, D)
    q = torch.randn(sum(counts), 4, D, generator=torch.Generator().manual_seed(9)).to(BF16)
    q[:60] = (q[:60].double() / k_size).to(BF16)
    want, _, bound, _ = attention4_64(values, table, n, 0, q, counts, D ** -0.5, False)
    bound = bound - 2.0 ** -24 + 2.0 ** -24 * min(1.0, v_size)
    cache = to_cache4(fbq, pool, table, n, refs, BF16, D)
    got = fbq.attention(cache, 0, q.cuda(), q_start=starts(counts).cuda(), max_q=max(counts)).cpu().double()
    assert ((got - want).abs() <= bound).all()


@pytest.mark.parametrize("D,kv_heads,rows", [(64, 8, 18), (80, 4, 30), (128, 4, 18)])
@pytest.mark.parametrize("which,size", [(0, 1e-6), (1, 1e5), (1, 1e-20)])
def test_shared_tokens_over_scales_that_fp16_operands_are_not_made_for(which, size, D, kv_heads, rows):
    """bf16: pages of the shared tokens have such keys or values, the others ordinary ones; the rows' own tokens are in the same launch."""
    import paper_2501_16385_amd as fbq
    from cache4_cases import unpack
    from cache_cases import make_cache
    lengths = [8192 + 1 + 7 * b for b in range(rows)]
    x, table, n, refs = make_cache(lengths, kv_heads, D, 64, BF16, shared_pages=128, seed=D)
    for page in (3, 70, 127):
        at = int(table[0, page])
        x[0, at, which] = (x[0, at, which].double() * size).to(BF16)
    pool = pack(x, 64)
    values, counts = unpack(pool, BF16, D), [1] * rows
    q = torch.randn(rows, kv_heads, D, generator=torch.Generator().manual_seed(9)).to(BF16)
    want, _, bound, _ = attention4_64(values, table, n, 0, q, counts, D ** -0.5, False)
    cache = to_cache4(fbq, pool, table, n, refs, BF16, D)
    got = fbq.attention(cache, 0, q.cuda(), shared=table[0, :128].contiguous().cuda()).cpu().double()
    assert ((got - want).abs() <= bound).all()
