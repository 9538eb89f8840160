"""Attention over the paged cache against the formula in 64 bits (tests/cache_cases.py), element by element within a bound that is derived from the
roundings the kernels make; every place of the pool without a token holds NaN."""
import math

import pytest
import torch

from cache_cases import attention64, make_cache, starts, to_cache

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def check(lengths, counts, heads, kv_heads, D, page, dtype, shared_pages=0, fused=0, seed=0, scale=None, layers=1, layer=0, gain=2.0, token_form=None, width=None):
    """One call against the formula; token_form: whether q_start is left out (default: where every row has one token)."""
    import paper_2501_16385_amd as fbq
    pool, table, n, refs = make_cache(lengths, kv_heads, D, page, dtype, shared_pages, layers, seed=seed, width=width)
    T = sum(counts)
    g = torch.Generator().manual_seed(seed + 1)
    wide = (torch.randn(T, heads + fused, D, generator=g) * gain).to(dtype)
    scale = D ** -0.5 if scale is None else scale
    want, want_lse, bound, lse_bound = attention64(pool, table, n, layer, wide[:, :heads], counts, scale)
    cache = to_cache(fbq, pool, table, n, refs)
    q = wide.cuda()[:, :heads]
    lse = torch.full((T, heads), 77.0, device="cuda")
    out = torch.full((T, heads, D), 55.0, dtype=dtype, device="cuda")
    single = all(c == 1 for c in counts) if token_form is None else token_form
    shared = table[0, :shared_pages].contiguous().cuda() if shared_pages else None
    workspace = fbq.attention_workspace(cache, q, max_q=max(counts), shared=shared, q_start=None if single else starts(counts).cuda())
    workspace.fill_(0xFF)                                      # NaN wherever something is read that was not written
    got = fbq.attention(cache, layer, q, q_start=None if single else starts(counts).cuda(), max_q=max(counts), shared=shared, scale=scale, out=out, lse=lse,
                        workspace=workspace)
    torch.cuda.synchronize()
    got, lse = got.cpu().double(), lse.cpu().double()
    assert torch.isfinite(got).all()
    off = (got - want).abs()
    assert (off <= bound).all(), f"{(off / bound).max():.2f} times the bound, at {int((off / bound).argmax())} of {off.numel()}"
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), empty) and (lse[empty] < 0).all()
    assert (got[empty] == 0).all()
    assert ((lse - want_lse)[~empty].abs() <= lse_bound[~empty]).all()
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 40, 64, 72, 80, 96, 128, 136, 192, 256])
def test_single_tokens_every_head_size(D, dtype):
    check([1, 33, 0, 15, 16, 17, 200], [1] * 7, 4, 2, D, 16, dtype, seed=D)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (8, 1), (16, 2), (15, 3), (16, 1)])
def test_single_tokens_head_layouts_and_pages(heads, kv_heads, page):
    check([300, 1, 64, 257, 31], [1] * 5, heads, kv_heads, 64, page, F16, seed=page + heads)


@pytest.mark.parametrize("lengths", [[1], [2], [31], [32], [33], [63, 64, 65], [0], [0, 0, 0], [0, 5, 0], [1000, 0, 3], [2049], [1] * 70 + [500] + [0] * 70 + [40] * 3])
def test_single_tokens_lengths(lengths):
    check(lengths, [1] * len(lengths), 4, 2, 128, 16, F16, seed=len(lengths))


def test_single_tokens_one_long_row_among_short_ones():
    check([7, 20000, 100], [1] * 3, 2, 1, 64, 32, BF16, seed=3)


@pytest.mark.parametrize("lengths", [[9000, 4000, 1, 12345], [33000], [0, 16000, 31, 16001, 64], [2500] * 20, [40 * b for b in range(60)]])
@pytest.mark.parametrize("heads,kv_heads,shared_pages", [(8, 8, 0), (16, 4, 0), (3, 1, 0), (8, 8, 2)])
def test_single_tokens_more_steps_than_waves(lengths, heads, kv_heads, shared_pages):
    """Rows long and many enough that a wave has several steps: pieces that begin and end anywhere, whole blocks of them in one row, rows within one piece."""
    if shared_pages:
        lengths = [max(n, 32) for n in lengths]
    check(lengths, [1] * len(lengths), heads, kv_heads, 16, 16, F16, shared_pages=shared_pages, seed=sum(lengths) % 1000)


@pytest.mark.parametrize("counts", [None, 3])
def test_an_item_a_wave(counts):
    """Many short rows: a wave has a row's head to itself."""
    lengths = [(7 * b) % 200 for b in range(300)]
    c = [1] * 300 if counts is None else [b % counts for b in range(300)]
    lengths = [max(n, k) for n, k in zip(lengths, c)]
    check(lengths, c, 4, 4, 16, 16, F16, seed=8, width=16)


def test_more_pages_than_a_register_holds():
    """A wave that goes through more than 64 pages: in the few-row kernel's line, and along the keys of a tile."""
    check([66000], [1], 32, 32, 16, 16, F16, seed=3)
    check([12000], [300], 32, 32, 16, 16, BF16, seed=4)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("heads,kv_heads,max_count", [(4, 4, 5), (8, 4, 8), (8, 2, 4), (6, 2, 9), (32, 1, 3), (40, 1, 7), (3, 1, 100)])
def test_several_tokens_a_row(heads, kv_heads, max_count, dtype):
    lengths, counts = [120, 40, 9, 333], [max_count, 1, min(3, max_count), max(1, max_count - 1)]
    lengths = [max(n, c) for n, c in zip(lengths, counts)]
    check(lengths, counts, heads, kv_heads, 64, 16, dtype, seed=heads)


@pytest.mark.parametrize("rows,heads,kv_heads", [(80, 136, 8), (70, 1050, 5), (64, 136, 8), (66, 17, 1)])
def test_single_tokens_of_wide_groups(rows, heads, kv_heads):
    """More heads a key/value head than the few-row kernel has rows: one tile a row and more, for so many rows that none is cut, and for fewer."""
    check([(13 * b) % 90 for b in range(rows)], [1] * rows, heads, kv_heads, 16, 16, F16, seed=rows)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [16, 64, 80, 128, 200, 256])
def test_prompts(D, dtype):
    check([150, 64, 1, 129], [150, 30, 1, 129], 4, 2, D, 16, dtype, seed=D)


@pytest.mark.parametrize("count", [1, 2, 127, 128, 129, 300])
def test_prompt_lengths(count):
    check([count], [count], 2, 2, 128, 32, F16, seed=count, token_form=False)
    check([count + 77], [count], 4, 1, 64, 16, BF16, seed=count, token_form=False)


def test_rows_without_query_tokens_and_tokens_that_see_nothing():
    # row 0 has more new tokens than it holds: its first ones see nothing; rows 1 and 3 have none; row 4 holds nothing
    check([3, 50, 70, 20, 0], [5, 0, 2, 0, 4], 4, 4, 64, 16, F16, seed=1)
    check([30, 50, 70, 20, 0], [45, 0, 40, 0, 33], 4, 4, 64, 16, F16, seed=2)
    check([3, 40], [20, 40], 8, 1, 128, 32, BF16, seed=3)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,heads,kv_heads", [(2, 4, 4), (8, 2, 2), (9, 4, 2), (16, 4, 4), (40, 8, 2), (150, 2, 2)])
@pytest.mark.parametrize("page,pages", [(16, 1), (16, 9), (64, 5)])
def test_shared_prefix(rows, heads, kv_heads, page, pages, dtype):
    lengths = [page * pages + (37 * b) % 90 for b in range(rows)]      # some rows end with the prefix
    check(lengths, [1] * rows, heads, kv_heads, 64, page, dtype, shared_pages=pages, seed=rows)


@pytest.mark.parametrize("counts", [[4, 4, 4], [1, 2, 3], [20, 1, 17], [70, 3, 5]])
def test_shared_prefix_and_several_tokens(counts):
    lengths = [96 + 10, 96 + 33, 96 + 70]
    lengths = [max(n, 96 + c) for n, c in zip(lengths, counts)]
    check(lengths, counts, 4, 2, 128, 16, F16, shared_pages=6, seed=sum(counts))


def taken_apart(rows, tokens, kv_heads, heads, D, page, pages, max_count, dtype):
    """Whether a call with these sizes reads the shared tokens apart: then its workspace is another."""
    import paper_2501_16385_amd as fbq
    cache = fbq.cache_create(1, pages + 1, page, kv_heads, D, rows, -(-tokens // page), dtype)
    T = rows * max_count
    q, starts_ = torch.empty(T, heads, D, dtype=dtype, device="cuda"), torch.empty(rows + 1, dtype=torch.int32, device="cuda") if max_count > 1 else None
    size = lambda shared: fbq.attention_workspace(cache, q, q_start=starts_, max_q=max_count, shared=shared).numel()
    return size(torch.empty(pages, dtype=torch.int32, device="cuda")) != size(None)


# (rows, heads, kv_heads, D, page, shared pages): what is shared is long enough to be read apart
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,heads,kv_heads,D,page,pages", [
    (2, 4, 4, 64, 16, 200), (5, 3, 1, 128, 64, 70), (16, 2, 2, 40, 16, 150), (3, 4, 1, 256, 32, 90),          # in the few-row kernel's line
    (20, 4, 4, 64, 16, 130), (17, 8, 1, 64, 32, 100), (40, 4, 2, 80, 16, 140), (33, 4, 4, 128, 16, 90), (150, 2, 1, 128, 128, 12), (24, 16, 1, 96, 64, 40),   # beside it
    (20, 4, 2, 256, 16, 80), (18, 2, 2, 200, 64, 30)])                                                        # in front of it
def test_shared_tokens_read_apart(rows, heads, kv_heads, D, page, pages, dtype):
    lengths = [page * pages + (37 * b) % 90 for b in range(rows)]
    lengths[1] = page * pages // 2 + 3                          # a row that ends inside the shared pages
    if rows > 4:
        lengths[rows - 2] = 0
    assert taken_apart(rows, max(lengths), kv_heads, heads, D, page, pages, 1, dtype)
    check(lengths, [1] * rows, heads, kv_heads, D, page, dtype, shared_pages=pages, seed=rows)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,heads,kv_heads,D,page,pages,most", [
    (9, 2, 2, 64, 16, 300, 3), (4, 4, 1, 128, 32, 100, 4),                                                   # few rows
    (12, 4, 2, 64, 16, 500, 12), (10, 8, 1, 128, 64, 130, 4), (20, 2, 2, 80, 16, 600, 50), (8, 4, 4, 256, 32, 100, 30)])   # many rows, twice
def test_shared_tokens_read_apart_for_several_tokens_a_row(rows, heads, kv_heads, D, page, pages, most, dtype):
    counts = [1 + (5 * b) % most for b in range(rows)]
    counts[0], counts[2] = most, 0
    lengths = [page * pages + c + (11 * b) % 60 for b, c in enumerate(counts)]
    lengths[3] = page * pages - 5                              # its new tokens end inside the shared pages
    assert taken_apart(rows, max(lengths), kv_heads, heads, D, page, pages, most, dtype)
    check(lengths, counts, heads, kv_heads, D, page, dtype, shared_pages=pages, seed=rows, token_form=False)


def test_shared_prefix_longer_than_a_row():
    # rows that hold less than the shared pages see only what they hold, an empty one nothing
    check([70, 0, 13, 64, 200], [1] * 5, 4, 2, 64, 16, F16, shared_pages=4, seed=5, width=13)
    check([70, 0, 13, 64, 200] * 5, [1] * 25, 4, 2, 64, 16, F16, shared_pages=4, seed=6, width=13)
    check([70, 0, 13, 64, 200], [3, 2, 20, 1, 4], 4, 2, 64, 16, BF16, shared_pages=4, seed=7, width=13)


def test_queries_of_a_fused_projection_and_other_layers():
    check([100, 33], [1, 1], 8, 2, 128, 16, F16, fused=4, seed=1, layers=3, layer=2)
    check([100, 133], [60, 133], 8, 2, 64, 16, BF16, fused=4, seed=2, layers=3, layer=1)


@pytest.mark.parametrize("gain", [0.0, 40.0])
def test_flat_and_sharp_softmax(gain):
    check([500, 70], [1, 1], 4, 4, 64, 16, F16, gain=gain, seed=1)
    check([200, 70], [100, 70], 4, 4, 64, 16, F16, gain=gain, seed=2)


def test_nan_and_infinity_where_a_row_sees_them():
    """A NaN among the keys a row sees shows in its result, as the formula has it, and in no other row's."""
    import paper_2501_16385_amd as fbq
    pool, table, n, refs = make_cache([40, 40], 1, 64, 16, F16, seed=9)
    pool[0, table[1, 1], 0, 0, 3] = float("nan")
    cache = to_cache(fbq, pool, table, n, refs)
    q = torch.randn(2, 1, 64).half().cuda()
    out = fbq.attention(cache, 0, q).cpu()
    assert torch.isfinite(out[0]).all() and torch.isnan(out[1]).all()


def test_a_page_number_outside_the_pool_is_not_followed():
    """Zeros stand in for its tokens: no access outside the pool, finite results."""
    import paper_2501_16385_amd as fbq
    pool, table, n, refs = make_cache([40, 100], 2, 64, 16, F16, seed=9)
    table[1, 2], table[1, 4] = 1 << 30, -5
    cache = to_cache(fbq, pool, table, n, refs)
    one = fbq.attention(cache, 0, torch.randn(2, 2, 64).half().cuda())
    many = fbq.attention(cache, 0, torch.randn(60, 2, 64).half().cuda(), q_start=starts([20, 40]).cuda(), max_q=40)
    assert torch.isfinite(one).all() and torch.isfinite(many).all()
    n[0], n[1] = 1 << 30, -7                                   # lengths: at most the table's width, at least 0
    pool.zero_()
    cache = to_cache(fbq, pool, table.clamp(min=0, max=3), n, refs)
    out = fbq.attention(cache, 0, torch.randn(2, 2, 64).half().cuda())
    assert (out == 0).all()


def test_sharing_changes_last_bits_only_and_runs_repeat():
    import paper_2501_16385_amd as fbq
    lengths = [160 + 3 * b for b in range(24)]
    pool, table, n, refs = make_cache(lengths, 2, 128, 16, F16, shared_pages=10, seed=4)
    cache = to_cache(fbq, pool, table, n, refs)
    q = torch.randn(24, 8, 128).half().cuda()
    shared = table[3, :10].contiguous().cuda()
    apart, together = fbq.attention(cache, 0, q), fbq.attention(cache, 0, q, shared=shared)
    assert (apart.float() - together.float()).abs().max() <= 4e-3
    for _ in range(3):
        assert torch.equal(fbq.attention(cache, 0, q), apart) and torch.equal(fbq.attention(cache, 0, q, shared=shared), together)


def test_pool_beyond_32_bits_of_bytes():
    """Pages that lie more than 4 GiB into a layer, in the second layer."""
    import paper_2501_16385_amd as fbq
    layers, pages, heads, page, D = 2, 10400, 8, 128, 128      # 524 KiB a page, 5.4 GB a layer
    cache = fbq.cache_create(layers, pages, page, heads, D, 2, 4)
    cache.pool[1, pages - 6:].normal_()
    cache.table[0] = torch.tensor([pages - 1, pages - 3, pages - 6, -1])
    cache.table[1] = torch.tensor([pages - 2, pages - 5, pages - 4, -1])
    cache.lengths.copy_(torch.tensor([384, 300]))
    small = fbq.Cache(cache.pool[1:, pages - 6:].contiguous(), torch.where(cache.table >= 0, cache.table - (pages - 6), -1).int(), cache.lengths,
                      torch.zeros(6, dtype=torch.int32, device="cuda"))
    for counts in ([1, 1], [50, 60]):
        q = torch.randn(sum(counts), heads, D, device="cuda").half()
        qs = None if max(counts) == 1 else starts(counts).cuda()
        assert torch.equal(fbq.attention(cache, 1, q, q_start=qs, max_q=max(counts)), fbq.attention(small, 0, q, q_start=qs, max_q=max(counts)))


def test_other_streams_and_graph_replays():
    import paper_2501_16385_amd as fbq
    lengths = [160 + 13 * b for b in range(6)]
    pool, table, n, refs = make_cache(lengths, 2, 64, 16, F16, shared_pages=8, seed=4, width=24)
    cache = to_cache(fbq, pool, table, n, refs)
    cache.pool.nan_to_num_(0.0)
    shared = table[0, :8].contiguous().cuda()
    q = torch.randn(6, 4, 64).half().cuda()
    out, ws = torch.empty_like(q), fbq.attention_workspace(cache, q, shared=shared)
    want = fbq.attention(cache, 0, q, shared=shared)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fbq.attention(cache, 0, q, shared=shared, out=out, workspace=ws)
    side.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    torch.cuda.synchronize()
    fbq.attention(cache, 0, q, shared=shared, out=out, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fbq.attention(cache, 0, q, shared=shared, out=out, workspace=ws)
    for step in range(4):                                      # lengths change between replays: the work is laid out on the device
        cache.lengths.copy_(torch.tensor([max(0, x - 31 * step) for x in lengths], dtype=torch.int32))
        q.copy_(torch.randn(6, 4, 64).half())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, fbq.attention(cache, 0, q, shared=shared)), step


def test_on_a_stream_that_is_not_the_current_one():
    """Workspace and result of a call's own, on a side stream that is busy: what the current stream allocates meanwhile gets other memory."""
    import paper_2501_16385_amd as fbq
    pool, table, n, refs = make_cache([700, 33, 256], 2, 64, 16, F16, seed=4, width=90)
    cache = to_cache(fbq, pool, table, n, refs)
    q = torch.randn(3, 4, 64).half().cuda()
    want = fbq.attention(cache, 0, q)
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    results = []
    for _ in range(5):
        with torch.cuda.stream(side):
            busy = busy @ busy * 1e-3
        results.append(fbq.attention(cache, 0, q, stream=side))
        for _ in range(20):
            torch.full((1 << 20,), float("nan"), device="cuda")
    torch.cuda.synchronize()
    for got in results:
        assert torch.equal(got, want)


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 3.0])
def test_scales(scale):
    check([100, 33], [1, 1], 4, 2, 64, 16, F16, scale=scale, seed=1, gain=0.5)
    check([100, 33], [60, 33], 4, 2, 64, 16, BF16, scale=scale, seed=2, gain=0.5)


def test_the_compiled_call_and_the_python_one_refuse_the_same():
    import paper_2501_16385_amd as fbq
    pool, table, n, refs = make_cache([40, 100], 2, 64, 16, F16, seed=9)
    cache = to_cache(fbq, pool, table, n, refs)
    q = torch.randn(2, 4, 64).half().cuda()
    ws, out = torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    good = dict(out=out, workspace=ws)
    fbq.attention(cache, 0, q, **good)
    for bad in (dict(out=out[:1]), dict(out=out.float()), dict(lse=torch.empty(2, 4, device="cuda").half()), dict(lse=torch.empty(4, 2, device="cuda")),
                dict(q_start=torch.zeros(2, dtype=torch.int32, device="cuda")), dict(q_start=torch.zeros(3, device="cuda")), dict(shared=torch.zeros(1, device="cuda"))):
        for form in (good, dict()):
            with pytest.raises(ValueError):
                fbq.attention(cache, 0, q, **{**form, **bad})
    for wrong in (q.cpu(), q.float(), q[0], q.transpose(1, 2), q[:, :, :32]):
        with pytest.raises((ValueError, RuntimeError)):
            fbq.attention(cache, 0, wrong, **good)
    for layer, kw in ((1, {}), (-1, {}), (0, dict(max_q=2)), (0, dict(workspace=ws[:8]))):
        with pytest.raises(fbq.FbqError):
            fbq.attention(fbq.Cache(cache.pool, torch.cat([cache.table] * 20, 1).contiguous(), cache.lengths, cache.refs), layer, q, **{**good, **kw})
    k = torch.randn(2, 2, 64).half().cuda()
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    for args in ((k.float(), k, start), (k, k[:1], start), (k, k, start.float()), (k, k, start[:1]), (k[:, :1], k[:, :1], start)):
        with pytest.raises((ValueError, fbq.FbqError)):
            fbq.cache_append(cache, 0, *args)
