"""Calls whose shared tokens are really read apart - in the few-row kernel's line, beside it, in front of it, and as many rows twice - on repeats, other streams and in replayed graphs, and
the join of very many rows.  (Whether they are is asked of the size of the workspace: it is another without.)"""
import pytest
import torch

from cache_cases import attention64, make_cache, starts, to_cache
from test_gpu_attention import check, taken_apart

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16

# rows, heads, kv_heads, D, page, shared pages, most tokens a row
LINE, BESIDE, FRONT, TWICE = (5, 3, 1, 128, 64, 70, 1), (33, 4, 4, 128, 16, 90, 1), (20, 4, 2, 256, 16, 80, 1), (12, 4, 2, 64, 16, 500, 12)


def shape(rows, heads, kv_heads, D, page, pages, most, dtype=F16, seed=4):
    """(cache, queries, arguments of the call, lengths, counts, host tensors)"""
    import paper_2501_16385_amd as fbq
    counts = [1 + (5 * b) % most for b in range(rows)]
    lengths = [page * pages + c + (37 * b) % 90 for b, c in enumerate(counts)]
    lengths[1] = page * pages // 2 + 3 + counts[1]                      # a row that ends inside the shared pages
    pool, table, n, refs = make_cache(lengths, kv_heads, D, page, dtype, shared_pages=pages, seed=seed)
    assert taken_apart(rows, table.shape[1] * page, kv_heads, heads, D, page, pages, most, dtype)
    q = torch.randn(sum(counts), heads, D, generator=torch.Generator().manual_seed(seed + 1)).to(dtype)
    kw = dict(q_start=starts(counts).cuda() if most > 1 else None, max_q=most, shared=table[0, :pages].contiguous().cuda())
    return to_cache(fbq, pool, table, n, refs), q.cuda(), kw, lengths, counts, (pool, table, n, q)


def within_bounds(out, host, counts):
    pool, table, n, q = host
    want, _, bound, _ = attention64(pool, table, n, 0, q, counts, q.shape[2] ** -0.5)
    assert ((out.cpu().double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("what", [LINE, BESIDE, FRONT, TWICE])
def test_calls_repeat(what, dtype):
    import paper_2501_16385_amd as fbq
    cache, q, kw, _, counts, host = shape(*what, dtype)
    first, without = fbq.attention(cache, 0, q, **kw), fbq.attention(cache, 0, q, **{**kw, "shared": None})
    within_bounds(first, host, counts)
    within_bounds(without, host, counts)
    for _ in range(5):
        assert torch.equal(fbq.attention(cache, 0, q, **kw), first)


@pytest.mark.parametrize("what", [LINE, BESIDE, FRONT, TWICE])
def test_other_streams(what):
    import paper_2501_16385_amd as fbq
    cache, q, kw, *_ = shape(*what)
    want, side = fbq.attention(cache, 0, q, **kw), torch.cuda.Stream()
    out, ws = torch.empty_like(q), fbq.attention_workspace(cache, q, q_start=kw["q_start"], max_q=kw["max_q"], shared=kw["shared"])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        fbq.attention(cache, 0, q, out=out, workspace=ws, **kw)
    side.synchronize()
    assert torch.equal(out, want)
    out.zero_()
    torch.cuda.synchronize()
    fbq.attention(cache, 0, q, out=out, workspace=ws, stream=side, **kw)
    got = [fbq.attention(cache, 0, q, stream=side, **kw) for _ in range(3)]
    side.synchronize()
    assert torch.equal(out, want) and all(torch.equal(g, want) for g in got)


@pytest.mark.parametrize("what", [LINE, BESIDE, FRONT, TWICE])
def test_replays_of_a_graph_with_other_lengths(what):
    import paper_2501_16385_amd as fbq
    cache, q, kw, lengths, counts, (pool, table, n, _) = shape(*what)
    cache.pool.nan_to_num_(0.0)
    pool = pool.nan_to_num(0.0)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    ws = fbq.attention_workspace(cache, q, q_start=kw["q_start"], max_q=kw["max_q"], shared=kw["shared"])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    fbq.attention(cache, 0, q, out=out, lse=lse, workspace=ws, **kw)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        fbq.attention(cache, 0, q, out=out, lse=lse, workspace=ws, **kw)
    shared = kw["shared"].numel() * cache.page_size
    for step in range(4):
        now = [max(0, x - 29 * step - (shared - 7 if b == step + 2 else 0)) for b, x in enumerate(lengths)]     # one row nearly empties, rows fall below the shared tokens
        host_q = torch.randn(q.shape, generator=torch.Generator().manual_seed(step)).half()
        cache.lengths.copy_(torch.tensor(now, dtype=torch.int32))
        q.copy_(host_q)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager_lse = torch.empty_like(lse)
        assert torch.equal(out, fbq.attention(cache, 0, q, lse=eager_lse, **kw)) and torch.equal(lse, eager_lse), step
        within_bounds(out, (pool, table, torch.tensor(now, dtype=torch.int32), host_q), counts)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128, 200])
@pytest.mark.parametrize("shared_pages", [0, 34])
def test_join_of_very_many_rows(D, shared_pages, dtype):
    """A wave joins a row: some rows are cut over whole blocks of waves, some lie within one piece, some hold nothing."""
    lengths = [(1500 if b % 16 == 3 else 1290 + b if b % 16 == 9 else (23 * b) % 70 + (16 * shared_pages if b % 5 else 0)) * (b % 7 != 6) for b in range(64)]
    if shared_pages:
        assert taken_apart(64, 1536, 8, 32, D, 16, shared_pages, 1, dtype)
    check(lengths, [1] * 64, 32, 8, D, 16, dtype, shared_pages=shared_pages, seed=D, width=96)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_join_of_very_many_rows_in_one_line_with_the_shared_tokens(dtype):
    assert taken_apart(4, 1200, 128, 512, 16, 16, 40, 1, dtype)
    check([1100, 640, 300, 655], [1] * 4, 512, 128, 16, 16, dtype, shared_pages=40, seed=2, width=75)


def test_join_of_very_many_rows_for_several_tokens_a_row():
    counts = [1 + b % 4 for b in range(40)]
    check([max(c, (97 * b) % 1400) for b, c in enumerate(counts)], counts, 32, 8, 64, 16, F16, seed=3, width=90)


def test_samples_behind_a_prompt_that_is_read_apart():
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd import batch_decode
    from paper_2501_16385_amd.decode_loop import DecoderStack, random_stack
    hidden, inter, D, prompt, samples, tokens = 256, 640, 64, 1100, 6, 10
    layers = random_stack(2, hidden, inter, 16, 4, kv_hidden=hidden)
    x0 = torch.randn(prompt, hidden, generator=torch.Generator().manual_seed(5)).half().cuda()
    record, cache, x = batch_decode.run(layers, hidden, inter, D, 4, prompt, samples, tokens, x0=x0)
    assert taken_apart(samples, cache.table.shape[1] * 16, 4, 4, D, 16, prompt // 16, 1, F16)
    assert record["finite"] and record["pages_lacking"] == 0 and record["rows_left_out"] == [] and record["fork"] == [0, 0]
    assert record["lengths"] == [prompt] + [prompt + 2 * tokens] * 3 + [0] * 3
    # one sample alone, nothing shared: within what eight linears of 1e-3 each a step may differ by
    alone = fbq.cache_create(2, 80, 16, 4, D, 1, 80)
    pre = DecoderStack(layers, hidden, inter, batch=prompt, cache=alone, counts=[prompt])
    pre.x.copy_(x0)
    pre.step()
    one = DecoderStack(layers, hidden, inter, batch=1, cache=alone)
    one.x.copy_(pre.x[-1:])
    for _ in range(2 * tokens):
        one.step()
    torch.cuda.synchronize()
    for row in range(3):
        assert float((x[row].float() - one.x[0].float()).norm() / one.x[0].float().norm()) <= 2e-2
