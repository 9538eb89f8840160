"""Attention with as many query tokens and rows as the header allows: more tiles than one dimension of a grid has blocks, and more rows."""
import ctypes
import math

import pytest
import torch

from cache_cases import attention64, make_cache, starts, to_cache

ADDRESS, ODD = 0x10000, 0x10008


@pytest.mark.parametrize("T,heads,kv_heads,rows,max_q,q_start", [(1 << 20, 32, 8, 1, 1 << 20, True), (1 << 20, 32, 32, 1, 7, True), (40000, 4, 2, 40000, 1, False), (65536, 512, 1, 65536, 1, False),
                                                                 (100, 8, 8, 65536, 100, True)])
def test_sizes_of_the_header_are_accepted(T, heads, kv_heads, rows, max_q, q_start):
    """(No launch: the workspace's address is refused last of all.)"""
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.cache import _CAttentionCall, _CCache, _CCacheDesc
    cache = _CCache(_CCacheDesc(1, 100, 16, kv_heads, 64, 0), rows, 40, ADDRESS, ADDRESS, ADDRESS, None)
    stride = heads * 64
    call = lambda T: _CAttentionCall(cache, 0, heads, T, max_q, ADDRESS if q_start else None, ADDRESS, stride, ADDRESS, stride, None, None, 0, 1.0)
    go = lambda T: fbq.load().fbq_attention(ctypes.byref(call(T)), ODD, 1 << 50, None)
    assert go(T) == 4
    if q_start and T * heads == 1 << 25:
        assert go(T + 1) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_prompt_of_more_tiles_than_a_grid_has_in_a_dimension(dtype):
    """Most of its tokens lie before what the row still holds: they see nothing."""
    import paper_2501_16385_amd as fbq
    T, heads, D, held = 1 << 18, 33, 16, 150
    pool, table, n, refs = make_cache([held], 1, D, 16, dtype, seed=2)
    last = torch.randn(held, heads, D, generator=torch.Generator().manual_seed(3)).to(dtype)
    want, want_lse, bound, lse_bound = attention64(pool, table, n, 0, last, [held], 0.25)
    q = torch.randn(T, heads, D, device="cuda", dtype=torch.float32).to(dtype)
    q[T - held:] = last.cuda()
    out, lse = torch.full_like(q, 55.0), torch.full((T, heads), 77.0, device="cuda")
    fbq.attention(to_cache(fbq, pool, table, n, refs), 0, q, q_start=starts([T]).cuda(), max_q=T, scale=0.25, out=out, lse=lse)
    assert (out[:T - held] == 0).all() and (lse[:T - held] == -math.inf).all()
    assert ((out[T - held:].cpu().double() - want).abs() <= bound).all()
    assert ((lse[T - held:].cpu().double() - want_lse).abs() <= lse_bound).all()


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads,width", [(2, 1, 3), (2, 1, 90), (17, 1, 3)])
def test_more_rows_than_a_grid_has_in_a_dimension(heads, kv_heads, width):
    """Single tokens of 65536 rows, most of them empty: an item a wave, one line of steps, a tile a row."""
    import paper_2501_16385_amd as fbq
    rows, D = 65536, 16
    full = list(range(5, rows, 997)) + [rows - 1]
    lengths = [1 + (31 * b) % 45 for b in full]
    pool, small, _, refs = make_cache(lengths, kv_heads, D, 16, torch.float16, seed=4)
    table, n = torch.full((rows, width), -1, dtype=torch.int32), torch.zeros(rows, dtype=torch.int32)
    table[full, :small.shape[1]], n[full] = small, torch.tensor(lengths, dtype=torch.int32)
    q = torch.randn(rows, heads, D, generator=torch.Generator().manual_seed(5)).half()
    want, want_lse, bound, lse_bound = attention64(pool, small, lengths, 0, q[full], [1] * len(full), 0.25)
    lse = torch.full((rows, heads), 77.0, device="cuda")
    got = fbq.attention(to_cache(fbq, pool, table, n, refs), 0, q.cuda(), scale=0.25, lse=lse).cpu()
    lse = lse.cpu()
    assert ((got[full].double() - want).abs() <= bound).all() and ((lse[full].double() - want_lse).abs() <= lse_bound).all()
    empty = torch.ones(rows, dtype=torch.bool)
    empty[full] = False
    assert (got[empty] == 0).all() and (lse[empty] == -math.inf).all()


@pytest.mark.gpu
def test_shared_tokens_for_more_tiles_than_a_grid_has_in_a_dimension():
    """Nine rows of a token each, among many tokens of no row, behind shared pages that are read apart."""
    import paper_2501_16385_amd as fbq
    T, rows, heads, D, page, pages, first = 1 << 18, 9, 33, 64, 256, 192, (1 << 18) - 2000
    lengths = [page * pages + 1 + 5 * b for b in range(rows)]
    lengths[4] = page * pages // 2
    pool, table, n, refs = make_cache(lengths, 1, D, page, torch.float16, shared_pages=pages, seed=6)
    mine = torch.randn(rows, heads, D, generator=torch.Generator().manual_seed(7)).half()
    want, want_lse, bound, lse_bound = attention64(pool, table, n, 0, mine, [1] * rows, 0.125)
    q = torch.zeros(T, heads, D, dtype=torch.float16, device="cuda")
    q[first:first + rows] = mine.cuda()
    cache, edges, shared = to_cache(fbq, pool, table, n, refs), (starts([1] * rows) + first).cuda(), table[0, :pages].contiguous().cuda()
    size = lambda s: fbq.attention_workspace(cache, q, q_start=edges, max_q=1, shared=s).numel()
    assert size(shared) != size(None)
    out, lse = torch.full_like(q, 55.0), torch.full((T, heads), 77.0, device="cuda")
    fbq.attention(cache, 0, q, q_start=edges, max_q=1, shared=shared, scale=0.125, out=out, lse=lse)
    assert (out[:first] == 55).all() and (out[first + rows:] == 55).all() and (lse[:first] == 77).all() and (lse[first + rows:] == 77).all()
    assert ((out[first:first + rows].cpu().double() - want).abs() <= bound).all()
    assert ((lse[first:first + rows].cpu().double() - want_lse).abs() <= lse_bound).all()
