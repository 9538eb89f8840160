"""What a query token does not see does not reach it, whatever it is: keys and values of later tokens of the same call, and shared tokens behind the end of a short row, hold infinities
and NaN here.  Against the formula in 64 bits (tests/cache_cases.py): finite where that is, within its bound; not finite where a token sees them."""
import math

import pytest
import torch

from cache_cases import attention64, make_cache, starts, to_cache

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
NAN, INF = float("nan"), float("inf")


def poison(pool, table, b, j, kind):
    """Token j of row b: some features of its values, or its keys."""
    page, D = pool.shape[4], pool.shape[5]
    at = pool[:, table[b, j // page], :, :, j % page]                    # [layers, 2, kv_heads, D]
    if kind == "keys":
        at[:, 0, :, D // 3] = NAN
    else:
        at[:, 1, :, 1], at[:, 1, :, D // 2], at[:, 1, :, D - 1] = NAN, INF, -INF


def check(lengths, counts, heads, kv_heads, D, page, dtype, where, kind="values", shared_pages=0, seed=0, width=None, single=False):
    """where: (row, token) that are poisoned."""
    import paper_2501_16385_amd as fbq
    pool, table, n, refs = make_cache(lengths, kv_heads, D, page, dtype, shared_pages, seed=seed, width=width)
    for b, j in where:
        assert 0 <= j < max(lengths[b], shared_pages * page)
        poison(pool, table, b, j, kind)
    T = sum(counts)
    q = torch.randn(T, heads, D, generator=torch.Generator().manual_seed(seed + 1)).to(dtype)
    want, want_lse, bound, lse_bound = attention64(pool, table, n, 0, q, counts, D ** -0.5)
    cache, edges = to_cache(fbq, pool, table, n, refs), None if single else starts(counts).cuda()
    shared = table[0, :shared_pages].contiguous().cuda() if shared_pages else None
    kw = dict(q_start=edges, max_q=max(counts))
    if shared_pages:                                                     # (the shared tokens are really read apart)
        size = lambda s: fbq.attention_workspace(cache, q.cuda(), shared=s, **kw).numel()
        assert size(shared) != size(None)
    lse = torch.empty(T, heads, device="cuda")
    got = fbq.attention(cache, 0, q.cuda(), shared=shared, lse=lse, **kw).cpu().double()
    lse, ok = lse.cpu().double(), torch.isfinite(want)
    assert ok.any() and not ok.all()
    assert torch.isfinite(got[ok]).all(), f"{int((~torch.isfinite(got[ok])).sum())} of {int(ok.sum())} that see no such token are not finite"
    assert ((got - want).abs()[ok] <= bound[ok]).all()
    assert not torch.isfinite(got[~ok]).any()
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
    finite = torch.isfinite(want_lse)
    assert ((lse - want_lse).abs()[finite] <= lse_bound[finite]).all() and torch.isnan(lse[torch.isnan(want_lse)]).all()


def late(lengths, counts):
    """For every row with several new tokens: its last one, and one in the middle of them."""
    return [(b, n - 1 - k) for b, (n, c) in enumerate(zip(lengths, counts)) if c > 1 and n > 1 for k in {0, c // 2} if n - 1 - k >= max(1, n - c)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("kind", ["values", "keys"])
@pytest.mark.parametrize("lengths,counts,heads,kv_heads,D,width", [
    ([120, 40, 9, 333], [5, 1, 3, 4], 4, 4, 64, None), ([120, 40, 9, 333], [16, 2, 9, 1], 2, 2, 128, None), ([120, 40, 9, 100], [2, 1, 3, 4], 4, 1, 200, None),   # an item a block
    ([(7 * b) % 200 + 3 for b in range(300)], [b % 4 for b in range(300)], 4, 4, 16, 16),                                                                     # an item a wave
    ([3000, 40, 2000], [4, 2, 3], 8, 4, 128, None), ([3000, 40, 2000, 33], [5, 2, 3, 4], 3, 1, 40, None), ([1500, 40, 2000], [4, 2, 3], 4, 2, 256, None),       # pieces of one line
])
def test_later_tokens_few_rows(lengths, counts, heads, kv_heads, D, width, kind, dtype):
    check(lengths, counts, heads, kv_heads, D, 16, dtype, late(lengths, counts), kind, seed=D, width=width)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("kind", ["values", "keys"])
@pytest.mark.parametrize("lengths,counts,heads,kv_heads,D", [
    ([150, 64, 1, 129], [150, 30, 1, 129], 4, 2, 64), ([150, 64, 1, 129], [150, 30, 1, 129], 4, 2, 80), ([150, 64, 1, 129], [150, 30, 1, 129], 2, 2, 128),
    ([150, 64, 1, 129], [150, 30, 1, 129], 2, 1, 256), ([70, 200], [7, 3], 40, 1, 64), ([300], [250], 1, 1, 16),
    ([2000], [90], 4, 4, 128), ([900, 30], [40, 2], 8, 2, 96)])                                                                                               # keys cut into pieces
def test_later_tokens_many_rows(lengths, counts, heads, kv_heads, D, kind, dtype):
    check(lengths, counts, heads, kv_heads, D, 16, dtype, late(lengths, counts), kind, seed=D)


def test_every_token_of_a_prompt_poisoned_from_the_middle_on():
    lengths, counts = [200], [200]
    check(lengths, counts, 2, 2, 64, 32, F16, [(0, j) for j in range(77, 200)], seed=1)
    check(lengths, counts, 4, 1, 128, 16, BF16, [(0, j) for j in range(130, 200, 2)], seed=2)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("kind", ["values", "keys"])
@pytest.mark.parametrize("rows,heads,kv_heads,D,page,pages,most", [
    (9, 2, 2, 64, 16, 300, 3), (4, 4, 1, 128, 32, 100, 4), (3, 4, 1, 256, 32, 90, 1),                           # in the few-row kernel's line
    (20, 4, 4, 64, 16, 130, 1), (24, 16, 1, 96, 64, 40, 1), (33, 4, 4, 128, 16, 90, 1),                         # beside it
    (20, 4, 2, 256, 16, 80, 1),                                                                                # in front of it
    (12, 4, 2, 64, 16, 500, 12), (10, 8, 1, 128, 64, 130, 4), (8, 4, 4, 256, 32, 100, 30)])                    # many rows, twice
def test_shared_tokens_behind_a_short_row(rows, heads, kv_heads, D, page, pages, most, kind, dtype):
    counts = [1 + (5 * b) % most for b in range(rows)]
    lengths = [page * pages + c + (11 * b) % 60 for b, c in enumerate(counts)]
    lengths[1], lengths[2] = page * pages // 2 + 3, page * pages - counts[2] - 9                # two rows that end inside the shared pages
    # tokens that the short rows do not see: right behind the first one's end, and in the last shared page
    where = [(0, lengths[1]), (0, page * pages - 2)]
    check(lengths, counts, heads, kv_heads, D, page, dtype, where, kind, shared_pages=pages, seed=rows, single=most == 1)
