"""Every token of a long row counts once, wherever its steps and pieces end: rows of tests/marked_cases.py through attention over caches of 16 and of 4 bits."""
import pytest
import torch

from cache4_cases import BF16, F16
from cache_cases import starts
from marked_cases import kept_as, marks, tolerances, wanted

pytestmark = pytest.mark.gpu


def check(lengths, counts, heads, kv_heads, D, page, dtype, bits, shared=0):
    """The rows' tokens appended from fp32 marks and attended to by queries of zeros; shared: tokens of whole pages that all rows begin with."""
    import paper_2501_16385_amd as fbq
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    rows, own = len(lengths), [n - shared for n in lengths]
    held = [-(-n // page) for n in own]
    cache = fbq.cache_create(1, shared // page + sum(held) + 2, page, kv_heads, D, rows + 1, shared // page + max(held), dtype=dtype, bits=bits)
    cache.pool.fill_(float("nan") if bits == 16 else 0xFF)
    of = marks(max(lengths), D).to(dtype).cuda()
    append = lambda c, v, counts_: fbq.cache_append(c, 0, torch.ones_like(v), v, fbq.cache_reserve(c, ints(counts_)), q_start=starts(counts_).cuda())
    repeated = lambda first, n: of[first:first + n, None].expand(n, kv_heads, D).contiguous()
    if shared:
        append(cache, repeated(0, shared), [0] * rows + [shared])
        fbq.cache_fork(cache, ints([rows] * rows), ints(list(range(rows))))
    part = cache.rows(0, rows)
    for b, n in enumerate(own):                                # (row by row: the marks of one are those of all)
        append(part, repeated(shared, n), [n if x == b else 0 for x in range(rows)])
    assert cache.lengths.tolist()[:rows] == list(lengths)
    T = sum(counts)
    q, lse = torch.zeros(T, heads, D, dtype=dtype, device="cuda"), torch.empty(T, heads, device="cuda")
    pages = cache.table[0, :shared // page].contiguous() if shared else None
    got = fbq.attention(part, 0, q, q_start=None if counts == [1] * rows else starts(counts).cuda(), max_q=max(counts), shared=pages, lse=lse).cpu().double()
    lse, t = lse.cpu().double(), 0
    few = max(counts) * heads // kv_heads <= 16 and not shared
    for n, c in zip(lengths, counts):
        for i in range(c):
            out, of_lse = wanted(n - c + i + 1, D, kept_as(dtype, bits))
            off_out, off_lse = tolerances(out, of_lse, dtype, 1 if few or bits == 16 else 2)
            assert ((got[t] - out).abs() <= off_out).all() and ((lse[t] - of_lse).abs() <= off_lse).all(), (n, i)
            t += 1


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
def test_one_long_row_among_short_ones(D, dtype, bits):
    check([7, 20000, 100], [1] * 3, 2, 1, D, 32, dtype, bits)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("lengths", [[900], [2049], [65537], [9000, 4000, 1, 12345], [16000, 31, 16001, 64], [2500] * 20, [1 + 40 * b for b in range(60)]])
def test_lengths(lengths, bits):
    check(lengths, [1] * len(lengths), 8, 2, 128, 16, F16, bits)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("counts", [[4, 1], [2, 16], [70, 3], [300, 129]])
def test_several_tokens(counts, bits):
    check([5003, 700], counts, 1, 1, 64, 64, F16, bits)
    check([3001, 2100], counts, 4, 2, 128, 16, BF16, bits)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("rows,heads,kv_heads,count,D", [(3, 8, 8, 1, 64), (12, 4, 2, 1, 128), (24, 16, 2, 1, 96), (5, 8, 4, 3, 256), (9, 8, 4, 20, 128)])
def test_shared_tokens(rows, heads, kv_heads, count, D, bits):
    check([8192 + count + 5 * b for b in range(rows)], [count] * rows, heads, kv_heads, D, 64, BF16, bits, shared=8192)
