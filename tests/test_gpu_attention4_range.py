"""Few query rows over a cache in 4 bits at both ends of its type's range: results and attention weights against the formula in 64 bits, element by element within the bounds of
tests/cache4_cases.py, of which only what they grant to results near zero is less here."""
import math

import pytest
import torch

from cache4_cases import BF16, F16, attention4_64, pack, to_cache4, unpack
from cache_cases import make_cache, starts

pytestmark = pytest.mark.gpu

LEAST = {F16: 2.0 ** -24, BF16: 2.0 ** -133}                  # the types' least numbers


def sized(lengths, kv_heads, D, page, dtype, k_size, v_size, seed):
    """(pool, table, lengths, refs, what the pool stands for): normal keys and values times their sizes, none beyond the type's largest."""
    x, table, n, refs = make_cache(lengths, kv_heads, D, page, dtype, seed=seed)
    most = torch.finfo(dtype).max
    for i, size in ((0, k_size), (1, v_size)):
        x[:, :, i] = (x[:, :, i].double() * size).clamp(-most, most).to(dtype)
    pool = pack(x, page)
    return pool, table, n, refs, unpack(pool, dtype, D)


def check(lengths, counts, heads, kv_heads, D, dtype, k_size, v_size, seed=1):
    import paper_2501_16385_amd as fbq
    pool, table, n, refs, values = sized(lengths, kv_heads, D, 16, dtype, k_size, v_size, seed)
    T = sum(counts)
    q = (torch.randn(T, heads, D, generator=torch.Generator().manual_seed(seed + 1)).double() / k_size).to(dtype)
    assert max(counts) * heads // kv_heads <= 16
    # (results go with values' size: worked out at about 1, where the bound's 2^-24 for results near zero can be taken off)
    size = 2.0 ** math.floor(math.log2(v_size))
    values[:, :, 1] /= size
    want, want_lse, bound, lse_bound = attention4_64(values, table, n, 0, q, counts, D ** -0.5, True)
    want, bound = want * size, (bound - 2.0 ** -24) * size + LEAST[dtype]
    lse = torch.empty(T, heads, device="cuda")
    got = fbq.attention(to_cache4(fbq, pool, table, n, refs, dtype, D), 0, q.cuda(), q_start=starts(counts).cuda(), max_q=max(counts), lse=lse)
    got, lse = got.cpu().double(), lse.cpu().double()
    assert torch.isfinite(got).all() and torch.isfinite(lse).all()
    off = (got - want).abs()
    assert (off <= bound).all(), f"{float((off / bound).max()):.2f} times the bound"
    assert ((lse - want_lse).abs() <= lse_bound).all()


@pytest.mark.parametrize("size", [1e32, 5e36, 3e37, 3e38, 1e-29, 1e-33, 1e-36])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_values(D, size):
    check([200, 77], [1, 1], 4, 2, D, BF16, 1.0, size)
    check([200, 77], [4, 3], 4, 2, D, BF16, 1.0, size)


@pytest.mark.parametrize("size", [1e32, 3e38, 1e-36])
def test_values_of_rows_that_are_joined(size):
    """Pieces of a block in LDS, and of many workers by the join kernel."""
    check([900], [1], 2, 1, 64, BF16, 1.0, size)
    check([9000, 33], [1, 1], 2, 1, 64, BF16, 1.0, size)


@pytest.mark.parametrize("size", [1e32, 5e36, 3e38, 1e-30, 1e-35])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_keys(D, size):
    """Queries so much smaller, or larger: with features of 2^110 and more, too."""
    check([200, 77], [1, 1], 4, 2, D, BF16, size, 1.0)


@pytest.mark.parametrize("size", [3e4, 1e-3])
def test_values_and_keys_of_fp16(size):
    check([200, 77], [4, 1], 4, 2, 128, F16, 1.0, size)
    check([200, 77], [1, 1], 4, 2, 128, F16, size, 1.0)


def large_among_new(length, count, heads, D, dtype, size, back):
    """A row's `count` new tokens, the one `back` from the last with values so much larger than the others'.  The tokens before it have the results, bit for bit, that they have without, all keep to the
    formula's bounds.  With more than 16 query rows, where a block's operands of bf16 have the rounding that its largest scales leave them, all keep to that rounding's bounds."""
    import paper_2501_16385_amd as fbq
    kv_heads, few, place = 1, count * heads <= 16, length - 1 - back
    x, table, n, refs = make_cache([length, 20], kv_heads, D, 16, dtype, seed=length)
    q = torch.randn(count + 1, heads, D, generator=torch.Generator().manual_seed(7)).to(dtype)
    results, at = [], (0, int(table[0, place // 16]), 1, 0, place % 16)
    for times in (1.0, size):
        y, most = x.clone(), torch.finfo(dtype).max
        y[at] = (y[at].double() * times).clamp(-most, most).to(dtype)
        pool = pack(y, 16)
        lse = torch.empty(count + 1, heads, device="cuda")
        out = fbq.attention(to_cache4(fbq, pool, table, n, refs, dtype, D), 0, q.cuda(), q_start=starts([count, 1]).cuda(), max_q=count, lse=lse)
        results.append((out, lse))
        want, _, bound, _ = attention4_64(unpack(pool, dtype, D), table, n, 0, q, [count, 1], D ** -0.5, few)
        assert ((out.cpu().double() - want).abs() <= bound).all()
    others = [t for t in range(count + 1) if t < count - 1 - back or t == count] if few else []
    for one, other in zip(*results):
        assert torch.equal(one[others], other[others])


@pytest.mark.parametrize("dtype,size", [(F16, 3e4), (F16, 100.0), (BF16, 1e4), (BF16, 1e30), (BF16, 3e38)])
@pytest.mark.parametrize("length,count,heads", [(90, 4, 4), (40, 8, 2), (600, 3, 10), (64, 16, 1), (33, 2, 4), (9000, 5, 2)])
def test_large_values_that_a_token_does_not_see(length, count, heads, dtype, size):
    large_among_new(length, count, heads, 128, dtype, size, 0)


@pytest.mark.parametrize("dtype,size", [(F16, 1e4), (BF16, 1e4), (BF16, 1e36)])
@pytest.mark.parametrize("D", [64, 96, 192, 256])
def test_large_values_that_some_tokens_see(D, dtype, size):
    large_among_new(70, 7, 2, D, dtype, size, 3)
    large_among_new(2100, 16, 1, D, dtype, size, 15)
    large_among_new(5, 4, 4, D, dtype, size, 1)


@pytest.mark.parametrize("dtype,size", [(F16, 1e4), (BF16, 1e4), (BF16, 1e36)])
@pytest.mark.parametrize("rows,length,count,kv_heads", [(32, 33, 2, 32), (32, 66, 5, 32), (1, 8996, 6, 16), (1, 8995, 6, 16)])
def test_large_values_in_a_step_of_their_own(rows, length, count, kv_heads, dtype, size):
    """New tokens on both sides of a step's end, in waves that have both steps: an item each, or pieces of several steps."""
    import paper_2501_16385_amd as fbq
    D = 64
    x, table, n, refs = make_cache([length] * rows, kv_heads, D, 16, dtype, seed=length)
    q, counts = torch.randn(rows * count, kv_heads, D, generator=torch.Generator().manual_seed(7)).to(dtype), [count] * rows
    last, results = table[:, (length - 1) // 16].long(), []
    for times in (1.0, size):
        y, most = x.clone(), torch.finfo(dtype).max
        y[0, last, 1, :, (length - 1) % 16] = (y[0, last, 1, :, (length - 1) % 16].double() * times).clamp(-most, most).to(dtype)
        pool = pack(y, 16)
        results.append(fbq.attention(to_cache4(fbq, pool, table, n, refs, dtype, D), 0, q.cuda(), q_start=starts(counts).cuda(), max_q=count).cpu())
        want, _, bound, _ = attention4_64(unpack(pool, dtype, D), table, n, 0, q, counts, D ** -0.5, True)
        assert ((results[-1].double() - want).abs() <= bound).all()
    one, other = (r.view(rows, count, kv_heads, D)[:, :-1] for r in results)
    assert torch.equal(one, other)


@pytest.mark.parametrize("dtype,size", [(F16, 1e4), (BF16, 1e4), (BF16, 1e36)])
@pytest.mark.parametrize("D,kv_heads", [(64, 8), (96, 6), (128, 4)])
def test_large_values_behind_shared_tokens(D, kv_heads, dtype, size):
    """The rows' own tokens in one launch with the shared ones, which 80 query rows a head read apart."""
    import paper_2501_16385_amd as fbq
    rows, shared, count, own = 20, 8192, 2, 40
    assert 4 * shared * kv_heads * D * (rows - 1) >= 256 << 20
    lengths, counts = [shared + own + b for b in range(rows)], [count] * rows
    x, table, n, refs = make_cache(lengths, kv_heads, D, 64, dtype, shared_pages=shared // 64, seed=D)
    q = torch.randn(rows * count, 2 * kv_heads, D, generator=torch.Generator().manual_seed(7)).to(dtype)
    results = []
    for times in (1.0, size):
        y, most = x.clone(), torch.finfo(dtype).max
        for b, length in enumerate(lengths):
            at = (0, int(table[b, (length - 1) // 64]), 1, slice(None), (length - 1) % 64)
            y[at] = (y[at].double() * times).clamp(-most, most).to(dtype)
        pool = pack(y, 64)
        cache = to_cache4(fbq, pool, table, n, refs, dtype, D)
        results.append(fbq.attention(cache, 0, q.cuda(), q_start=starts(counts).cuda(), max_q=count, shared=table[0, :shared // 64].contiguous().cuda()).cpu())
    # The result is sum p v over the shared tokens, rounded as many rows' are, and over the rows' own, rounded as few rows' are, in one quotient.  With o = o' + o'' each part is off by no more than its form's
    # bound over all tokens, of which its own are a part: by both in all.  (Of the own ones that is a part of the largest value, also in features where the token that has it holds little: few rows round p s.)
    values = unpack(pool, dtype, D)
    (want, _, many, _), (_, _, few, _) = (attention4_64(values, table, n, 0, q, counts, D ** -0.5, which) for which in (False, True))
    assert ((results[-1].double() - want).abs() <= many + few).all()
    one, other = (r.view(rows, count, -1, D)[:, 0] for r in results)
    assert torch.equal(one, other)


@pytest.mark.parametrize("counts,size", [([n, 1], size) for n in (1, 7) for size in (1e30, 5e36, 3e38, 1e-30)] + [([40, 20], size) for size in (1e30, 1e-30)])
def test_weights(counts, size):
    """Sums of what attention gave each key; beyond 16 query rows a head up to 1e30, where the queries are numbers that the matrix cores take as they are."""
    import paper_2501_16385_amd as fbq
    from test_gpu_eviction import weights64
    D, dtype = 128, BF16
    pool, table, n, refs, values = sized([200, 77], 2, D, 16, dtype, size, 1.0, 3)
    T = sum(counts)
    q = (torch.randn(T, 4, D, generator=torch.Generator().manual_seed(4)).double() / size).to(dtype)
    cache, qs = to_cache4(fbq, pool, table, n, refs, dtype, D), starts(counts).cuda()
    lse = torch.empty(T, 4, device="cuda")
    fbq.attention(cache, 0, q.cuda(), q_start=qs, max_q=max(counts), lse=lse)
    assert torch.isfinite(lse).all()
    out = torch.zeros(2, 2, table.shape[1] * 16)
    want, bound = weights64(values, table, n, 0, q, lse.cpu(), counts, D ** -0.5, None, 1.0, out)
    got = fbq.attention_weights(cache, 0, q.cuda(), lse, None, q_start=qs, max_q=max(counts), out=out.cuda()).cpu().double()
    assert ((got - want).abs() <= bound).all()
