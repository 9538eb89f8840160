"""A cache in 4 bits, weights and workspaces beyond 4 GiB: the same calls on a row in a large pool's last pages, and in a small one's, give equal bits."""
import pytest
import torch

from cache4_cases import BF16, F16
from cache_cases import starts

pytestmark = pytest.mark.gpu


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,bits", [(F16, 4), (BF16, 4), (F16, 16)])
def test_pages_beyond_4_gib(dtype, bits):
    import paper_2501_16385_amd as fbq
    D, kv_heads, heads, page, n = 128, 32, 64, 256, 600
    page_bytes = 2 * kv_heads * page * (72 if bits == 4 else 256)
    pages = (5 << 30) // page_bytes + 9
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(n, kv_heads, D, generator=g).to(dtype).cuda() for _ in range(2))
    many = torch.randn(40, heads, D, generator=g).to(dtype).cuda()
    weights = torch.rand(1, 1, kv_heads, 3 * page, generator=g).cuda()
    seen = []
    for total, own in ((pages, [pages - 1, pages - 4, pages - 2]), (4, [3, 0, 2])):
        c = fbq.cache_create(1, total, page, kv_heads, D, 1, 3, dtype=dtype, bits=bits)
        c.table.copy_(ints(own))
        c.lengths.fill_(n)
        c.refs[torch.tensor(own, device="cuda")] = 1
        fbq.cache_append(c, 0, k, v, ints(0), q_start=ints(0, n))
        out = list(fbq.cache_read(c, 0, n, ints(0), q_start=ints(0, n)))
        for q in (many[:1], many[:5], many):
            qs = ints(0, q.shape[0])
            lse = torch.empty(q.shape[:2], device="cuda")
            out.append(fbq.attention(c, 0, q, q_start=qs, max_q=q.shape[0], lse=lse))
            out += [lse, fbq.attention_weights(c, 0, q, lse, None, q_start=qs, max_q=q.shape[0], out=torch.zeros_like(weights[0]))]
        info, w = ints(0, 0), weights.clone()
        fbq.cache_evict(c, w, ints(333), first=10, recent=20, info=info)
        assert info.tolist() == [1, 0] and c.lengths.tolist() == [333]
        out += [w, *fbq.cache_read(c, 0, 333, ints(0), q_start=ints(0, 333))]
        seen.append(out)
        del c
    for a, b in zip(*seen):
        assert torch.equal(a, b)


def test_weights_beyond_8_gib():
    """Layers, rows and heads times a width that pass 2^31: the last row's, in the last layer."""
    import paper_2501_16385_amd as fbq
    D, kv_heads, page, rows, layers, width, n = 64, 8, 16, 66, 4, 1 << 20, 50
    c = fbq.cache_create(layers, 8, page, kv_heads, D, rows, 4)
    small = fbq.cache_create(layers, 8, page, kv_heads, D, 1, 4)
    g = torch.Generator().manual_seed(1)
    counts = [0] * (rows - 1) + [n]
    start = fbq.cache_reserve(c, ints(*counts))
    start_small = fbq.cache_reserve(small, ints(n))
    w, w_small = torch.zeros(layers, rows, kv_heads, width, device="cuda"), torch.zeros(layers, 1, kv_heads, 64, device="cuda")
    assert w.numel() > 1 << 31
    q, lse = torch.randn(rows, 16, D, generator=g).half().cuda(), torch.empty(rows, 16, device="cuda")
    for layer in range(layers):
        k, v = (torch.randn(n, kv_heads, D, generator=g).half().cuda() for _ in range(2))
        fbq.cache_append(c, layer, k, v, start, q_start=starts(counts).cuda())
        fbq.cache_append(small, layer, k, v, start_small, q_start=ints(0, n))
        fbq.attention(c, layer, q, lse=lse)
        fbq.attention_weights(c, layer, q, lse, None, out=w[layer])
        one = lse[-1:].clone()
        fbq.attention(small, layer, q[-1:], lse=one)
        fbq.attention_weights(small, layer, q[-1:], one, None, out=w_small[layer])
    assert torch.equal(w[:, -1:, :, :64], w_small)
    fbq.cache_evict(c, w, ints(*([-1] * (rows - 1)), 20), first=1, recent=2)
    fbq.cache_evict(small, w_small, ints(20), first=1, recent=2)
    assert c.lengths.tolist() == [0] * (rows - 1) + [20] and torch.equal(w[:, -1:, :, :64], w_small)
    for layer in range(layers):
        a, b = fbq.cache_read(c, layer, 20, ints(*([-1] * (rows - 1)), 0), q_start=starts([0] * (rows - 1) + [20]).cuda()), fbq.cache_read(small, layer, 20, ints(0), q_start=ints(0, 20))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
