"""A cache in 4 bits, attention weights and eviction on a stream that is not the current one, which is busy; two captured graphs of them replayed in turn, with eager calls between."""
import pytest
import torch

from cache4_cases import make_cache4, to_cache4
from test_gpu_streams import BusyCurrentStream

pytestmark = pytest.mark.gpu
F16 = torch.float16


def small_cache(seed=4):
    import paper_2501_16385_amd as fbq
    pool, table, n, refs, _ = make_cache4([700, 33, 256], 2, 64, 16, F16, seed=seed, width=90)
    return to_cache4(fbq, pool, table, n, refs, F16, 64)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def same(a, b):
    return all(torch.equal(x, y) for x, y in ((a.pool, b.pool), (a.table, b.table), (a.lengths, b.lengths), (a.refs, b.refs)))


def test_attention_and_what_is_read_back():
    import paper_2501_16385_amd as fbq
    cache, q, side, start = small_cache(), torch.randn(3, 4, 64).half().cuda(), torch.cuda.Stream(), ints(5, 0, 255)
    want, (wk, wv) = fbq.attention(cache, 0, q), fbq.cache_read(cache, 0, 3, start)
    room = fbq.attention_workspace(cache, q).numel()
    for _ in range(3):
        busy = BusyCurrentStream(q.numel() * 2, room, wk.numel() * 4)
        got = fbq.attention(cache, 0, q, stream=side)
        k, v = fbq.cache_read(cache, 0, 3, start, stream=side)
        busy.check(side, got, k, v)
        assert torch.equal(got, want) and torch.equal(k, wk) and torch.equal(v, wv)


def test_append_weights_and_eviction():
    import paper_2501_16385_amd as fbq
    a, b, side = small_cache(), small_cache(), torch.cuda.Stream()
    k, v, q = (torch.randn(3, h, 64).half().cuda() for h in (2, 2, 4))
    start, keep = ints(699, 32, 255), ints(100, -1, 250)
    lse, one = torch.randn(3, 4, device="cuda") + 6, torch.rand(1, 3, 2, 90 * 16, device="cuda")
    other = one.clone()

    def run(cache, weights, stream):
        fbq.cache_append(cache, 0, k, v, start, stream=stream)
        fbq.attention_weights(cache, 0, q, lse, weights[0], stream=stream)
        fbq.cache_evict(cache, weights, keep, first=4, recent=8, stream=stream)

    run(a, one, None)
    room = fbq.cache_evict_workspace(a, one).numel()
    busy = BusyCurrentStream(room)
    run(b, other, side)
    busy.check(side)
    assert torch.equal(one, other) and same(a, b) and a.lengths.tolist() == [100, 33, 250]


def test_two_graphs_and_eager_calls_in_turn():
    """Each with its own cache; the workspaces are the graphs' own, and what an eager call allocates lies elsewhere."""
    import paper_2501_16385_amd as fbq
    caches, q = [small_cache(s) for s in (1, 2, 3)], torch.randn(3, 4, 64).half().cuda()
    weights = [torch.zeros(1, 3, 2, 90 * 16, device="cuda") for _ in range(3)]
    fresh = [(c.pool.clone(), c.table.clone(), c.lengths.clone(), c.refs.clone()) for c in caches]
    keep, k, v, start = ints(130, 33, 77), *(torch.randn(3, 2, 64).half().cuda() for _ in range(2)), ints(9, 9, 9)
    lse, out = [torch.zeros(3, 4, device="cuda") for _ in range(3)], [torch.zeros_like(q) for _ in range(3)]

    def step(i):
        fbq.cache_append(caches[i], 0, k, v, start)
        fbq.attention(caches[i], 0, q, out=out[i], lse=lse[i])
        fbq.attention_weights(caches[i], 0, q, lse[i], weights[i][0], decay=0.5)
        fbq.cache_evict(caches[i], weights[i], keep, first=2, recent=5)

    def again(i):
        for t, f in zip((caches[i].pool, caches[i].table, caches[i].lengths, caches[i].refs), fresh[i]):
            t.copy_(f)
        weights[i].zero_()

    graphs = []
    for i in (0, 1):
        step(i)
        again(i)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(i)
        graphs.append(g)
    for i in (0, 1):
        again(i)
        step(i)
    torch.cuda.synchronize()
    want = [(out[i].clone(), weights[i].clone(), caches[i].pool.clone(), caches[i].table.clone(), caches[i].lengths.clone()) for i in (0, 1)]
    for _ in range(3):
        for i in (0, 1):
            again(i)
            graphs[i].replay()
            again(2)
            step(2)
        torch.cuda.synchronize()
        for i in (0, 1):
            got = (out[i], weights[i], caches[i].pool, caches[i].table, caches[i].lengths)
            assert all(torch.equal(x, y) for x, y in zip(got, want[i]))
