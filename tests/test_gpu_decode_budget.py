"""The decode loop over a cache in 4 bits and under a budget: against the same calls made one by one, graph replays against eager steps, and samples of one prompt."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, INTER, RANK, D = 256, 640, 16, 64


def layers_of(n, kv_heads):
    from paper_2501_16385_amd.decode_loop import random_stack
    return random_stack(n, HIDDEN, INTER, RANK, 4, seed=1, kv_hidden=kv_heads * D)


def begun(bits, kv_heads, budget):
    """A cache with three rows' prompts, the weights of their passes, and a stack of single steps over it."""
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.decode_loop import Budget, DecoderStack
    layers = layers_of(2, kv_heads)
    cache = fbq.cache_create(2, 40, 16, kv_heads, D, 3, 12, bits=bits)
    cache.pool.zero_()
    pre = DecoderStack(layers, HIDDEN, INTER, batch=60, cache=cache, counts=[33, 10, 17], budget=Budget(60))
    pre.x.copy_(torch.randn(60, HIDDEN, generator=torch.Generator().manual_seed(3)).half())
    pre.step()
    assert pre.evicted.tolist() == [0, 0]
    stack = DecoderStack(layers, HIDDEN, INTER, batch=3, cache=cache, budget=budget, keep_per_layer_buffers=True)
    stack.weights.copy_(pre.weights)
    stack.x.copy_(pre.x[-3:])
    return stack


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("kv_heads", [4, 2])
def test_a_step_is_its_calls(bits, kv_heads):
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.decode_loop import Budget
    budget = Budget(24, first=3, recent=6, decay=0.9)
    stack, other = begun(bits, kv_heads, budget), begun(bits, kv_heads, budget)
    c, w, one = other.cache, other.weights, torch.ones(3, dtype=torch.int32, device="cuda")
    for rep in range(5):
        stack.step()
        start = fbq.cache_reserve(c, one)
        for li in range(2):
            b = stack.buf[li]
            fbq.cache_append(c, li, b["k"].view(3, kv_heads, D), b["v"].view(3, kv_heads, D), start)
            lse = torch.empty(3, HIDDEN // D, device="cuda")
            a = fbq.attention(c, li, b["q"].view(3, HIDDEN // D, D), lse=lse)
            assert torch.equal(a.view(3, HIDDEN), b["a"])
            fbq.attention_weights(c, li, b["q"].view(3, HIDDEN // D, D), lse, w[li], decay=0.9)
        info = torch.zeros(2, dtype=torch.int32, device="cuda")
        fbq.cache_evict(c, w, torch.full((3,), 24, dtype=torch.int32, device="cuda"), first=3, recent=6, info=info)
        torch.cuda.synchronize()
        assert info.tolist() == stack.evicted.tolist() == [1 if rep < 7 else 2, 0]
        for x, y in ((c.lengths, stack.cache.lengths), (c.table, stack.cache.table), (c.refs, stack.cache.refs), (c.pool, stack.cache.pool), (w, stack.weights)):
            assert torch.equal(x, y), rep
    assert stack.cache.lengths.tolist() == [24, 15, 22]


@pytest.mark.parametrize("bits", [16, 4])
def test_replays_are_eager_steps(bits):
    from paper_2501_16385_amd.decode_loop import Budget
    eager, graphed = (begun(bits, 2, Budget(28, first=2, recent=8)) for _ in range(2))
    graph = graphed.capture()
    eager.step()                                               # as the eager step that capture() makes
    for rep in range(20):
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager.step()
        torch.cuda.synchronize()
        for x, y in ((eager.x, graphed.x), (eager.cache.lengths, graphed.cache.lengths), (eager.cache.table, graphed.cache.table), (eager.weights, graphed.weights)):
            assert torch.equal(x, y), rep
    assert eager.cache.lengths.tolist() == [28, 28, 28]


@pytest.mark.parametrize("bits,keep", [(4, 0), (16, 120), (4, 101), (4, 110)])
def test_samples_of_one_prompt(bits, keep):
    from paper_2501_16385_amd import batch_decode
    prompt, samples, tokens = 100, 4, 12
    x0 = torch.randn(prompt, HIDDEN, generator=torch.Generator().manual_seed(5)).half().cuda()
    record, cache, x = batch_decode.run(layers_of(2, 2), HIDDEN, INTER, D, 2, prompt, samples, tokens, x0=x0, cache_bits=bits, keep=keep)
    n = min(prompt + 2 * tokens, keep or 1 << 20)
    assert record["finite"] and record["pages_lacking"] == 0 and record["rows_not_cut_back"] == 0 and record["lengths"] == [prompt, n, n, 0, 0]
    held = [p for row in cache.table.tolist() for p in row if p >= 0]
    refs = cache.refs.tolist()
    assert all(refs[p] == held.count(p) for p in range(len(refs)))


def test_budgets_that_are_refused():
    from paper_2501_16385_amd import batch_decode
    from paper_2501_16385_amd.decode_loop import Budget, DecoderStack
    with pytest.raises(ValueError, match="budget"):
        DecoderStack(layers_of(1, 4), HIDDEN, INTER, budget=Budget(5))
    with pytest.raises(ValueError, match="keep"):
        batch_decode.run(layers_of(1, 4), HIDDEN, INTER, D, 4, 64, 2, 4, keep=64)
