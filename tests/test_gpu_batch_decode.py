"""The decode loop with a cache: attention inside it against the formula in 64 bits on what it really saw, graph replays against eager steps, and a batch of samples of one
prompt - forked, decoded behind shared pages, half of them dropped, the pool compacted - against the same tokens decoded alone."""
import pytest
import torch

from cache_cases import attention64

pytestmark = pytest.mark.gpu

HIDDEN, INTER, RANK, D = 256, 640, 16, 64


def layers_of(n, kv_heads, seed=1):
    from paper_2501_16385_amd.decode_loop import random_stack
    return random_stack(n, HIDDEN, INTER, RANK, 4, seed=seed, kv_hidden=kv_heads * D)


@pytest.mark.parametrize("kv_heads", [4, 2])
@pytest.mark.parametrize("counts", [[1, 1, 1], [40, 1, 7], [0, 3, 90]])
def test_attention_inside_the_loop(kv_heads, counts):
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.decode_loop import DecoderStack
    layers = layers_of(2, kv_heads)
    cache = fbq.cache_create(2, 40, 16, kv_heads, D, 3, 14)
    cache.pool.fill_(float("nan"))
    before = DecoderStack(layers, HIDDEN, INTER, batch=60, cache=cache, counts=[33, 0, 27])
    before.x.normal_()
    before.step()
    stack = DecoderStack(layers, HIDDEN, INTER, keep_per_layer_buffers=True, batch=sum(counts), cache=cache, counts=counts)
    stack.x.normal_()
    stack.step()
    torch.cuda.synchronize()
    assert cache.lengths.tolist() == [33 + counts[0], counts[1], 27 + counts[2]] and int(stack.lacking) == 0
    assert torch.isfinite(stack.x).all()
    for li in range(2):
        b = stack.buf[li]
        q, a = (b[n].view(sum(counts), HIDDEN // D, D).cpu() for n in ("q", "a"))
        want, _, bound, _ = attention64(cache.pool.cpu(), cache.table.cpu(), cache.lengths.cpu(), li, q, counts, D ** -0.5)
        assert ((a.double() - want).abs() <= bound).all(), li
        # the step's own keys are the last that each row holds
        at = 0
        for row, c in enumerate(counts):
            for i in range(c):
                pos = int(cache.lengths[row]) - c + i
                held = cache.pool[li, int(cache.table[row, pos // 16]), :, :, pos % 16]
                assert torch.equal(held[0].reshape(-1), b["k"][at]) and torch.equal(held[1].reshape(-1), b["v"][at])
                at += 1


def test_replays_are_eager_steps():
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.decode_loop import DecoderStack
    layers = layers_of(2, 4)
    stacks = []
    for _ in range(2):
        cache = fbq.cache_create(2, 60, 16, 4, D, 3, 12)
        cache.pool.zero_()
        first = DecoderStack(layers, HIDDEN, INTER, batch=60, cache=cache, counts=[33, 10, 17])
        first.x.copy_(torch.randn(60, HIDDEN, generator=torch.Generator().manual_seed(3)).half())
        first.step()
        stacks.append(DecoderStack(layers, HIDDEN, INTER, batch=3, cache=cache))
        stacks[-1].x.copy_(first.x[-3:])
    eager, graphed = stacks
    graph = graphed.capture()
    eager.step()                                               # as the eager step that capture() makes
    for rep in range(20):                                      # over a page's end
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager.step()
        torch.cuda.synchronize()
        assert torch.equal(eager.x, graphed.x) and torch.equal(eager.cache.lengths, graphed.cache.lengths) and torch.equal(eager.cache.table, graphed.cache.table), rep


@pytest.mark.parametrize("prompt,samples,kv_heads", [(100, 6, 2), (64, 3, 4), (9, 2, 4), (33, 1, 4)])
def test_samples_of_one_prompt(prompt, samples, kv_heads):
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd import batch_decode
    from paper_2501_16385_amd.decode_loop import DecoderStack
    tokens, layers = 12, layers_of(2, kv_heads)
    x0 = torch.randn(prompt, HIDDEN, generator=torch.Generator().manual_seed(5)).half().cuda()
    record, cache, x = batch_decode.run(layers, HIDDEN, INTER, D, kv_heads, prompt, samples, tokens, x0=x0)
    kept = samples // 2 if samples > 1 else 1
    assert record["finite"] and record["pages_lacking"] == 0 and record["fork"] == [0, 0]
    assert record["lengths"] == [prompt] + [prompt + 2 * tokens] * kept + [0] * (samples - kept)
    held = [p for row in cache.table.tolist() for p in row if p >= 0]
    refs = cache.refs.tolist()
    assert all(refs[p] == held.count(p) for p in range(len(refs)))
    # alone, nothing shared: a prompt pass and single steps.  Every linear is within 1e-3 (its own bar) whatever kernel serves it; eight of them a step, and a residual
    # that halves what came before
    alone = fbq.cache_create(2, 40, 16, kv_heads, D, 1, 40)
    pre = DecoderStack(layers, HIDDEN, INTER, batch=prompt, cache=alone, counts=[prompt])
    pre.x.copy_(x0)
    pre.step()
    one = DecoderStack(layers, HIDDEN, INTER, batch=1, cache=alone)
    one.x.copy_(pre.x[-1:])
    for _ in range(2 * tokens):
        one.step()
    torch.cuda.synchronize()
    for row in range(kept):
        assert float((x[row].float() - one.x[0].float()).norm() / one.x[0].float().norm()) <= 2e-2
