"""The decode loop under a budget with rows that a step leaves out - no pages for them, or nothing to append: their attention weights are as they were, bit for bit, and go on when they do."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, INTER, D = 256, 640, 64


def begun(pages, width, counts, step_counts, bits, kv_heads=2, layers=2):
    """A stack of steps over rows that hold `counts` tokens, with the weights of their prompts."""
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.decode_loop import Budget, DecoderStack, random_stack
    linears = random_stack(layers, HIDDEN, INTER, 16, 4, seed=1, kv_hidden=kv_heads * D)
    cache = fbq.cache_create(layers, pages, 16, kv_heads, D, len(counts), width, bits=bits)
    cache.pool.zero_()
    pre = DecoderStack(linears, HIDDEN, INTER, batch=sum(counts), cache=cache, counts=counts, budget=Budget(1 << 16))
    g = torch.Generator().manual_seed(3)
    pre.x.copy_(torch.randn(sum(counts), HIDDEN, generator=g).half())
    pre.step()
    assert (pre.weights[:, :, :, 0] > 0).all()
    stack = DecoderStack(linears, HIDDEN, INTER, batch=sum(step_counts), cache=cache, counts=step_counts, budget=Budget(1 << 16, decay=0.5))
    stack.weights.copy_(pre.weights)
    stack.x.copy_(torch.randn(sum(step_counts), HIDDEN, generator=g).half())
    return stack


def changed(stack, step, expect):
    """One step; the rows of `expect` alone have other weights after it."""
    before = stack.weights.clone()
    step()
    torch.cuda.synchronize()
    assert torch.isfinite(stack.weights).all()
    assert [not torch.equal(stack.weights[:, b], before[:, b]) for b in range(before.shape[1])] == expect


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("graphed", [False, True])
def test_rows_that_no_pages_are_left_for(graphed, bits):
    import paper_2501_16385_amd as fbq
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    stack = begun(5, 4, [30, 30, 1], [1, 1, 1], bits)          # two, two and one of five pages
    step = stack.capture().replay if graphed else stack.step   # (capture: with a first step)
    if not graphed:
        changed(stack, step, [True] * 3)
    changed(stack, step, [True] * 3)
    changed(stack, step, [False, False, True])                 # two rows are full
    assert stack.start.tolist() == [-1, -1, 3]
    changed(stack, step, [False, False, True])
    fbq.cache_free(stack.cache, ints(0))
    stack.count.copy_(ints(0, 1, 1))
    changed(stack, step, [False, True, True])                  # room again for one; an empty row
    stack.count.copy_(ints(0, 0, 1))
    changed(stack, step, [False, False, True])                 # nothing for a row that holds tokens
    assert stack.cache.lengths.tolist() == [0, 33, 7]
    stack.count.copy_(ints(0, 1, 1))
    changed(stack, step, [False, True, True])


@pytest.mark.parametrize("bits", [16, 4])
def test_rows_of_several_tokens(bits):
    """More than 16 query rows a head, too; a table that is too narrow for a row."""
    stack = begun(12, 3, [30, 42, 3], [3, 12, 1], bits)
    changed(stack, stack.step, [True, False, True])
    assert stack.start.tolist() == [30, -1, 3]
    changed(stack, stack.step, [True, False, True])
    assert stack.cache.lengths.tolist() == [36, 42, 5]
