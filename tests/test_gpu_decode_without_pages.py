"""The decode loop over a cache that runs short for some steps: what was left out is still told after steps that fit, eager and in a graph's replays."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, INTER, D = 256, 640, 64


def stack_of(pages, width, counts):
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.decode_loop import DecoderStack, random_stack
    layers = random_stack(1, HIDDEN, INTER, 16, 4, kv_hidden=HIDDEN)
    cache = fbq.cache_create(1, pages, 16, 4, D, len(counts), width)
    cache.pool.zero_()
    before = DecoderStack(layers, HIDDEN, INTER, batch=sum(counts), cache=cache, counts=counts)
    before.x.normal_()
    before.step()
    assert before.lowest_start.tolist() == [0] * len(counts) and before.most_lacking.tolist() == [0]
    stack = DecoderStack(layers, HIDDEN, INTER, batch=len(counts), cache=cache)
    stack.x.normal_()
    return stack


@pytest.mark.parametrize("graphed", [False, True])
def test_a_pool_that_runs_short_and_has_room_again(graphed):
    import paper_2501_16385_amd as fbq
    stack = stack_of(5, 4, [30, 30, 1])                        # two, two and one of five pages
    step = stack.step
    if graphed:
        step = stack.capture().replay                          # (with a first step)
    else:
        step()
    step()
    assert stack.lowest_start.tolist() == [0, 0, 0] and stack.most_lacking.tolist() == [0]
    step()                                                     # two rows are full
    assert stack.lacking.tolist() == [2] and stack.start.tolist() == [-1, -1, 3]
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    fbq.cache_free(stack.cache, ints(0))
    stack.count.copy_(ints(0, 1, 1))
    for _ in range(3):
        step()
    assert stack.lacking.tolist() == [0] and stack.cache.lengths.tolist() == [0, 35, 7]
    assert stack.most_lacking.tolist() == [2] and [x < 0 for x in stack.lowest_start.tolist()] == [True, True, False]


def test_a_table_that_is_too_narrow():
    """No page is lacking, and the row is left out all the same."""
    stack = stack_of(9, 2, [31, 5])
    stack.step()
    assert stack.lowest_start.tolist() == [0, 0]
    stack.step()
    assert stack.start.tolist() == [-1, 6] and stack.lacking.tolist() == [0] and stack.lowest_start.tolist() == [-1, 0]
    stack.count[0] = 0
    stack.step()
    assert stack.start.tolist() == [32, 7] and stack.lowest_start.tolist() == [-1, 0] and stack.cache.lengths.tolist() == [32, 8]


def test_the_record_of_samples_of_one_prompt():
    from paper_2501_16385_amd import batch_decode
    from paper_2501_16385_amd.decode_loop import random_stack
    record, _, _ = batch_decode.run(random_stack(1, HIDDEN, INTER, 16, 4, kv_hidden=HIDDEN), HIDDEN, INTER, D, 4, 40, 4, 6)
    assert record["pages_lacking"] == 0 and record["rows_left_out"] == []
