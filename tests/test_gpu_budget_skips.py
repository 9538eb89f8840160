"""The decode loop under a budget: rows that a step could not cut back are still told after steps that could, eager and in a graph's replays."""
import pytest
import torch

pytestmark = pytest.mark.gpu

HIDDEN, INTER, D = 256, 640, 64


@pytest.mark.parametrize("graphed", [False, True])
def test_a_row_whose_pages_another_holds_for_a_while(graphed):
    import paper_2501_16385_amd as fbq
    from paper_2501_16385_amd.decode_loop import Budget, DecoderStack, random_stack
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    linears = random_stack(1, HIDDEN, INTER, 16, 4, kv_hidden=HIDDEN)
    cache = fbq.cache_create(1, 16, 16, 4, D, 3, 6)
    cache.pool.zero_()
    pre = DecoderStack(linears, HIDDEN, INTER, batch=60, cache=cache.rows(0, 2), counts=[40, 20], budget=Budget(60))
    pre.x.normal_()
    pre.step()
    assert pre.most_skipped.tolist() == [0]
    stack = DecoderStack(linears, HIDDEN, INTER, batch=2, cache=cache.rows(0, 2), budget=Budget(44, recent=4))
    stack.weights.copy_(pre.weights)
    stack.x.normal_()
    step = stack.capture().replay if graphed else stack.step   # (capture: with a first step)
    for _ in range(3 if graphed else 4):
        step()
    assert stack.evicted.tolist() == [0, 0] and stack.most_skipped.tolist() == [0] and cache.lengths.tolist() == [44, 24, 0]
    fbq.cache_fork(cache, ints(0), ints(2))
    step()
    assert stack.evicted.tolist() == [0, 1] and stack.most_skipped.tolist() == [1] and cache.lengths.tolist() == [45, 25, 44]
    fbq.cache_free(cache, ints(2))
    step()
    assert stack.evicted.tolist() == [1, 0] and stack.most_skipped.tolist() == [1] and cache.lengths.tolist() == [44, 26, 0]


def test_the_record_of_samples_of_one_prompt():
    from paper_2501_16385_amd import batch_decode
    from paper_2501_16385_amd.decode_loop import random_stack
    linears = random_stack(1, HIDDEN, INTER, 16, 4, kv_hidden=HIDDEN)
    whole, _, _ = batch_decode.run(linears, HIDDEN, INTER, D, 4, 40, 4, 6, keep=42)
    assert whole["rows_not_cut_back"] == 0
    # two rows that hold each other's pages for the first steps
    from paper_2501_16385_amd import cache as kv
    held, fork = [], kv.cache_fork

    def fork_and_hold(cache, parent, child, info=None, **how):
        fork(cache, parent, child, info=info, **how)
        held.append(cache)
        cache.refs[cache.table[1, 2]] += 1                     # a holder more of the first sample's last page ...

    free = kv.cache_free

    def free_and_let_go(cache, rows, **how):
        free(cache, rows, **how)
        cache.refs[cache.table[1, 2]] -= 1                     # ... until half of the samples are dropped
    batch_decode.kv.cache_fork, batch_decode.kv.cache_free = fork_and_hold, free_and_let_go
    try:
        record, _, _ = batch_decode.run(linears, HIDDEN, INTER, D, 4, 40, 4, 6, keep=42)
    finally:
        batch_decode.kv.cache_fork, batch_decode.kv.cache_free = fork, free
    assert len(held) == 1 and record["rows_not_cut_back"] == 1 and record["lengths"][:3] == [40, 42, 42]
